"""The kernels that linear's launch has (launch_products in csrc/linear_kernels.hip) are those that its cut into workgroups asks for: none
that no call reaches, none asked for that is not there."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
BF16, Q8, MX = range(3)


def test_every_kernel_is_reached_and_no_other(tmp_path):
    exe = str(tmp_path / "reach")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", os.path.join(HERE, "host", "linear_plan_reach.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300, check=True).stdout
    asked = {tuple(int(v) for v in line.split()) for line in out.splitlines()}
    direct = {(kind, 0, nt, 1) for kind in (BF16, Q8, MX) for nt in (1, 2, 4)} | {(kind, 0, 4, 2) for kind in (Q8, MX)}
    tiled = {(kind, 1, nt, mt) for kind in (BF16, Q8, MX) for nt, mt in ((16, 16), (16, 4), (8, 4))} | {(MX, 1, 16, 8)}
    assert asked == direct | tiled, (asked ^ (direct | tiled))
    # what only some kinds have stands behind a condition of the compiler's
    with open(os.path.join(HERE, "..", "paper_2605_08565_amd", "csrc", "linear_kernels.hip")) as f:
        text = f.read().split("hipError_t launch_products")[1].split("hipError_t launch_by_block")[0]
    assert "if constexpr (XT != kXBf16)" in text.split("launch_direct<XT, SB, 4, 2, 1>")[0].split("launch_tiled")[-1]
    assert "if constexpr (!kWide)" in text.split("launch_tiled<XT, SB, 4, 2, 4, 4, 3>")[0]
