"""Projections of rows that lie far apart, as the last tokens of long prompts do: how many go together, and that they are right."""
import os
import subprocess

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))


def test_rows_of_a_launch(tmp_path):
    exe = str(tmp_path / "rows")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", os.path.join(HERE, "host", "linear_rows_check.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "bad=0" in res.stdout, res.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 2, 16, 17, 40])
@pytest.mark.parametrize("ld", [(1 << 22) - 8, 1 << 22, (1 << 26) - 8, 1 << 26])
def test_rows_far_apart(m, ld):
    """The same bits as from rows side by side, 16 at a time (offsets up to 2 GiB at the third stride), with adapters."""
    from paper_2605_08565_amd import layers
    if m > 17 and ld > 1 << 25:
        m = 18                                            # 2.4 GB of rows
    gen = torch.Generator(device="cuda")
    gen.manual_seed(m)
    k, n = 512, 100
    store = torch.empty((m - 1) * ld + 4096, device="cuda", dtype=torch.bfloat16)
    x = store.as_strided((m, k), (ld, 1), 16)
    x.copy_(torch.randint(-4, 5, (m, k), generator=gen, device="cuda"))
    codes = torch.randint(0, 256, (n, k // 2), generator=gen, device="cuda").to(torch.uint8)
    scales = (torch.randint(6, 10, (n, k // 16), generator=gen, device="cuda") * 8).to(torch.uint8)
    ad = layers.Adapters(torch.randint(-1, 2, (3, 16, k), generator=gen, device="cuda").bfloat16(),
                         torch.randint(-1, 2, (3, n, 16), generator=gen, device="cuda").bfloat16(), torch.ones(3, device="cuda"))
    ids = (torch.arange(m, device="cuda") % 4).int()
    w = layers.W4(codes, scales, 16, 1)
    for args in ((), (ad, ids)):
        got = layers.linear(x, w, *args, out_dtype=torch.float32)
        assert torch.equal(got, layers.linear(x.contiguous(), w, *args, out_dtype=torch.float32))      # exact sums: any order
