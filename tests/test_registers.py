"""The layer operators' kernels keep what they work on in registers: none needs scratch memory, by what the compiler says of them."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_08565_amd import build

KERNELS = ["norm_kernels.hip", "swiglu_kernels.hip", "linear_kernels.hip"]


def usage(name):
    """{kernel: (bytes of scratch a lane, spilled vector registers)}"""
    flags = [f for f in build.FLAGS if f != "-Wall"]
    res = subprocess.run(["hipcc", *flags, "-Rpass-analysis=kernel-resource-usage", "--cuda-device-only", "-c", os.path.join(build.CSRC, name),
                          "-o", os.devnull], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-2000:]
    found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+).*?VGPRs Spill: (\d+)", res.stderr, re.S)
    return {kernel: (int(scratch), int(spilled)) for kernel, scratch, spilled in found}


@pytest.mark.skipif(not any(os.access(os.path.join(p, "hipcc"), os.X_OK) for p in os.environ["PATH"].split(os.pathsep)), reason="needs hipcc")
def test_no_kernel_needs_scratch():
    with ThreadPoolExecutor(3) as pool:
        for name, kernels in zip(KERNELS, pool.map(usage, KERNELS)):
            assert len(kernels) >= 4, (name, kernels)
            assert all(v == (0, 0) for v in kernels.values()), (name, {k: v for k, v in kernels.items() if v != (0, 0)})
