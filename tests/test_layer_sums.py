"""The choice of how linear holds its sums, at the C ABI and at the native call (no GPU needed)."""
import ctypes

import torch

from paper_2605_08565_amd import layers

P, Q = 0x10000, 0x20000                                   # aligned addresses that nobody reads
OK, INVALID = 0, -1


def test_only_the_two_are_taken():
    L = layers._layers()
    for sums, want in ((layers.SUMS_F32, OK), (layers.SUMS_MX, OK), (2, INVALID), (-1, INVALID)):
        args = layers._Linear(x=P, ld_x=128, m=0, n=8, k=128, w_codes=P, w_scales=P, block=32, scale_fmt=0, tensor_scale=1.0, y=Q, ld_y=8, sums=sums)
        assert L.mxq_linear(ctypes.byref(args), None) == want
    assert layers._Linear().sums == layers.SUMS_F32        # what a caller who does not ask gets


def test_the_header_has_the_same_values():
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(layers.__file__))), "include", "mxq_layers.h")).read()
    assert f"MXQ_SUMS_F32 = {layers.SUMS_F32}, MXQ_SUMS_MX = {layers.SUMS_MX}" in text


def test_the_native_call_declines_what_is_not_plain():
    layers._layers()
    x = torch.zeros((2, 64))
    q = layers.Q8(x.to(torch.float8_e4m3fn), torch.zeros((2, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu))
    w = layers.W4(torch.zeros((3, 32), dtype=torch.uint8), torch.zeros((3, 2), dtype=torch.uint8), 32, 0, 1.0)
    for sums in (layers.SUMS_F32, layers.SUMS_MX, "mx"):
        assert layers._calls.linear(q, w, None, None, torch.bfloat16, sums) is None
