"""The norm's backward pass where a group of threads goes over several rows and the last round is not whole, for each of its kernels
(64, 256 and 1024 threads a row), and the in-place forms of the backward passes."""
import ctypes

import pytest
import torch

from test_gpu_layers import DTYPES, check, layers, tensors, value  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(9000, 32), (9001, 608), (5000, 1024), (2500, 1056), (1100, 4096), (700, 6176), (700, 8192), (300, 8224), (300, 16384)]


def groups_of(layers, rows, cols):
    return layers._layers().mxq_add_rmsnorm_backward_workspace_size(rows, cols) // (4 * cols)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rows_in_turn(layers, rows, cols, dtype):
    dtype = DTYPES[dtype]
    groups = groups_of(layers, rows, cols)
    assert rows > groups and rows % groups != 0
    x, dy, dh, w = tensors(rows + 3 * cols, (rows, cols), (rows, cols), (rows, cols), (cols,), dtype=dtype)
    _, _, saved = layers.add_rmsnorm(x, eps=1e-5, checkpoint=True)
    n, rstd = value(saved.n), saved.rstd.double()[:, None]
    for weight, dhidden in ((w, dh), (w, None), (None, dh)):
        g = dy.double() * (weight.double() if weight is not None else 1)
        want = rstd * (g - n * (g * n).mean(dim=1, keepdim=True)) + (dhidden.double() if dhidden is not None else 0)
        size = rstd * (g.abs() + n.abs() * (g * n).abs().mean(dim=1, keepdim=True)) + (dhidden.double().abs() if dhidden is not None else 0)
        dx, dweight = layers.add_rmsnorm_backward(dy, saved, weight, dhidden=dhidden)
        check(dx, want, slack=size * 2.0 ** -18)
        if weight is not None:
            # a product and an addition a row of the group, one addition for each 128 groups, 15 and 3 behind them
            sums = -(-rows // groups) + 1 + -(-groups // 128) + 18
            err = (dweight.double() - (dy.double() * n).sum(dim=0)).abs()
            assert bool((err <= sums * 2.0 ** -24 * (dy.double() * n).abs().sum(dim=0)).all())
        for given in ("dy", "dhidden"):
            if given == "dhidden" and dhidden is None:
                continue
            a, b = dy.clone(), None if dhidden is None else dhidden.clone()
            out = a if given == "dy" else b
            got, got_w = layers.add_rmsnorm_backward(a, saved, weight, dhidden=b, dx_out=out)
            assert got is out and torch.equal(got, dx) and (weight is None or torch.equal(got_w, dweight))
            assert torch.equal(a, dx if given == "dy" else dy) and (b is None or torch.equal(b, dx if given == "dhidden" else dhidden))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("rows,cols", [(3, 32), (130, 1056), (700, 4096)])
@pytest.mark.parametrize("given", ["dgate", "dup"])
def test_the_gated_activations_gradient_in_place(layers, rows, cols, dtype, given):
    """Through the C ABI: either output may be the incoming gradient itself, rows apart as they are."""
    dtype = DTYPES[dtype]
    gate, up, wide = tensors(rows + cols, (rows, cols), (rows, cols), (rows, 2 * cols), dtype=dtype)
    dh = wide[:, cols:]
    _, saved = layers.swiglu(gate, up, dense=True, checkpoint=True)
    dgate, dup, h = layers.swiglu_backward(dh, saved, again=True)
    kept = wide[:, :cols].clone()
    other, again = torch.empty_like(gate), torch.empty_like(gate)
    outs = {"dgate": (dh, other), "dup": (other, dh)}[given]
    status = layers._layers().mxq_swiglu_backward(
        dh.data_ptr(), dh.stride(0), saved.gate.codes.data_ptr(), saved.gate.scales.data_ptr(), saved.up.codes.data_ptr(),
        saved.up.scales.data_ptr(), rows, cols, 0 if dtype == torch.bfloat16 else 1, outs[0].data_ptr(), outs[0].stride(0),
        outs[1].data_ptr(), outs[1].stride(0), again.data_ptr(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert status == 0
    assert torch.equal(outs[0], dgate) and torch.equal(outs[1], dup) and torch.equal(again, h) and torch.equal(wide[:, :cols], kept)
