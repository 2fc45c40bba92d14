"""Infinities and NaN in the adapters of layers.linear follow the formula, scaling * (x A^T) first, on every path."""
import pytest
import torch

from test_gpu_linear import E4M3, activations, adapters_of, generator, ids_of, layers, times, weights  # noqa: F401

pytestmark = pytest.mark.gpu
PATHS = [1, 16, 24, 64, 70, 300]                  # the kernels for few tokens, and the two that join tiles


@pytest.mark.parametrize("m", PATHS)
@pytest.mark.parametrize("bad", ["a", "b", "scaling", "both"])
def test_infinities_in_an_adapter_follow_the_formula(layers, m, bad):
    """Infinite where the formula in 64 bits is, with its sign, and NaN where that is NaN (infinity * 0, infinity - infinity)."""
    gen = generator(m + 56)
    k, n, count, rank = 512, 90, 4, 40
    x, x64 = activations(layers, gen, m, k, "bf16", True)
    codes, scales, w64 = weights(gen, n, k, 16, E4M3, True)
    ad, ids = adapters_of(layers, gen, count, rank, n, k, True), ids_of(gen, m, count)
    ids[0] = 2
    if bad in ("a", "both"):
        x[:, 11] = 1
        x64[:, 11] = 1
        ad.a[2, 7, 11] = float("inf")
        ad.b[2, 30, 7] = 0
    if bad in ("b", "both"):
        ad.b[2, 10:20, 39] = float("inf")
        ad.b[2, 20:30, 3] = float("-inf")
    if bad == "scaling":
        ad.scaling[2] = float("inf")
        ad.b[2, :, 1:] = 0
    y = layers.linear(x, layers.W4(codes, scales, 16, E4M3), ad, ids, out_dtype=torch.float32).double()
    want = times(x64, w64)
    for i in range(count):
        at = (ids == i).nonzero()[:, 0]
        want[at] += times(times(x64[at], ad.a[i].double()) * ad.scaling[i].double(), ad.b[i].double())
    assert torch.equal(y.isnan(), want.isnan())
    assert torch.equal(y[~want.isnan()], want[~want.isnan()])
    assert bad == "scaling" or bool(want.isinf().any())
