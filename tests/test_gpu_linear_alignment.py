"""Operands of layers.linear at the least alignment that include/mxq_layers.h asks for give the bits of aligned ones, on every path."""
import pytest
import torch

from test_gpu_linear import E4M3, E8M0, activations, adapters_of, generator, ids_of, layers, weights  # noqa: F401

pytestmark = pytest.mark.gpu


def moved(t, by):
    """The same tensor `by` bytes behind an aligned address, in memory that ends with it and holds 0xFF around it."""
    flat = t.contiguous().view(torch.uint8).reshape(-1)
    store = torch.full((by + flat.numel(),), 255, device="cuda", dtype=torch.uint8)
    store[by:] = flat
    return store[by:].view(t.dtype).view(t.shape)


@pytest.mark.parametrize("m", [1, 9, 20, 40, 150, 600])
@pytest.mark.parametrize("k", [160, 512, 1056])
def test_least_alignment(layers, m, k):
    gen = generator(m + k)
    n, count = 90, 3
    ad, ids = adapters_of(layers, gen, count, 16, n, k, True), ids_of(gen, m, count)
    low = layers.Adapters(moved(ad.a, 16), moved(ad.b, 16), moved(ad.scaling, 4))
    for kind, block, fmt, sums in (("q8", 32, E8M0, layers.SUMS_MX), ("q8", 32, E8M0, layers.SUMS_F32), ("q8", 16, E4M3, layers.SUMS_F32),
                                   ("bf16", 16, E4M3, layers.SUMS_F32)):
        x, _ = activations(layers, gen, m, k, kind, True)
        codes, scales, _ = weights(gen, n, k, block, fmt, True)
        want = layers.linear(x, layers.W4(codes, scales, block, fmt), ad, ids, sums=sums)
        for by in (1, 2, 3, 4, 8):
            xm = moved(x, 16) if kind == "bf16" else layers.Q8(moved(x.codes, 16), moved(x.scales, by))
            w = layers.W4(moved(codes, 16), moved(scales, 4 if by < 8 else 8), block, fmt)
            assert torch.equal(layers.linear(xm, w, low, moved(ids, 4), sums=sums), want), (kind, block, by)
