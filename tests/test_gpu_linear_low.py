"""The adapters' inner product (layers.linear) between its two products: held in 32 bits on every path."""
import pytest
import torch

from test_gpu_linear import E4M3, generator, layers, product  # noqa: F401

pytestmark = pytest.mark.gpu
PATHS = [1, 16, 24, 64, 70, 300]                  # the kernels for few tokens, and the two that join tiles


def nothing(layers, n, k):
    """Weights of zeros."""
    return layers.W4(torch.zeros((n, k // 2), device="cuda", dtype=torch.uint8), torch.full((n, k // 16), 8 * 7, device="cuda", dtype=torch.uint8), 16, E4M3)


@pytest.mark.parametrize("m", PATHS)
@pytest.mark.parametrize("rank", [8, 40])
def test_the_inner_product_is_held_in_32_bits(layers, m, rank):
    """Inner products of 24 bits, which fp32 holds, in the last of the adapter's rows; every factor is one that bf16 holds."""
    gen = generator(m + rank)
    k, n, count = 64, 75, 3
    x = torch.zeros((m, k), device="cuda")
    x[:, :3] = 1.0
    a = torch.zeros((count, rank, k), device="cuda")
    a[:, rank - 1, 0] = torch.randint(128, 256, (count,), generator=gen, device="cuda") * 65536.0
    a[:, rank - 1, 1] = torch.randint(128, 256, (count,), generator=gen, device="cuda") * 256.0
    a[:, rank - 1, 2] = torch.randint(64, 128, (count,), generator=gen, device="cuda") * 2.0 + 1.0
    b = torch.zeros((count, n, rank), device="cuda")
    b[:, :, rank - 1] = torch.exp2(torch.randint(-3, 4, (count, n), generator=gen, device="cuda").float())
    ad = layers.Adapters(a.bfloat16(), b.bfloat16(), torch.tensor([1.0, -2.0, 0.5], device="cuda"))
    ids = (torch.arange(m, device="cuda") % (count + 1)).int()
    y = layers.linear(x.bfloat16(), nothing(layers, n, k), ad, ids, out_dtype=torch.float32)
    want = product(x.double(), torch.zeros((n, k), device="cuda", dtype=torch.float64), 1.0, ad, ids)[0]
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("m", PATHS)
def test_an_inner_product_beyond_the_largest_bf16(layers, m):
    """2^127 * (2 - 2^-8): fp32 holds it, bf16 rounds it to infinity."""
    k, n = 64, 20
    x = torch.zeros((m, k), device="cuda")
    x[:, 0], x[:, 1] = 2.0 ** 64 * 1.9921875, 2.0 ** 64 * 2.0 ** -8
    a = torch.zeros((1, 8, k), device="cuda")
    a[:, 5, :2] = 2.0 ** 63
    b = torch.zeros((1, n, 8), device="cuda")
    b[:, :, 5] = 2.0 ** -20
    ad = layers.Adapters(a.bfloat16(), b.bfloat16(), torch.ones(1, device="cuda"))
    y = layers.linear(x.bfloat16(), nothing(layers, n, k), ad, out_dtype=torch.float32)
    assert bool((y.double() == 2.0 ** 107 * (2 - 2.0 ** -8)).all())
