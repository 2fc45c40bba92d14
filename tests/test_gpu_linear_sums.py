"""How linear's sums are held: in 32 bits unless the caller takes those of the scaled matrix instruction."""
import pytest
import torch

from test_gpu_linear import (E4M3, E8M0, SHAPES, activations, adapters_of, check, generator, ids_of, layers, product, times,  # noqa: F401
                             weights)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 12, 24, 64, 200])
@pytest.mark.parametrize("n,k", [(4096, 128), (1024, 1056)])
@pytest.mark.parametrize("block", [32, 64])
def test_sums_of_bf16_outputs_are_held_in_32_bits(layers, m, n, k, block):
    """Q8 against power-of-two scales that lie far apart.  One output is rounded to bf16, and what fp32 sums may be off by is allowed on
    the sum of magnitudes: outputs whose terms cancel show the sums themselves."""
    gen = generator(m + n + k + block)
    x, x64 = activations(layers, gen, m, k // 64 * 64, "q8", False)
    k = k // 64 * 64
    codes, scales, w64 = weights(gen, n, k, block, E8M0, False)
    check(layers.linear(x, layers.W4(codes, scales, block, E8M0)), *product(x64, w64, 1.0), k)


# ---- the scaled instruction's sums, by choice ----

@pytest.mark.parametrize("m,n,k", SHAPES + [(2100, 1300, 64), (1030, 4100, 160), (4097, 257, 96), (3000, 130, 2048)])
def test_exact_sums_of_the_scaled_instruction(layers, m, n, k):
    gen = generator(m * 1000 + n + k)
    x, x64 = activations(layers, gen, m, k, "q8", True)
    for block in (32, 64, 128):
        if k % block:
            continue
        codes, scales, w64 = weights(gen, n, k, block, E8M0, True)
        y = layers.linear(x, layers.W4(codes, scales, block, E8M0, 0.5), sums=layers.SUMS_MX)
        assert torch.equal(y, (times(x64, w64) * 0.5).bfloat16()), block


@pytest.mark.parametrize("count,rank", [(1, 8), (3, 16), (5, 24), (20, 32), (4, 64), (40, 8)])
@pytest.mark.parametrize("m,n,k", [(1, 100, 512), (16, 33, 96), (24, 260, 1056), (70, 64, 128), (300, 520, 256)])
def test_exact_sums_of_the_scaled_instruction_with_adapters(layers, m, n, k, count, rank):
    gen = generator(m + n + k + count + rank)
    x, x64 = activations(layers, gen, m, k, "q8", True)
    ad = adapters_of(layers, gen, count, rank, n, k, True)
    codes, scales, w64 = weights(gen, n, k, 32, E8M0, True)
    for order in ("mixed", "sorted"):
        ids = ids_of(gen, m, count, order)
        y = layers.linear(x, layers.W4(codes, scales, 32, E8M0, 2.0), ad, ids, sums=layers.SUMS_MX)
        assert torch.equal(y, product(x64, w64, 2.0, ad, ids)[0].bfloat16()), order


@pytest.mark.parametrize("block", [32, 64])
@pytest.mark.parametrize("m,n,k", [(1, 200, 4096), (20, 97, 1024), (90, 260, 2048), (520, 300, 1024)])
def test_random_values_by_the_scaled_instruction(layers, m, n, k, block):
    """Within what the header promises; and where types, format or block do not allow it, the choice changes nothing."""
    gen = generator(m + 7 * n + k + block)
    x, x64 = activations(layers, gen, m, k, "q8", False)
    ad, ids = adapters_of(layers, gen, 6, 16, n, k, False), ids_of(gen, m, 6)
    codes, scales, w64 = weights(gen, n, k, block, E8M0, False)
    w = layers.W4(codes, scales, block, E8M0)
    check(layers.linear(x, w, sums=layers.SUMS_MX), *product(x64, w64, 1.0), k, True)
    check(layers.linear(x, w, ad, ids, sums=layers.SUMS_MX), *product(x64, w64, 1.0, ad, ids), k, True)
    dense = x.float().bfloat16()
    w16 = layers.W4(*weights(gen, n, k, 16, E4M3, False)[:2], 16, E4M3)
    for args, out in (((dense, w), torch.bfloat16), ((x, w16), torch.bfloat16), ((x, w), torch.float32)):
        assert torch.equal(layers.linear(*args, ad, ids, out_dtype=out, sums=layers.SUMS_MX), layers.linear(*args, ad, ids, out_dtype=out))


@pytest.mark.parametrize("sums", ["SUMS_F32", "SUMS_MX"])
@pytest.mark.parametrize("m", [1, 5, 20, 40, 150, 600])
@pytest.mark.parametrize("k,block", [(160, 32), (192, 64), (1056, 32), (384, 128)])
def test_rows_do_not_mix_with_power_of_two_scales(layers, m, k, block, sums):
    """NaN scale bytes and codes stay in their row of x or of w: also the first byte of a row, which lies behind the last, incomplete
    chunk of the row before."""
    gen = generator(m + k + block)
    n = 50
    sums = getattr(layers, sums)
    codes, scales, _ = weights(gen, n, k, block, E8M0, True)
    w = layers.W4(codes, scales, block, E8M0)
    x, _ = activations(layers, gen, m, k, "q8", True)
    want = layers.linear(x, w, sums=sums)
    assert bool(want.isfinite().all())
    for bad, at in ((m // 2, 0), (m - 1, k // 32 - 1), (0, 1)):
        byte = x.scales.view(torch.uint8)
        keep = int(byte[bad, at])
        byte[bad, at] = 255
        y = layers.linear(x, w, sums=sums)
        rest = torch.arange(m, device="cuda") != bad
        assert torch.equal(y[rest], want[rest]) and bool(y[bad].isnan().all()), (bad, at)
        byte[bad, at] = keep
    for bad, at, nan in ((m // 2, 0, 0x7F), (m - 1, k - 1, 0xFF)):
        byte = x.codes.view(torch.uint8)
        keep = int(byte[bad, at])
        byte[bad, at] = nan
        y = layers.linear(x, w, sums=sums)
        rest = torch.arange(m, device="cuda") != bad
        assert torch.equal(y[rest], want[rest]) and bool(y[bad].isnan().all()), (bad, at)
        byte[bad, at] = keep
    for bad, at in ((n // 2, 0), (n - 1, k // block - 1), (16, 0), (0, 0)):
        keep = int(scales[bad, at])
        scales[bad, at] = 255
        y = layers.linear(x, w, sums=sums)
        rest = torch.arange(n, device="cuda") != bad
        assert torch.equal(y[:, rest], want[:, rest]) and bool(y[:, bad].isnan().all()), (bad, at)
        scales[bad, at] = keep


def test_refusals_of_sums(layers):
    from paper_2605_08565_amd.mxq import MxqError
    gen = generator(1)
    x, _ = activations(layers, gen, 4, 128, "q8", True)
    w = layers.W4(*weights(gen, 40, 128, 32, E8M0, True)[:2], 32, E8M0)
    for wrong in (2, -1):
        with pytest.raises(MxqError, match="INVALID_ARG"):
            layers.linear(x, w, sums=wrong)
    with pytest.raises(TypeError):
        layers.linear(x, w, sums="mx")
