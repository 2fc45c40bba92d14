"""One MLP block of a language model on the layer operators, as a server and as a trainer run it.

Serving (``MLP.serve``): norm with the residual's addition -> gate and up in one projection -> gated activation -> down, the
activations between them in 8 bits, the weights in packed FP4, every row with its request's low-rank adapters.
Training (``train_block``): the same block with dense products; what norm and activation keep for the backward pass is in 8 bits.

    python -m paper_2605_08565_amd.mlp [--hidden 4096] [--mlp 14336] [--adapters 8] [--tokens 1,16,512] [--train 2048] [--mx-sums]

Prints one JSON line: times, the serving path's distance from the block in fp32, and what training keeps and how far its gradients are.
"""
from __future__ import annotations

import argparse
import json
import time

import torch
from torch.autograd.function import once_differentiable

from . import layers, mxq
from .layers import Adapters, Q8, SavedNorm, SavedSwiglu, W4


def pack(weight: torch.Tensor, block: int = 32, scale_fmt: int = mxq.SCALE_E8M0, recipe: int = mxq.RECIPE_ABSMAX) -> W4:
    """Dense weights [n, k] as linear takes them.  Power-of-two scales of 32 can multiply with 8-bit activations as they are
    (layers.SUMS_MX); E4M3 scales of 16 (with RECIPE_4OVER6) are closer to the weights."""
    if scale_fmt == mxq.SCALE_E8M0:
        codes, scales, _ = mxq.quantize(weight, block, scale_fmt, recipe, want_sse=False)
        return W4(codes, scales, block, scale_fmt)
    codes, scales, _, t = mxq.quantize_hier(weight, block, scale_fmt, recipe, mxq.tensor_absmax(weight), want_sse=False)
    return W4(codes, scales, block, scale_fmt, t)


class MLP:
    """A served block: packed weights and the adapters of its two projections (or None).  `sums`: how the projections hold their
    sums (layers.linear)."""

    def __init__(self, norm_weight: torch.Tensor, gate_up: W4, down: W4, adapters_gate_up: Adapters | None = None,
                 adapters_down: Adapters | None = None, eps: float = 1e-5, sums: int = layers.SUMS_F32):
        self.norm_weight, self.gate_up, self.down, self.eps, self.sums = norm_weight, gate_up, down, eps, sums
        self.adapters_gate_up, self.adapters_down = adapters_gate_up, adapters_down
        self.width = gate_up.codes.shape[0] // 2

    def serve(self, x: torch.Tensor, residual: torch.Tensor, ids: torch.Tensor | None = None):
        """(the block's output, the updated residual stream): x and residual [tokens, hidden], ids the adapter of each token.  The
        residual is updated in place."""
        y, hidden, _ = layers.add_rmsnorm(x, self.norm_weight, residual, self.eps, hidden_out=residual)
        both = layers.linear(y, self.gate_up, self.adapters_gate_up, ids if self.adapters_gate_up is not None else None, sums=self.sums)
        h, _ = layers.swiglu(both[:, :self.width], both[:, self.width:])
        return layers.linear(h, self.down, self.adapters_down, ids if self.adapters_down is not None else None, sums=self.sums), hidden


class AddRMSNorm(torch.autograd.Function):
    """(y, hidden) = apply(x, weight, residual, eps), with the normalised rows kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        y, hidden, saved = layers.add_rmsnorm(x, weight, residual, eps, dense=True, checkpoint=True)
        ctx.save_for_backward(weight, saved.n.codes, saved.n.scales, saved.rstd)
        ctx.set_materialize_grads(False)
        return y, hidden

    @staticmethod
    @once_differentiable                                  # the kernels record nothing: second derivatives are an error, not zero
    def backward(ctx, dy, dhidden):
        weight, codes, scales, rstd = ctx.saved_tensors
        if dy is None:
            return dhidden, None, dhidden, None
        dx, dweight = layers.add_rmsnorm_backward(dy.contiguous(), SavedNorm(Q8(codes, scales), rstd), weight,
                                                  dhidden=None if dhidden is None else dhidden.contiguous())
        return dx, dweight.to(weight.dtype), dx, None


class SwiGLU(torch.autograd.Function):
    """h = apply(both): gate and up are the halves of [tokens, 2 * width], kept in 8 bits.  h itself stays with the product behind it, whose
    weight gradient is then that of the h it multiplied; swiglu_backward(again=True) forms h from the 8 bits for who would rather not keep it."""

    @staticmethod
    def forward(ctx, both):
        width = both.shape[1] // 2
        h, saved = layers.swiglu(both[:, :width], both[:, width:], dense=True, checkpoint=True)
        ctx.save_for_backward(*saved.gate, *saved.up)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        gc, gs, uc, us = ctx.saved_tensors
        dgate, _, _ = layers.swiglu_backward(dh.contiguous(), SavedSwiglu(Q8(gc, gs), Q8(uc, us)))
        return dgate.as_strided((dh.shape[0], 2 * dh.shape[1]), (2 * dh.shape[1], 1))        # the halves of one tensor


def train_block(x, residual, norm_weight, gate_up, down, eps: float = 1e-5):
    """(output, residual stream) of the block with dense weights, for autograd."""
    y, hidden = AddRMSNorm.apply(x, norm_weight, residual, eps)
    return SwiGLU.apply(y @ gate_up.t()) @ down.t(), hidden


def plain_block(x, residual, norm_weight, gate_up, down, eps: float = 1e-5):
    """The same by elementary operations, in the inputs' type."""
    t = x + residual
    y = t * torch.rsqrt(t.float().square().mean(dim=1, keepdim=True) + eps).to(t.dtype) * norm_weight
    gate, up = (y @ gate_up.t()).chunk(2, dim=1)
    return (gate * torch.sigmoid(gate) * up) @ down.t(), t


def _random(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return (scale * torch.randn(shape, generator=gen, device="cuda")).to(dtype)


def make(hidden: int, width: int, count: int, rank: int = 16, seed: int = 1, **packing):
    """A block with random weights: (MLP, its dense fp32 weights as they read back from FP4)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dense = [_random(gen, 2 * width, hidden, scale=hidden ** -0.5), _random(gen, hidden, width, scale=width ** -0.5)]
    norm_weight = _random(gen, hidden, scale=0.1) + 1
    packed = [pack(w, **packing) for w in dense]
    adapters = [None, None]
    if count:
        adapters = [Adapters(_random(gen, count, rank, w.shape[1], scale=w.shape[1] ** -0.5), _random(gen, count, w.shape[0], rank, scale=0.02),
                             torch.full((count,), 2.0, device="cuda")) for w in dense]
    back = [mxq.dequantize(w.codes, w.scales, w.block, w.scale_fmt, w.tensor_scale) for w in packed]
    return MLP(norm_weight, *packed, *adapters), back


def _timed(f, reps=50):
    f()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(reps):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - began) / reps * 1e6


def run(hidden: int, width: int, count: int, tokens, train: int, sums: int = layers.SUMS_F32) -> dict:
    out = {"hidden": hidden, "mlp": width, "adapters": count, "serve": {}}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    block, back = make(hidden, width, count)
    block.sums = sums
    for m in tokens:
        x, residual = _random(gen, m, hidden), _random(gen, m, hidden)
        ids = torch.randint(0, max(count, 1), (m,), generator=gen, device="cuda", dtype=torch.int32) if count else None
        y, stream = block.serve(x, residual.clone(), torch.full_like(ids, -1) if count else None)
        want, t = plain_block(x.float(), residual.float(), block.norm_weight.float(), *back)
        out["serve"][str(m)] = {"us": round(_timed(lambda: block.serve(x, residual, ids)), 1),
                                "off": round(float((y.float() - want).norm() / want.norm()), 4)}
    if train:
        del block
        leaves = [_random(gen, train, hidden), (_random(gen, hidden, scale=0.1) + 1), _random(gen, train, hidden),
                  back[0].bfloat16(), back[1].bfloat16()]
        leaves = [v.requires_grad_() for v in leaves]
        x, nw, residual, gu, down = leaves
        c = _random(gen, train, hidden)
        grads = {}
        for name, f in (("plain", plain_block), ("saved in 8 bits", train_block)):
            before = torch.cuda.memory_allocated()
            y, stream = f(x, residual, nw, gu, down)
            kept = torch.cuda.memory_allocated() - before
            grads[name] = torch.autograd.grad((y.float() * c).sum() + stream.float().sum(), leaves)
            out.setdefault("train", {})[name] = {"kept_MiB": round(kept / 2 ** 20, 1)}
            del y, stream
        out["train"]["off"] = [round(float((a.float() - b.float()).norm() / b.float().norm()), 4)
                               for a, b in zip(grads["saved in 8 bits"], grads["plain"])]
    return out


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--mlp", type=int, default=14336)
    ap.add_argument("--adapters", type=int, default=8)
    ap.add_argument("--tokens", default="1,16,512")
    ap.add_argument("--train", type=int, default=2048)
    ap.add_argument("--mx-sums", action="store_true", help="sums of the scaled matrix instruction: about 21 bits, up to twice as fast")
    a = ap.parse_args()
    print(json.dumps(run(a.hidden, a.mlp, a.adapters, [int(t) for t in a.tokens.split(",")], a.train,
                         layers.SUMS_MX if a.mx_sums else layers.SUMS_F32)), flush=True)


if __name__ == "__main__":
    main()
