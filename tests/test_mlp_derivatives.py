"""Derivatives of the training block's functions (paper_2605_08565_amd.mlp) beyond the first: the kernels record nothing for autograd, so
asking for them is an error and never a silent zero.  On the CPU with stand-ins of the operators that record nothing either."""
import pytest
import torch

from paper_2605_08565_amd import layers, mlp


@pytest.fixture
def stand_ins(monkeypatch):
    def add_rmsnorm(x, weight, residual, eps, dense, checkpoint):
        with torch.no_grad():
            t = x + residual
            rstd = 1 / (t.square().mean(dim=1) + eps).sqrt()
            return t * rstd[:, None] * weight, t, layers.SavedNorm(layers.Q8(t * rstd[:, None], rstd), rstd)

    def add_rmsnorm_backward(dy, saved, weight, dhidden=None):
        with torch.no_grad():
            n, g = saved.n.codes, dy * weight
            dx = saved.rstd[:, None] * (g - n * (g * n).mean(dim=1, keepdim=True))
            return dx if dhidden is None else dx + dhidden, (dy * n).sum(dim=0)

    def swiglu(gate, up, dense, checkpoint):
        with torch.no_grad():
            return gate * gate.sigmoid() * up, layers.SavedSwiglu(layers.Q8(gate.clone(), gate.clone()), layers.Q8(up.clone(), up.clone()))

    def swiglu_backward(dh, saved):
        with torch.no_grad():
            g, u = saved.gate.codes, saved.up.codes
            s = g.sigmoid()
            both = torch.cat((dh * u * s * (1 + g * (1 - s)), dh * g * s), dim=1)
            return both[:, :g.shape[1]], both[:, g.shape[1]:], None
    for f in (add_rmsnorm, add_rmsnorm_backward, swiglu, swiglu_backward):
        monkeypatch.setattr(layers, f.__name__, f)


def leaves():
    gen = torch.Generator().manual_seed(1)
    return [torch.randn(s, generator=gen, dtype=torch.float64).requires_grad_() for s in ((5, 64), (64,), (5, 64))]


def test_first_derivatives_are_those_of_the_stand_ins(stand_ins):
    x, w, r = leaves()
    assert torch.autograd.gradcheck(lambda *a: mlp.AddRMSNorm.apply(*a, 1e-5), (x, w, r))
    assert torch.autograd.gradcheck(mlp.SwiGLU.apply, (torch.cat((x, r), dim=1).detach().requires_grad_(),))


@pytest.mark.parametrize("which", ["norm", "swiglu"])
def test_second_derivatives_are_an_error(stand_ins, which):
    x, w, r = leaves()
    if which == "norm":
        y, _ = mlp.AddRMSNorm.apply(x, w, r, 1e-5)
    else:
        y = mlp.SwiGLU.apply(torch.cat((x, r), dim=1))
    first, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        first.square().sum().backward()
