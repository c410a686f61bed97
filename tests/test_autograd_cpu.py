"""The autograd functions over a stand-in for the handle, on the CPU: which calls they make of it, and what they answer where a
derivative does not exist.  The stand-in computes the operators' formulas in 64 bits and, like the native calls, records no graph."""
import pytest
import torch

from paper_2505_03983_b200 import autograd

F64 = torch.float64


class Stand:
    def __init__(self):
        self.calls = []

    @torch.no_grad()
    def add_rmsnorm(self, x, weight, residual=None, eps=1e-6):
        self.calls.append(("add_rmsnorm",))
        s = x if residual is None else x + residual
        y = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + eps)
        return (y if weight is None else y * weight), s

    @torch.no_grad()
    def add_rmsnorm_backward(self, dy, s, weight, ds=None, eps=1e-6, need_dweight=True, need_dx=True):
        self.needed_dx = need_dx
        self.calls.append(("add_rmsnorm_backward", ds is not None, need_dweight))
        rho = torch.rsqrt(s.square().mean(-1, keepdim=True) + eps)
        z, dz = s * rho, dy if weight is None else dy * weight
        dx = rho * (dz - z * (dz * z).mean(-1, keepdim=True))
        return (None if not need_dx else dx if ds is None else dx + ds), ((dy * z).sum(0) if need_dweight else None)

    @torch.no_grad()
    def gated_mlp(self, x, w_in, w_out, act="silu"):
        self.calls.append(("gated_mlp",))
        g, u = (x @ w_in.T).chunk(2, -1)
        return (torch.nn.functional.silu(g) * u) @ w_out.T

    @torch.no_grad()
    def gated_mlp_forward(self, x, w_in, w_out, act="silu"):
        y = self.gated_mlp(x, w_in, w_out)
        self.calls[-1] = ("gated_mlp_forward",)
        return y, torch.empty(0)

    @torch.no_grad()
    def gated_mlp_backward(self, dy, x, w_in, w_out, saved, act="silu", need=(True, True, True)):
        self.calls.append(("gated_mlp_backward", tuple(need)))
        (g, u), dh = (x @ w_in.T).chunk(2, -1), dy @ w_out
        p = torch.sigmoid(g)
        d = torch.cat([dh * u * p * (1 + g * (1 - p)), dh * g * p], -1)
        return tuple(v if n else None for n, v in zip(need, (d @ w_in, d.T @ x, dy.T @ (g * p * u))))


@pytest.fixture
def stand(monkeypatch):
    s = Stand()
    monkeypatch.setattr(autograd, "default_ops", lambda: s)
    return s


def make(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=F64)


def leaves(*shapes):
    return [make(*s, seed=i).requires_grad_() for i, s in enumerate(shapes)]


def operators_of(x, r, w, wi, wo):
    yield "norm with a residual", lambda v: autograd.add_rmsnorm(v, w, r)[0]
    yield "norm", lambda v: autograd.add_rmsnorm(v, w)[0]
    yield "gated MLP", lambda v: autograd.gated_mlp(v, wi, wo)


@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("direction", ["of the loss", "constant"])
def test_second_derivatives_raise(stand, which, direction):
    """A penalty on a gradient, behind an operation that has a second derivative of its own; the direction of the first derivative
    may itself depend on the inputs, or (a divergence along a fixed vector) not."""
    x, r, w, wi, wo = leaves((5, 8), (5, 8), (8,), (12, 8), (8, 6))
    _, f = list(operators_of(x, r, w, wi, wo))[which]
    y = f(x * x)
    if direction == "constant":
        dx, = torch.autograd.grad(y, x, make(5, 8, seed=9), create_graph=True)
    else:
        dx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives"):
        dx.square().sum().backward()


@pytest.mark.parametrize("which", range(3))
def test_first_derivatives_with_a_graph_are_the_same(stand, which):
    """create_graph alone is no error, and what does not go through the operator can still be differentiated."""
    x, r, w, wi, wo = leaves((5, 8), (5, 8), (8,), (12, 8), (8, 6))
    _, f = list(operators_of(x, r, w, wi, wo))[which]
    want, = torch.autograd.grad(f(x * x).square().sum(), x)
    got, = torch.autograd.grad(f(x * x).square().sum(), x, create_graph=True)
    assert torch.equal(got, want)
    z = make(5, 8, seed=9).requires_grad_()
    dz, = torch.autograd.grad(f(x).square().sum() + z.pow(3).sum(), z, create_graph=True)
    ddz, = torch.autograd.grad(dz.sum(), z)
    assert torch.allclose(ddz, 6 * z)


@pytest.mark.parametrize("off", [torch.no_grad, torch.inference_mode])
def test_serving_keeps_nothing_for_a_backward_pass(stand, off):
    """Parameters that require gradients, in a region that records none: the forward that keeps nothing."""
    x, wi, wo = leaves((5, 8), (12, 8), (8, 6))
    with off():
        y = autograd.gated_mlp(x, wi, wo)
    assert stand.calls == [("gated_mlp",)] and not y.requires_grad
    stand.calls.clear()
    autograd.gated_mlp(x.detach(), wi.detach(), wo.detach())
    assert stand.calls == [("gated_mlp",)]
    stand.calls.clear()
    autograd.gated_mlp(x.detach(), wi.detach(), wo).sum().backward()
    assert stand.calls == [("gated_mlp_forward",), ("gated_mlp_backward", (False, False, True))]


def test_forward_mode_raises(stand):
    x, w, wi, wo = make(5, 8), make(8), make(12, 8), make(8, 6)
    with torch.autograd.forward_ad.dual_level():
        d = torch.autograd.forward_ad.make_dual(x, make(5, 8, seed=9))
        for f in (lambda: autograd.gated_mlp(d, wi, wo), lambda: autograd.add_rmsnorm(d, w)):
            with pytest.raises((RuntimeError, NotImplementedError)):
                f()


def test_outputs_that_are_not_used_bring_no_zeros(stand):
    """Where s, or y, is not used further its gradient is absent, not a tensor of zeros that a kernel reads."""
    x, r, w = leaves((5, 8), (5, 8), (8,))
    for residual in (None, r):
        stand.calls.clear()
        autograd.add_rmsnorm(x, w, residual)[0].square().sum().backward()
        assert stand.calls[1:] == [("add_rmsnorm_backward", False, True)]
    # s alone: its gradient is that of x and of the residual, and the weight's is zero
    stand.calls.clear()
    ds = make(5, 8, seed=9)
    dx, dw, dr = torch.autograd.grad(autograd.add_rmsnorm(x, w, r)[1], (x, w, r), ds)
    assert len(stand.calls) == 1 and torch.equal(dx, ds) and torch.equal(dr, ds) and not dw.any()
    # both, against the formula's own graph
    y, s = autograd.add_rmsnorm(x, w, r)
    got = torch.autograd.grad((y.square().sum() + s.pow(3).sum()), (x, w, r))
    s = x + r
    y = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * w
    for a, b in zip(got, torch.autograd.grad((y.square().sum() + s.pow(3).sum()), (x, w, r))):
        assert torch.allclose(a, b)


def test_a_gradient_that_nothing_needs_is_not_computed(stand):
    """The first norm of a network: its inputs are data, its weight a parameter."""
    x, r, w = make(5, 8), make(5, 8, seed=1), make(8, seed=2).requires_grad_()
    for residual in (None, r):
        y, s = autograd.add_rmsnorm(x, w, residual)
        y.square().sum().backward()
        assert stand.calls[-1] == ("add_rmsnorm_backward", False, True) and not stand.needed_dx
    for leaf in (x, r):
        leaf.requires_grad_()
        autograd.add_rmsnorm(x, w, r)[0].sum().backward()
        assert stand.needed_dx and leaf.grad is not None
        leaf.requires_grad_(False)
