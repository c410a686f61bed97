"""The autograd functions on the device: types, parts of the gradients, serving with parameters, second derivatives."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS, WIDTH, HIDDEN = 70, 136, 200


def make(*shape, seed=0, scale=1.0, dtype=torch.float16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def inputs(dtype):
    return (make(ROWS, WIDTH, seed=1, dtype=dtype), make(ROWS, WIDTH, seed=2, dtype=dtype), make(WIDTH, seed=3, dtype=dtype),
            make(2 * HIDDEN, WIDTH, seed=4, scale=WIDTH ** -0.5, dtype=dtype), make(WIDTH, HIDDEN, seed=5, scale=HIDDEN ** -0.5, dtype=dtype))


def plain(x, r, w, wi, wo):
    s = x + r
    n = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * w
    a, u = (n @ wi.T).chunk(2, -1)
    return (torch.nn.functional.silu(a) * u) @ wo.T, s


@pytest.mark.parametrize("kind,unit", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
@pytest.mark.parametrize("needed", [(True,) * 5, (True, False, False, False, False), (False, True, False, True, False), (False, False, True, False, True)])
def test_parts_of_the_gradients(kind, unit, needed):
    """Against torch's graph of the formulas in 32 bits: each result is off by the 16-bit roundings of a few intermediate values."""
    from paper_2505_03983_b200.autograd import add_rmsnorm, gated_mlp
    data, dy, ds = inputs(kind), make(ROWS, WIDTH, seed=6, dtype=kind), make(ROWS, WIDTH, seed=7, dtype=kind)
    mine = [v.clone().requires_grad_(n) for v, n in zip(data, needed)]
    ref = [v.float().requires_grad_(n) for v, n in zip(data, needed)]
    n, s = add_rmsnorm(mine[0], mine[2], mine[1])
    y = gated_mlp(n, mine[3], mine[4])
    y0, s0 = plain(*ref)
    outs = [(y, y0, dy), (s, s0, ds)] if s0.requires_grad else [(y, y0, dy)]
    torch.autograd.backward([o[0] for o in outs], [o[2] for o in outs])
    torch.autograd.backward([o[1] for o in outs], [o[2].float() for o in outs])
    for a, b in [(o[0], o[1]) for o in outs] + [(p.grad, q.grad) for p, q in zip(mine, ref) if q.requires_grad]:
        assert a.dtype == kind and (a.float() - b).norm() <= 8 * unit * b.norm()
    assert all(p.grad is None for p, k in zip(mine, needed) if not k)


def test_serving_with_parameters():
    """The forward that keeps nothing: its bits, and no memory beyond its output and workspace."""
    from paper_2505_03983_b200 import default_ops
    from paper_2505_03983_b200.autograd import gated_mlp
    x, _, _, wi, wo = inputs(torch.bfloat16)
    want = default_ops().gated_mlp(x, wi, wo)
    p = [v.clone().requires_grad_() for v in (x, wi, wo)]
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            y = gated_mlp(*p)
        assert torch.equal(y, want) and not y.requires_grad

    def most(f):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        start = torch.cuda.memory_allocated()
        f()
        return torch.cuda.max_memory_allocated() - start

    with torch.no_grad():
        assert most(lambda: gated_mlp(*p)) == most(lambda: default_ops().gated_mlp(x, wi, wo))


def test_second_derivatives_raise():
    from paper_2505_03983_b200.autograd import add_rmsnorm, gated_mlp
    x, r, w, wi, wo = [v.clone().requires_grad_() for v in inputs(torch.bfloat16)]
    for f in (lambda v: add_rmsnorm(v, w, r)[0], lambda v: add_rmsnorm(v, w)[0], lambda v: gated_mlp(v, wi, wo)):
        dx, = torch.autograd.grad(f(x * x), x, make(ROWS, WIDTH, seed=6, dtype=torch.bfloat16), create_graph=True)
        first, = torch.autograd.grad(f(x * x), x, make(ROWS, WIDTH, seed=6, dtype=torch.bfloat16))
        assert torch.equal(dx, first)
        with pytest.raises(RuntimeError, match="first derivatives"):
            dx.float().square().sum().backward()
