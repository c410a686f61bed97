"""The example that trains a gated denoiser in 16 bits and serves it in 8, and the autograd functions it trains with."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if os.path.join(ROOT, "examples") not in sys.path:
    sys.path.insert(0, os.path.join(ROOT, "examples"))


def test_example_learns_and_the_8_bit_service_follows():
    import gated_denoiser
    r = gated_denoiser.run(steps=250, batch=2048, chains=1024, log=lambda *_: None)
    # the mixture's means lie in a box of +-4, so predicting their mean costs about 16 / 3; what is left of the loss at the end
    # is mostly the posterior's own variance at small t
    assert r["losses"][-1] < 0.5 * r["losses"][0]
    assert r["error_16"] < 0.5 * r["drift_rms"]
    # 8-bit rows: 1/254 of a row's largest value at most, some 3 standard deviations, in each of two products of three blocks
    assert r["gap"] < 0.1 * r["drift_rms"]
    assert r["near_a_component"] > 0.5


def test_autograd_functions_match_torch():
    """Against torch's own graph of the same formulas in 32 bits, on the same 16-bit inputs: each result is off by the
    16-bit roundings of a few intermediate values, each at most 2^-8 of its size."""
    from paper_2505_03983_b200.autograd import add_rmsnorm, gated_mlp
    g = torch.Generator(device="cuda").manual_seed(0)
    rows, width, hidden = 70, 136, 200

    def make(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)

    x, r, w = make(rows, width), make(rows, width), make(width)
    wi, wo = make(2 * hidden, width, scale=width ** -0.5), make(width, hidden, scale=hidden ** -0.5)
    dy, ds = make(rows, width), make(rows, width)

    def leaves(dtype):
        return [v.detach().clone().to(dtype).requires_grad_() for v in (x, r, w, wi, wo)]

    def plain(x, r, w, wi, wo):
        s = x + r
        n = s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * w
        a, u = (n @ wi.T).chunk(2, -1)
        return (torch.nn.functional.silu(a) * u) @ wo.T, s

    mine, ref = leaves(torch.bfloat16), leaves(torch.float32)
    n, s = add_rmsnorm(mine[0], mine[2], mine[1])
    y = gated_mlp(n, mine[3], mine[4])
    torch.autograd.backward([y, s], [dy, ds])
    y0, s0 = plain(*ref)
    torch.autograd.backward([y0, s0], [dy.float(), ds.float()])
    for a, b in [(y, y0), (s, s0)] + [(p.grad, q.grad) for p, q in zip(mine, ref)]:
        assert (a.float() - b).norm() <= 8 * 2.0 ** -8 * b.norm()
    assert torch.equal(mine[0].grad, mine[1].grad)

    # without a residual, with nothing that needs a gradient, and with a part of them
    n, s = add_rmsnorm(mine[0], None)
    (n.float().sum() + s.float().sum()).backward()
    with torch.no_grad():
        assert torch.equal(gated_mlp(x, wi, wo), gated_mlp(x, wi, wo))
    only = wo.clone().requires_grad_()
    gated_mlp(x, wi, only).sum().backward()
    assert only.grad.shape == wo.shape
