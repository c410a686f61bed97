"""A step of AdamW with an eps that 32 bits hardly hold or do not hold: gradients of 0 move nothing."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-37, 1.2e-38, 1e-38, 1e-40, 1e-45, 1e-60, 1e-300])
def test_least_eps(bits, eps):
    """The same as without one where there is a gradient (v is at least 2^-149 there, its root 3.7e-23), and nothing where there is none."""
    from paper_2505_03983_b200 import default_ops
    n, how = 2000, dict(lr=1e-2, betas=(0.9, 0.999), weight_decay=0.0)
    g = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 1e-3
    g[::3] = 0

    def step(e, grad):
        p, c = torch.ones(n, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
        m, v = (torch.zeros(n, dtype=t, device="cuda") for t in ((torch.float32,) * 2 if bits == 32 else (torch.int8, torch.uint8)))
        scales = [torch.zeros(((n + 255) // 256, 2), device="cuda")] if bits == 8 else None
        for _ in range(3):
            default_ops().adamw([p], [grad], [m], [v], c, eps=e, scales=scales, **how)
        return p

    p, q = step(eps, g), step(0.0, g)
    assert (p[::3] == 1).all() and torch.isnan(q[::3]).all()  # 0 / 0 without eps
    there = g != 0
    assert torch.equal(p[there], q[there]) and (p[there] != 1).all()
    assert (step(eps, torch.zeros(n, device="cuda")) == 1).all()
