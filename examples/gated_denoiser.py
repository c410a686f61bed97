"""A gated denoiser for the two-dimensional mixture of cfg1_gmm2d: trained in 16 bits, served with 8-bit integers.

The network learns the posterior mean m(t, y) = E[x* | y_t = y] of the stochastic-localization process (y_t = t x* + W_t) by
regression on x*, which is the drift that the sampler integrates.  Its blocks are

    n, s = norm(delta + s);   delta = gated MLP of n

and run on this library's operators: add_rmsnorm and gated_mlp with their gradients in the training, add_rmsnorm_i8,
matmul_i8 and quantize_i8 in the 8-bit service.  After the training the drift of both services is compared with the closed
form, and the Euler chain is run with the 8-bit one.

    python examples/gated_denoiser.py [--steps 1500] [--chains 4096]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import workloads  # noqa: E402
from paper_2505_03983_b200 import default_ops  # noqa: E402
from paper_2505_03983_b200.autograd import add_rmsnorm, gated_mlp  # noqa: E402

BF16 = torch.bfloat16


class GatedDenoiser:
    """Parameters in float32; each use casts them to bfloat16."""

    def __init__(self, d, width=256, hidden=768, blocks=3, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weights(*shape):
            return (torch.randn(shape, generator=gen, device="cuda") * shape[-1] ** -0.5).requires_grad_()

        self.width = width
        self.first, self.last = weights(width, d + 64), weights(d, width)
        self.norms = [torch.ones(width, device="cuda").requires_grad_() for _ in range(blocks + 1)]
        self.w_in, self.w_out = [weights(2 * hidden, width) for _ in range(blocks)], [weights(width, hidden) for _ in range(blocks)]

    def parameters(self):
        return [self.first, self.last, *self.norms, *self.w_in, *self.w_out]

    def features(self, t, y):
        """The first layer's output: y in units of its standard deviation, and 64 sines and cosines of log t."""
        angle = torch.log(t)[:, None] * torch.exp(torch.linspace(-2, 3, 32, device="cuda"))
        x = torch.cat([y / torch.sqrt(t * (1 + t))[:, None], torch.sin(angle), torch.cos(angle)], dim=1)
        return x.to(BF16) @ self.first.to(BF16).T

    def __call__(self, t, y):
        s, delta = None, self.features(t, y)
        for k, (w_in, w_out) in enumerate(zip(self.w_in, self.w_out)):
            n, s = add_rmsnorm(delta, self.norms[k], s)
            delta = gated_mlp(n, w_in.to(BF16), w_out.to(BF16))
        n, _ = add_rmsnorm(delta, self.norms[-1], s)
        return (n @ self.last.to(BF16).T).float()

    def in_8_bits(self):
        """The same function with the blocks' products in 8-bit integers: weights quantised once, by output channel."""
        ops = default_ops()
        with torch.no_grad():
            blocks = [(w.detach(), *ops.quantize_i8(w_in.detach()), *ops.quantize_i8(w_out.detach()))
                      for w, w_in, w_out in zip(self.norms, self.w_in, self.w_out)]

        @torch.no_grad()
        def drift(t, y):
            s, delta = None, self.features(t, y)
            for w, w_in, in_scale, w_out, out_scale in blocks:
                q, scale, s = ops.add_rmsnorm_i8(delta, w, residual=s)
                gate_up = ops.matmul_i8(q, scale, w_in, in_scale)
                h, scale = ops.quantize_i8(gate_up, act="silu")
                delta = ops.matmul_i8(h, scale, w_out, out_scale)
            n, _ = ops.add_rmsnorm(delta, self.norms[-1], residual=s)
            return (n @ self.last.to(BF16).T).float()

        return drift


def run(steps=1500, batch=4096, chains=4096, width=256, hidden=768, blocks=3, seed=0, log=print):
    wl = workloads.make("cfg1_gmm2d")
    torch.manual_seed(seed)
    means, weights = torch.tensor(wl.means, device="cuda"), torch.tensor(wl.weights, device="cuda")
    t_grid = torch.tensor(wl.t, device="cuda", dtype=torch.float32)

    def draw(n):
        x = means[torch.multinomial(weights, n, replacement=True)] + wl.sigma * torch.randn(n, wl.d, device="cuda")
        t = t_grid[torch.randint(1, wl.K, (n,), device="cuda")] * torch.rand(n, device="cuda").clamp_min(1e-3)
        return x, t, t[:, None] * x + torch.sqrt(t)[:, None] * torch.randn(n, wl.d, device="cuda")

    def closed_form(t, y):
        var = 1 + t[:, None] * wl.sigma ** 2  # y | component j ~ N(t c_j, t (1 + t s^2))
        off = y[:, None] - t[:, None, None] * means
        p = torch.softmax(torch.log(weights) - off.square().sum(-1) / (2 * t[:, None] * var), dim=1)
        return (p[..., None] * (means + wl.sigma ** 2 * off / var[..., None])).sum(1)

    net = GatedDenoiser(wl.d, width, hidden, blocks, seed)
    opt = torch.optim.Adam(net.parameters(), lr=2e-3, betas=(0.9, 0.98))
    schedule = torch.optim.lr_scheduler.LambdaLR(opt, lambda k: min(1.0, (k + 1) / 50) * 0.5 * (1 + math.cos(math.pi * k / steps)))
    losses = []
    for k in range(steps):
        x, t, y = draw(batch)
        loss = (net(t, y) - x).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        schedule.step()
        if k % max(1, steps // 10) == 0 or k == steps - 1:
            losses.append(float(loss.detach()))
            log(f"step {k:5d}  loss {losses[-1]:.4f}")

    served = net.in_8_bits()
    _, t, y = draw(chains)
    with torch.no_grad():
        exact, wide, narrow = closed_form(t, y), net(t, y), served(t, y)

    def rms(a):
        return float(a.square().mean().sqrt())

    report = {"losses": losses, "drift_rms": rms(exact), "error_16": rms(wide - exact), "error_8": rms(narrow - exact), "gap": rms(narrow - wide)}
    # Eq. 7 with the 8-bit drift, from the first grid point after 0 (y_0 = 0 has the drift E[x*], the mixture's mean)
    state = (t_grid[1] - t_grid[0]) * (weights @ means).expand(chains, -1) + (t_grid[1] - t_grid[0]).sqrt() * torch.randn(chains, wl.d, device="cuda")
    for i in range(1, wl.K):
        eta = t_grid[i + 1] - t_grid[i]
        state = state + eta * served(t_grid[i].expand(chains), state) + eta.sqrt() * torch.randn_like(state)
    sample = state / t_grid[-1]
    near = torch.cdist(sample, means).min(dim=1)
    report["near_a_component"] = float((near.values < 4 * wl.sigma).float().mean())
    report["components_hit"] = int(near.indices[near.values < 4 * wl.sigma].unique().numel())
    default_ops().check()
    log(f"drift: rms {report['drift_rms']:.3f}; off the closed form by {report['error_16']:.3f} in 16 bits, {report['error_8']:.3f} in 8 bits; "
        f"the two differ by {report['gap']:.3f}")
    log(f"{chains} chains of {wl.K} steps with the 8-bit drift: {100 * report['near_a_component']:.1f} % of the samples within 4 standard "
        f"deviations of a component, {report['components_hit']} of {len(means)} components hit")
    return report


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=1500)
    ap.add_argument("--chains", type=int, default=4096)
    args = ap.parse_args()
    run(steps=args.steps, chains=args.chains)
