"""Gradients of the linear layer in F16 from a dy in F32 whose size F16 does not hold: that of a mean over many outputs, and a large one.

dz goes to the products times a power of two that brings dy's largest magnitude to 2^14 or more, so that F16 rounds it by U of itself, or by
half of 2^-24 where it is below 2^-14: 2^-39 of that magnitude (LOW)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F16, F64 = torch.float16, torch.float64
U, LEAST, LOW = 2.0 ** -11, 2.0 ** -24, 2.0 ** -39
# one row, a cluster's share of the sum, whole tiles, a weight's gradient in slices, and rows of dy that are not on 16 bytes
SHAPES = [(1, 64, 128), (40, 72, 136), (70, 200, 333), (600, 520, 777), (2111, 1030, 1001), (2048, 512, 512), (5000, 72, 1000)]


def GAMMA(k):
    return (k + 8) * 2.0 ** -23


@pytest.fixture(scope="module")
def ops():
    from paper_2505_03983_b200 import AsdOps
    with AsdOps() as o:
        yield o
        o.check()


def rand(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def within(got, want, bound, what=""):
    off = (got.to(F64) - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), got.numel(), float((off / (bound + 1e-300)).max()), bad.nonzero()[:4].tolist())


def slope64(z, act):
    """act', a bound of |act''|, and what 32 bits lose of act' (tests of the layer itself: (8 + z^2) 2^-23 as far as it counts)."""
    slack = (8 + z.abs().clamp_max(13) ** 2) * 2.0 ** -23 * (1 + z.abs())
    if act is None:
        return torch.ones_like(z), 0.0, 0 * slack
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p)), 0.51, slack
    p = torch.special.ndtr(z)
    return p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 0.8, slack


def check(ops, rows, width, out, act, size, which, wide=True):
    """One of dx and dw, with the operand beside dz of a size that brings the result into F16's range."""
    reach = lambda n: min(2.0 ** 13, max(2.0 ** -9, 1 / (size * n ** 0.5)))  # noqa: E731
    at = reach(out if which == "dx" else rows)  # of w or x; the other one makes z of some units
    other = min(2.0 ** 13, max(2.0 ** -9, 1 / (at * width ** 0.5)))
    x, w = rand((rows, width), 1, F16, other if which == "dx" else at), rand((out, width), 2, F16, at if which == "dx" else other)
    b, dy = rand((out,), 3), rand((rows, out), 4, scale=size)
    if not wide:
        dy = torch.nn.functional.pad(dy, (3, 2))[:, 3:3 + out]
    _, saved = ops.linear_forward(x, w, b, act=act, dtype=torch.float32)
    dx, dw, db = ops.linear_backward(dy, x, w, saved, b, act=act)
    z, e_z = x.to(F64) @ w.to(F64).T + b.to(F64), (x.abs().to(F64) @ w.abs().to(F64).T + b.abs().to(F64)) * GAMMA(width)
    da, l2, slack = slope64(z, act)
    d = dy.to(F64)
    dz, e = d * da, d.abs() * (l2 * e_z + slack) + (d * da).abs() * 2.0 ** -24
    within(db, dz.sum(0), dz.sum(0).abs() * 2.0 ** -24 + e.sum(0) + (dz.abs() + e).sum(0) * GAMMA(rows) + 2.0 ** -149, "db")
    e = e + (dz.abs() + e) * U + d.abs().max() * LOW
    p, ep, q, k = (dz, e, w.to(F64), out) if which == "dx" else (dz.T, e.T, x.to(F64), rows)
    v, s = p @ q, (ep + (p.abs() + ep) * GAMMA(k)) @ q.abs()
    got = dx if which == "dx" else dw
    bound = v.abs() * U + s * (1 + U) + LEAST
    assert got.dtype == F16 and float(v.abs().max()) > 2.0 ** -14
    # a dy of 2^18 beside a w of 2^-9 and over sums of 777 has results of 14272 = 2^9 sqrt(777), of which the largest of 312000, some five
    # times that, are beyond F16, where half a step over 65504 is rounded to infinity
    most, least = v.abs() + s * (1 + U), v.abs() - s * (1 + U)
    beyond = torch.isinf(got)
    assert (beyond == (v.abs() >= 65520))[(most < 65520) | (least >= 65520)].all() and (got[beyond].sign() == v[beyond].sign()).all()
    within(got[~beyond], v[~beyond], bound[~beyond], which)
    for need in ((True, False, False), (False, True, False)):  # alone, the same bits
        for n, a, c in zip(need, ops.linear_backward(dy, x, w, saved, b, act=act, need=need), (dx, dw, db)):
            assert torch.equal(a, c) if n else a is None


@pytest.mark.parametrize("which", ["dx", "dw"])
@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("size", [2.0 ** -26, 2e-6, 1.0, 2.0 ** 18])
@pytest.mark.parametrize("rows,width,out", SHAPES)
def test_sizes(ops, rows, width, out, size, act, which):
    check(ops, rows, width, out, act, size, which)


@pytest.mark.parametrize("which", ["dx", "dw"])
@pytest.mark.parametrize("rows,width,out", SHAPES)
def test_rows_off_16_bytes(ops, rows, width, out, which):
    check(ops, rows, width, out, "silu", 2e-6, which, wide=False)


def test_a_mean_squared_error(ops):
    """The loss of a small network's last layer: its weight's gradient has the error of one rounding of dz beside its own."""
    rows, width, out = 1000, 64, 1001
    x, w, target = rand((rows, width), 1, F16), rand((out, width), 2, F16, width ** -0.5), rand((rows, out), 3)
    y = ops.linear(x, w, dtype=torch.float32)
    dy = (y - target) * (2.0 / y.numel())
    dw = ops.linear_backward(dy, x, w)[1].to(F64)
    want = dy.to(F64).T @ x.to(F64)
    # each of the two roundings is within U of its value, or of LEAST for dw's smallest; their mean square is less than a third of that
    assert (dw - want).norm() <= U * want.norm() + LEAST / 2 * want.numel() ** 0.5


@pytest.mark.parametrize("rows", [40, 600, 3000])
def test_what_is_not_finite_does_not_choose_the_scale(ops, rows):
    x, w, dy = rand((rows, 72), 1, F16), rand((104, 72), 2, F16, 512.0), rand((rows, 104), 3, scale=2e-6)
    dx, dw, _ = ops.linear_backward(dy, x, w)
    dy[1, 3], dy[2, 5] = float("inf"), float("nan")
    dx2, dw2, _ = ops.linear_backward(dy, x, w)
    rest, cols = [i for i in range(rows) if i not in (1, 2)], [j for j in range(104) if j not in (3, 5)]
    assert torch.equal(dx2[rest], dx[rest]) and torch.equal(dw2[cols], dw[cols])
    assert not torch.isfinite(dx2[1]).all() and torch.isnan(dx2[2]).all() and torch.isnan(dw2[5]).all()


def test_extreme_sizes(ops):
    """Nothing, the least that 32 bits hold, and the most: no result that is not a number."""
    x, w = rand((300, 72), 1, F16), rand((104, 72), 2, F16)
    for size in (0.0, 1e-44, 1e-38):
        dx, dw, _ = ops.linear_backward(rand((300, 104), 3, scale=size), x, w)
        assert not dx.any() and not dw.any()
    dx, dw, _ = ops.linear_backward(rand((300, 104), 3).sign() * 3e38, x, w)
    assert torch.isinf(dx).float().mean() > 0.99 and not torch.isnan(dx).any() and not torch.isnan(dw).any()


def test_captured(ops):
    """The power of two is chosen anew by every replay."""
    x, w, b, dy = rand((600, 72), 1, F16), rand((136, 72), 2, F16), rand((136,), 3), rand((600, 136), 4)
    _, saved = ops.linear_forward(x, w, b, act="silu", dtype=torch.float32)
    ops.linear_backward(dy, x, w, saved, b, act="silu")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ops.linear_backward(dy, x, w, saved, b, act="silu")
    for size in (1.0, 1e-7, 300.0):
        dy.copy_(rand((600, 136), 5, scale=size))
        graph.replay()
        for a, c in zip(held, ops.linear_backward(dy, x, w, saved, b, act="silu")):
            assert torch.equal(a, c)
