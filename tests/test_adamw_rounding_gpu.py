"""Moments in 8 bits whose codes are rounded up with the probability of their fraction: a code is one of the two around its exact place,
its mean is the place, and over thousands of steps the moments stay beside those in 32 bits.

A dither of 16 bits reaches to 2^-16 of a half on either side; SLACK is what the approximate roots may move a place of up to 255 by."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu

F64, SLACK = torch.float64, 1e-4


@pytest.fixture(scope="module")
def ops():
    from paper_2505_03983_b200 import AsdOps
    with AsdOps() as o:
        yield o
        o.check()


def rand(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def state(n):
    return [torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(((n + 255) // 256, 2), device="cuda")]


def counter(n=0):
    return torch.tensor([n, 0], device="cuda")


def blocks(v):
    return torch.nn.functional.pad(v.to(F64), (0, -v.numel() % 256)).view(-1, 256)


def places(m, v):
    """Exact places of the codes, without rounding."""
    a, r = blocks(m), blocks(v).sqrt()
    M, R = a.abs().amax(1, keepdim=True), r.amax(1, keepdim=True)
    n = m.numel()
    return (127 * (a.abs() / M).sqrt() * a.sign()).flatten()[:n], (255 * (r / R).sqrt()).flatten()[:n]


@pytest.mark.parametrize("n,off", [(1 << 20, 0), ((1 << 18) + 77, 0), ((1 << 18) + 77, 1)])
def test_codes_around_their_places(ops, n, off):
    """From zero moments, so that the places are those of 0.1 g and of 0.001 g^2; 0 and the largest stay whole.  A code's mean over n
    elements is off by its deviation of at most a half over sqrt(n); six of them are allowed."""
    g = rand((n,), 1) * torch.exp(rand((n,), 2))
    g[::7] = 0
    want = places(0.1 * g, 0.001 * g.to(F64) ** 2)

    def step(number):
        p, (m, v, s) = torch.zeros(n, device="cuda"), state(n)
        p, m, v = (torch.cat([t[:1]] * off + [t])[off:] for t in (p, m, v))
        ops.adamw([p], [g], [m], [v], counter(number), betas=(0.9, 0.999), scales=[s], unbiased=True)
        return m, v

    first = step(0)
    m, v = (t.to(F64) for t in first)
    pv = torch.where(want[1] > 0, want[1].clamp_min(1.0), want[1])  # a v above 0 has a code of 1 at least
    for code, place in ((m, want[0]), (v, pv)):
        assert float((code - place).abs().max()) < 1 + SLACK
        assert torch.equal(code[::7], torch.zeros_like(code[::7]))
        assert abs(float((code - place).mean())) <= 6 * 0.5 / n ** 0.5 + SLACK
        # the two moments' dithers, and those of neighbours, have nothing to do with one another
        e = code - place
        for k in (1, 2, 4, 8, 32, 256):
            assert abs(float((e[k:] * e[:-k]).mean())) <= 6 * 0.25 / n ** 0.5 + SLACK
    assert abs(float(((m - want[0]) * (v - pv)).mean())) <= 6 * 0.25 / n ** 0.5 + SLACK
    assert int(m.abs().max()) == 127 and int(v.max()) == 255
    again, later = step(0), step(1)
    for a, b, c in zip(first, again, later):
        assert torch.equal(a, b) and not torch.equal(a, c)


def test_codes_go_by_the_place_alone(ops):
    """The same codes wherever the tensor lies, and in whatever list."""
    n = 5000
    g, p, s = rand((n,), 1), torch.zeros(n, device="cuda"), counter()
    m, v, scales = state(n)
    ops.adamw([p], [g], [m], [v], s, scales=[scales], unbiased=True)
    for off in (1, 3, 8):
        q, a, b = (torch.zeros(n + off, dtype=t, device="cuda")[off:] for t in (torch.float32, torch.int8, torch.uint8))
        c, first = torch.zeros_like(scales), [torch.zeros(300, device="cuda"), torch.ones(300, device="cuda"), *state(300)]
        ops.adamw([first[0], q], [first[1], g], [first[2], a], [first[3], b], counter(), scales=[first[4], c], unbiased=True)
        assert torch.equal(p, q) and torch.equal(m, a) and torch.equal(v, b) and torch.equal(scales, c)


@pytest.mark.parametrize("spread", [0.0, 0.2, 1.0])
def test_second_moment_over_many_steps(ops, spread):
    """10000 steps at beta2 = 0.999.  Codes whose mean is kept make v, their fourth power, larger by some 1.5 / q and sqrt(v) by half of
    that, and let it wander by sqrt(2 / q) / 2 of itself about that; five deviations of the mean over the elements are allowed, and
    the bias twice.  Rounded to the nearest the mean is 1.33 (spread 0), 1.036 (0.2)."""
    n = 8192
    size = torch.exp(rand((n,), 3) * spread)
    gen = torch.Generator(device="cuda").manual_seed(4)
    p8, p32, v32, m32 = (torch.zeros(n, device="cuda") for _ in range(4))
    m, v, s = state(n)
    c8, c32 = counter(), counter()
    for _ in range(10000):
        g = torch.randn(n, generator=gen, device="cuda") * size
        ops.adamw([p8], [g], [m], [v], c8, scales=[s], unbiased=True)
        ops.adamw([p32], [g], [m32], [v32], c32)
    ratio = (ops.adamw_moments(m, v, s)[1].to(F64) / v32.to(F64)).sqrt()
    q = 255 * (v32.view(-1, 256) / v32.view(-1, 256).amax(1, keepdim=True)).to(F64) ** 0.25
    bound = float((1.5 / q).mean() + 5 * (1 / (2 * q)).mean().sqrt() / n ** 0.5)
    assert abs(float(ratio.mean()) - 1) <= bound
    # and the steps are of one size: 1 / sqrt(v) has no bias of the first order
    assert abs(float((1 / ratio).mean()) - 1) <= bound


def test_moments_of_a_gradient_that_ends(ops):
    """Half of each block has no gradient after 50 steps, while the other half keeps the scales: m comes to 0 (from a code of 1 it stays
    with a probability of sqrt(0.9) a step: after 1000 steps less than 1e-15 are left) and v falls by 0.999 a step, in the mean."""
    n, k = 4096, 1000
    p, (m, v, s), c = torch.zeros(n, device="cuda"), state(n), counter()
    g = torch.ones(n, device="cuda")
    for _ in range(50):
        ops.adamw([p], [g], [m], [v], c, scales=[s], unbiased=True)
    g[::2] = 0
    before = ops.adamw_moments(m, v, s)[1][::2].to(F64).mean()
    for _ in range(k):
        ops.adamw([p], [g], [m], [v], c, scales=[s], unbiased=True)
    assert not m[::2].any()
    q = v[::2].to(F64).mean()
    after = ops.adamw_moments(m, v, s)[1][::2].to(F64)
    # deviations of 2 / q of v a code's rounding, adding up in its squares over the steps as above; the mean is over 2048
    assert abs(float(after.mean() / (before * 0.999 ** k)) - 1) <= 3 / float(q) + 5 * (2 / float(q)) ** 0.5 / 2048 ** 0.5
    held = p[::2].clone()
    ops.adamw([p], [g], [m], [v], c, scales=[s], unbiased=True, weight_decay=0.0)
    assert torch.equal(p[::2], held)


def test_the_optimizer_rounds_so(ops):
    from paper_2505_03983_b200.optim import AdamW
    n = 3000
    p = rand((n,), 1).requires_grad_()
    q, (m, v, s), c = p.detach().clone(), state(n), counter()
    opt = AdamW([p], lr=1e-2, state_bits=8)
    for k in range(5):
        p.grad = rand((n,), 10 + k)
        opt.step()
        ops.adamw([q], [p.grad], [m], [v], c, lr=1e-2, scales=[s], unbiased=True)
    assert torch.equal(p, q) and torch.equal(opt.state[p]["exp_avg"], m) and torch.equal(opt.state[p]["exp_avg_sq"], v)


def test_refusals(ops):
    from paper_2505_03983_b200 import AsdError
    from paper_2505_03983_b200 import operators as o
    x = torch.zeros((4, 8), device="cuda")
    with pytest.raises(AsdError) as e:
        ops.adamw([x[0]], [x[1]], [x[2]], [x[3]], counter(), unbiased=True)
    assert e.value.status == 1 and "unbiased" in str(e.value)
    at, step = x.data_ptr(), counter()
    t = (o._AdamwTensor * 1)(o._AdamwTensor(n=8, param=at, grad=at, m=at, v=at, scales=at))
    for bits in (256, 32 | 256, 8 | 512, 9):
        a = o._Adamw(count=1, bits=bits, tensors=t, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step.data_ptr())
        assert ops.lib.asd_adamw(ops._handle, C.byref(a), torch.cuda.current_stream().cuda_stream) == 1, bits
    assert step.tolist() == [0, 0]
