"""The operators of a gated residual block against their definitions in 64 bits, element by element.

Every tolerance is a bound that follows from the number formats: U is the unit roundoff of the output's type, a sum of k
products in 32 bits is off by at most GAMMA(k) times the sum of the products' magnitudes, and what an operator rounds on
its way (h, dg and du to 16 bits, the kept projections to 24) enters with its own unit."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}  # smallest magnitudes
TINY = 2.0 ** -100
F64 = torch.float64


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
    got, want = got.to(F64), want.to(F64)
    assert got.shape == want.shape
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), got.numel(), float((off / (bound + 1e-300)).max()), bad.nonzero()[:4].tolist())


def act64(g, act):
    """act, act' and bounds of |act'| and |act''|."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)), 1.1, 0.51
    p = torch.special.ndtr(g)
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 1.13, 0.8


def padded(t, pad, offset=0):
    """The same values as rows of a wider buffer: a row distance of its own, `offset` elements off the allocation."""
    big = torch.full((t.shape[0], t.shape[1] + pad + offset), float("nan") if t.is_floating_point() else 77, dtype=t.dtype, device=t.device)
    view = big[:, offset:offset + t.shape[1]]
    view.copy_(t)
    return view


# ---- norm -----------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (4, 255), (7, 256), (2, 1000), (6, 1001), (9, 1024), (3, 1032), (4, 4095), (5, 4096), (2, 5000),
               (3, 16384), (2, 16385), (1, 20000), (1300, 72), (1200, 1024), (700, 2048), (1500, 333)]


def norm64(x, r, w, eps):
    s = x if r is None else (x.to(F64) + r.to(F64)).to(x.dtype)
    f = s.to(F64)
    rho = 1 / torch.sqrt((f * f).mean(-1, keepdim=True) + eps)
    return s, f, rho, f * rho * (1 if w is None else w.to(F64))


def sum_rounded_like(got, x, r):
    """x + r is exact in 64 bits; rounded to 16 bits by way of 32 it may be off by one more ulp in rare ties."""
    want = x.to(F64) + r.to(F64)
    within(got, want, want.abs() * U[x.dtype] * (1 + 2.0 ** -12) + LEAST[x.dtype], "sum")


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
def test_add_rmsnorm(ops, rows, width, kind):
    t = TYPES[kind]
    x, r, w = rand((rows, width), 1, t), rand((rows, width), 2, t, 2.0), rand((width,), 3, t)
    y, s = ops.add_rmsnorm(x, w, residual=r, eps=1e-5)
    sum_rounded_like(s, x, r)
    _, _, _, want = norm64(s, None, w, 1e-5)  # the norm of what was stored
    within(y, want, want.abs() * (U[t] + 1e-5) + LEAST[t], "y")
    y2, s2 = ops.add_rmsnorm(x, None)
    assert s2 is x
    want = norm64(x, None, None, 1e-6)[3]
    within(y2, want, want.abs() * (U[t] + 1e-5) + LEAST[t], "no residual, no weight")


def check_q8(q, scale, y64, slack=2e-5):
    """q and scale of rows whose exact values are y64, computed with a relative error of at most `slack`."""
    m = y64.abs().amax(-1).clamp_min(TINY)
    within(scale, m / 127, m / 127 * slack, "scale")
    exact = y64 * (127 / m)[..., None]
    within(q, exact, 0.5 + 127 * slack, "q")
    assert int(q.to(torch.int32).abs().max()) <= 127


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
def test_add_rmsnorm_i8(ops, rows, width, kind):
    t = TYPES[kind]
    x, r, w = rand((rows, width), 1, t), rand((rows, width), 2, t, 2.0), rand((width,), 3, torch.float32)
    q, scale, s = ops.add_rmsnorm_i8(x, w, residual=r)
    assert q.dtype == torch.int8 and scale.shape == (rows,)
    sum_rounded_like(s, x, r)
    check_q8(q, scale, norm64(s, None, w, 1e-6)[3])


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
def test_add_rmsnorm_backward(ops, rows, width, kind):
    t = TYPES[kind]
    s, dy, ds, w = rand((rows, width), 1, t, 2.0), rand((rows, width), 2, t), rand((rows, width), 4, t), rand((width,), 3, t)
    dx, dw = ops.add_rmsnorm_backward(dy, s, w, ds=ds)
    _, f, rho, _ = norm64(s, None, w, 1e-6)
    z, dz = f * rho, dy.to(F64) * w.to(F64)
    c = (dz * z).mean(-1, keepdim=True)
    want = rho * (dz - z * c) + ds.to(F64)
    big = rho * (dz.abs() + z.abs() * (dz * z).abs().mean(-1, keepdim=True)) + ds.to(F64).abs()
    within(dx, want, want.abs() * U[t] + big * 1e-5 + LEAST[t], "dx")
    terms = dy.to(F64) * z
    within(dw, terms.sum(0), terms.sum(0).abs() * U[t] + terms.abs().sum(0) * (GAMMA(rows) + 1e-5) + LEAST[t], "dw")
    # float32 weights, no ds, and the two gradients on their own
    w32 = w.float()
    dx2, dw2 = ops.add_rmsnorm_backward(dy, s, w32)
    within(dx2, want - ds.to(F64), (want - ds.to(F64)).abs() * U[t] + big * 1e-5 + LEAST[t], "dx without ds")
    assert dw2.dtype == torch.float32
    within(dw2, terms.sum(0), terms.abs().sum(0) * (GAMMA(rows) + 1e-5), "dw in 32 bits")
    dx3, none = ops.add_rmsnorm_backward(dy, s, w32, need_dweight=False)
    assert none is None and torch.equal(dx3, dx2)


def test_rmsnorm_gradient_against_differences(ops):
    """The directional derivative of sum(dy * y) along random directions, by central differences of the 64-bit definition."""
    rows, width, eps = 5, 96, 1e-3
    s, dy, w = (rand(sh, i).double() for i, sh in enumerate([(rows, width), (rows, width), (width,)]))
    dx, dw = ops.add_rmsnorm_backward(dy.float(), s.float(), w.float(), eps=eps)
    value = lambda a, b: (dy.float().double() * norm64(a, None, b, eps)[3]).sum()  # noqa: E731
    s, w = s.float().double(), w.float().double()
    for k in range(4):
        ps, pw, h = rand((rows, width), 50 + k).double(), rand((width,), 60 + k).double(), 1e-5
        num = (value(s + h * ps, w + h * pw) - value(s - h * ps, w - h * pw)) / (2 * h)
        ana = (dx.double() * ps).sum() + (dw.double() * pw).sum()
        assert abs(num - ana) <= 1e-5 * ((dx.double() * ps).abs().sum() + (dw.double() * pw).abs().sum())


@pytest.mark.parametrize("width", [64, 1000, 1024, 17000])
def test_norm_in_place_sum_and_strides(ops, width):
    """Through the C ABI: s may be stored over x or over the residual; rows of any distance and alignment."""
    import ctypes as C
    from paper_2505_03983_b200 import operators as o
    rows, t = 6, torch.bfloat16
    x, r, w = rand((rows, width), 1, t), rand((rows, width), 2, t), rand((width,), 3, t)
    y0, s0 = ops.add_rmsnorm(x, w, residual=r)
    for pad, off in ((8, 0), (8, 8), (3, 1)):
        y, s = ops.add_rmsnorm(padded(x, pad, off), w, residual=padded(r, pad, off))
        assert torch.equal(s, s0)
        within(y, y0, y0.to(F64).abs() * 2 * U[t], "strided rows")
        for over in ("x", "residual"):
            xs, rs = padded(x, pad, off), padded(r, pad, off)
            out = padded(torch.zeros_like(x), pad, off)
            dst = xs if over == "x" else rs
            a = o._Norm(rows=rows, width=width, type=2, w_type=2, eps=1e-6, x=xs.data_ptr(), ld_x=xs.stride(0), residual=rs.data_ptr(),
                        ld_residual=rs.stride(0), weight=w.data_ptr(), sum=dst.data_ptr(), ld_sum=dst.stride(0), y=out.data_ptr(),
                        ld_y=out.stride(0))
            assert ops.lib.asd_add_rmsnorm(ops._handle, C.byref(a), torch.cuda.current_stream().cuda_stream) == 0
            assert torch.equal(dst, s0) and torch.equal(out, y)
            whole = out.as_strided((rows, out.stride(0)), (out.stride(0), 1), out.storage_offset() - off)
            assert torch.isnan(whole[:, :off]).all() and torch.isnan(whole[:, off + width:]).all()  # nothing beside the rows


@pytest.mark.parametrize("rows,width", [(6, 64), (700, 33), (6, 1000), (1500, 1001), (6, 5000), (6, 9000), (6, 17003)])
def test_norm_gradient_in_place(ops, rows, width):
    """Through the C ABI: dx may be stored over dy or over ds, with dw as if it were not."""
    import ctypes as C
    from paper_2505_03983_b200 import operators as o
    t = torch.bfloat16
    s, dy, ds, w = rand((rows, width), 1, t), rand((rows, width), 2, t), rand((rows, width), 4, t), rand((width,), 3, t)
    dx, dw = ops.add_rmsnorm_backward(dy, s, w, ds=ds)
    for over in ("dy", "ds"):
        v = {"dy": dy.clone(), "ds": ds.clone()}
        got = torch.empty_like(dw)
        a = o._NormBackward(rows=rows, width=width, type=2, w_type=2, eps=1e-6, dy=v["dy"].data_ptr(), ld_dy=width, s=s.data_ptr(), ld_s=width,
                            ds=v["ds"].data_ptr(), ld_ds=width, weight=w.data_ptr(), dx=v[over].data_ptr(), ld_dx=width, dw=got.data_ptr())
        n = C.c_int64()
        assert ops.lib.asd_add_rmsnorm_backward_workspace(ops._handle, C.byref(a), C.byref(n)) == 0
        space = torch.empty(n.value, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = space.data_ptr(), n.value
        assert ops.lib.asd_add_rmsnorm_backward(ops._handle, C.byref(a), torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(v[over], dx) and torch.equal(got, dw), over


def test_norm_rows_that_cannot_be_represented(ops):
    x = rand((6, 640), 1, torch.float32)
    x[1, 5], x[2, 7], x[3, 9] = float("nan"), float("inf"), -float("inf")
    x[4] = 0
    q, scale, _ = ops.add_rmsnorm_i8(x, None)
    assert torch.isnan(scale[1:4]).all() and torch.isfinite(scale[[0, 4, 5]]).all()
    assert not q[1:5].any() and scale[4] > 0
    good = ops.add_rmsnorm_i8(x[[0, 5]].contiguous(), None)
    assert torch.equal(q[[0, 5]], good[0]) and torch.equal(scale[[0, 5]], good[1])
    y, _ = ops.add_rmsnorm(x, None)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 7]) and torch.isnan(y[3, 9]) and not y[4].any()


# ---- rows in 8 bits -------------------------------------------------------------------------------------

@pytest.mark.parametrize("act", [None, "silu", "gelu"])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 4096), (3, 7), (5, 8), (6, 257), (4, 1000), (3, 1003), (1500, 128), (1400, 1024), (700, 2050),
                                        (2, 16384), (2, 16390), (1, 17001)])
def test_quantize(ops, rows, width, kind, act):
    t = TYPES[kind]
    x = rand((rows, width * (1 if act is None else 2)), 1, t, 2.0)
    q, scale = ops.quantize_i8(x, act=act)
    f = x.to(F64)
    if act is None:
        check_q8(q, scale, f, slack=1e-6)
        assert torch.equal(scale, (f.abs().amax(-1) / 127).float())  # a quotient of 64 bits rounded to 32 is the 32-bit quotient
    else:
        g, u = f[:, :width], f[:, width:]
        # far on the negative side act is a product with 1 + erf, which 32 bits hold to 2^-23 of 1 and not of itself:
        # an error of g u 2^-23 next to a row's largest value
        h = act64(g, act)[0] * u
        m = h.abs().amax(-1).clamp_min(TINY)
        within(scale, m / 127, m / 127 * 2e-5 + (g * u).abs().amax(-1) * 2.0 ** -23, "scale")
        within(q, h * (127 / m)[:, None], 0.5 + 127 * 2e-5 + 127 * (g * u).abs() / m[:, None] * 2.0 ** -22, "q")
    assert torch.equal(ops.quantize_i8(padded(x, 5, 3), act=act)[0], q) and torch.equal(ops.quantize_i8(padded(x, 8), act=act)[1], scale)


# Rows that share a warp, by 4, 2 and 1, with rows missing in the last warp, and more of them than are worked on at once.
NARROW_SHAPES = [(1, 2), (5, 63), (7, 64), (13, 65), (3, 128), (9, 129), (17, 200), (33, 254), (2, 256), (40001, 24), (30001, 64), (20003, 100), (9001, 256)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,width", NARROW_SHAPES)
def test_narrow_rows(ops, rows, width, kind):
    test_add_rmsnorm(ops, rows, width, kind)
    test_add_rmsnorm_i8(ops, rows, width, kind)
    test_add_rmsnorm_backward(ops, rows, width, kind)
    for act in (None, "silu", "gelu"):
        test_quantize(ops, rows, width, kind, act)


@pytest.mark.parametrize("width", [24, 33, 64, 200])
def test_narrow_rows_that_cannot_be_represented(ops, width):
    """An infinity and a NaN stay in their rows, whose neighbours share the warp; rows of zeros with eps."""
    x = rand((37, width), 1)
    x[3], x[9, width // 2], x[20, 0] = 0.0, float("inf"), float("nan")
    others = [i for i in range(37) if i not in (9, 20)]
    y, _ = ops.add_rmsnorm(x, None)
    assert torch.isfinite(y[others]).all() and torch.isnan(y[20]).all() and torch.isnan(y[9, width // 2])
    q, scale, _ = ops.add_rmsnorm_i8(x, None)
    assert not q[[3, 9, 20]].any() and torch.isnan(scale[[9, 20]]).all() and torch.isfinite(scale[others]).all()
    q, scale = ops.quantize_i8(x)
    assert not q[[3, 9, 20]].any() and torch.isnan(scale[[9, 20]]).all() and torch.isfinite(scale[others]).all()
    dx, _ = ops.add_rmsnorm_backward(rand((37, width), 2), x, None)
    assert torch.isfinite(dx[others]).all() and torch.isnan(dx[20]).all()


def test_quantize_edges(ops):
    x = torch.zeros((5, 40), device="cuda")
    x[1], x[2, 3], x[3, 4] = 1e-38, float("inf"), float("nan")
    x[4] = 3e38
    q, scale = ops.quantize_i8(x)
    assert not q[:4].any() and (q[4] == 127).all()
    assert torch.isnan(scale[2:4]).all() and (scale[:2] == torch.tensor(TINY, device="cuda").float() / 127).all() and scale[4] > 0
    empty = ops.quantize_i8(torch.zeros((0, 40), device="cuda"))
    assert empty[0].shape == (0, 40) and empty[1].shape == (0,)


# ---- 8-bit product --------------------------------------------------------------------------------------

MATMUL_SHAPES = [(1, 1, 1), (1, 64, 128), (2, 4096, 640), (3, 17, 5), (8, 1000, 1001), (15, 129, 255), (16, 2048, 512), (17, 33, 130), (31, 512, 100),
                 (33, 96, 72), (64, 320, 1024), (65, 640, 129), (100, 1111, 77), (128, 256, 256), (129, 4100, 300), (200, 16, 1000), (256, 1024, 256),
                 (257, 1024, 513), (300, 3000, 1000), (1000, 200, 2000), (2100, 72, 520), (5000, 130, 1003), (4100, 257, 2049)]


def eight(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int8)


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,out", MATMUL_SHAPES)
def test_matmul_i8(ops, rows, k, out, kind):
    t = TYPES[kind]
    a, b = eight((rows, k), 1), eight((out, k), 2)
    sa, sb = rand((rows,), 3).abs() * 0.01 + 1e-4, rand((out,), 4).abs() * 0.01 + 1e-4
    bias = rand((out,), 5)
    total = a.to(F64) @ b.to(F64).T  # whole numbers: exact
    for bb in (None, bias):
        y = ops.matmul_i8(a, sa, b, sb, bias=bb, dtype=t)
        want = total * sa.to(F64)[:, None] * sb.to(F64)
        size = want.abs()
        if bb is not None:
            want = want + bb.to(F64)
            size = size + bb.to(F64).abs()
        # int32 to fp32, two products and a sum: four roundings of 2^-24, then the type's own
        within(y, want, want.abs() * U[t] + size * 4 * 2.0 ** -24 + LEAST[t], "y")


def test_matmul_i8_is_exact(ops):
    """With scales of 1 and sums below 2^24 the fp32 result is the integer itself: no product is lost or doubled, at every
    k-block, row and column, and at the extreme -128 * -128."""
    for rows, k, out in ((1, 1030, 300), (9, 1030, 300), (40, 1030, 300), (300, 1030, 300)):
        one = torch.ones
        for a, b in ((eight((rows, k), 1), eight((out, k), 2)), (torch.full((rows, k), -128, dtype=torch.int8, device="cuda"),) * 2):
            b = b[:out] if b.shape[0] >= out else b.expand(1, -1, -1).reshape(-1, k)[:1].repeat(out, 1)
            y = ops.matmul_i8(a, one(rows, device="cuda"), b, one(out, device="cuda"), dtype=torch.float32)
            assert torch.equal(y.to(F64), a.to(F64) @ b.to(F64).T)


@pytest.mark.parametrize("rows", [1, 5, 40, 300])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_matmul_i8_strides(ops, rows, kind):
    t, k, out = TYPES[kind], 208, 304
    a, b, sa, sb = eight((rows, k), 1), eight((out, k), 2), rand((rows,), 3).abs(), rand((out,), 4).abs()
    y = ops.matmul_i8(a, sa, b, sb, dtype=t)
    for pad, off in ((16, 0), (16, 16), (1, 0), (5, 3)):
        assert torch.equal(ops.matmul_i8(padded(a, pad, off), sa, padded(b, pad, off), sb, dtype=t), y)
    assert torch.equal(ops.matmul_i8(a.reshape(1, rows, k), sa.reshape(1, rows), b, sb, dtype=t)[0], y)
    assert torch.equal(ops.matmul_i8(a.T.contiguous().T, sa, b.T.contiguous().T, sb, dtype=t), y)


# ---- gated MLP ------------------------------------------------------------------------------------------

MLP_SHAPES = [(1, 64, 128), (1, 8, 8), (1, 1, 1), (2, 5, 3), (3, 130, 77), (7, 1024, 520), (8, 256, 264), (13, 72, 320), (16, 512, 1000), (17, 33, 65),
              (32, 320, 640), (40, 1000, 136), (64, 128, 512), (65, 264, 129), (128, 256, 384), (130, 1001, 259), (256, 256, 256), (300, 72, 1000),
              (600, 520, 777), (1030, 129, 300), (2048, 512, 512), (5000, 72, 1001), (4097, 257, 640)]


def mlp_data(rows, width, hidden, t):
    x, dy = rand((rows, width), 1, t), rand((rows, width), 2, t)
    return x, dy, rand((2 * hidden, width), 3, t, width ** -0.5), rand((width, hidden), 4, t, hidden ** -0.5)


def mlp64(x, dy, w_in, w_out, act, t):
    """Results of the definition, and bounds of what the formats may change in them."""
    h_ = w_in.shape[0] // 2
    x, dy, wi, wo = (v.to(F64) for v in (x, dy, w_in, w_out))
    u16, width, rows = U[t], x.shape[1], x.shape[0]
    gu, gu_size = x @ wi.T, x.abs() @ wi.abs().T
    g, u = gu[:, :h_], gu[:, h_:]
    e_gu = gu_size * GAMMA(width)
    e_g, e_u = e_gu[:, :h_], e_gu[:, h_:]
    a, da, l1, l2 = act64(g, act)
    h = a * u
    a_err = l1 * e_g + (a.abs() + g.abs() * 2.0 ** -22) * 2.0 ** -19  # the approximate exponential, reciprocal and erf
    e_h = a_err * u.abs() + (a.abs() + a_err) * e_u
    e_h = e_h + (h.abs() + e_h) * u16 + LEAST[t]
    out = {}
    y = h @ wo.T
    out["y"] = (y, y.abs() * u16 + (e_h + (h.abs() + e_h) * GAMMA(h_)) @ wo.abs().T * (1 + u16) + LEAST[t])
    # backward, from the gate's factors kept in 24 bits: the bound is that of g and u themselves kept so, which is wider
    k_g, k_u = e_g + (g.abs() + e_g) * 2.0 ** -15, e_u + (u.abs() + e_u) * 2.0 ** -15
    dh = dy @ wo
    e_dh = (dy.abs() @ wo.abs()) * GAMMA(width)
    a_err = l1 * k_g + (a.abs() + g.abs() * 2.0 ** -22) * 2.0 ** -19
    da_err = l2 * k_g + 2.0 ** -18
    dg, du = dh * u * da, dh * a
    e_du = a_err * dh.abs() + (a.abs() + a_err) * e_dh
    e_dg = (da.abs() + da_err) * (dh.abs() * k_u + (u.abs() + k_u) * e_dh) + dh.abs() * u.abs() * da_err
    e_du = e_du + (du.abs() + e_du) * u16 + LEAST[t]
    e_dg = e_dg + (dg.abs() + e_dg) * u16 + LEAST[t]
    d, e = torch.cat([dg, du], 1), torch.cat([e_dg, e_du], 1)
    for name, p, ep, q in (("dx", d, e, wi), ("dw_in", d.T, e.T, x), ("dw_out", dy.T, None, None)):
        if name == "dw_out":
            v, size = dy.T @ h, dy.abs().T @ (e_h + (h.abs() + e_h) * GAMMA(rows))
        else:
            v, size = p @ q, (ep + (p.abs() + ep) * GAMMA(p.shape[1])) @ q.abs()
        out[name] = (v, v.abs() * u16 + size * (1 + u16) + LEAST[t])
    return out


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,hidden", MLP_SHAPES)
def test_gated_mlp(ops, rows, width, hidden, kind, act):
    t = TYPES[kind]
    x, dy, wi, wo = mlp_data(rows, width, hidden, t)
    want = mlp64(x, dy, wi, wo, act, t)
    within(ops.gated_mlp(x, wi, wo, act=act), *want["y"], "y, nothing kept")
    y, saved = ops.gated_mlp_forward(x, wi, wo, act=act)
    within(y, *want["y"], "y")
    for name, got in zip(("dx", "dw_in", "dw_out"), ops.gated_mlp_backward(dy, x, wi, wo, saved, act=act)):
        within(got, *want[name], name)


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_gated_mlp_strides_and_parts(ops, rows):
    t, width, hidden = torch.bfloat16, 136, 200
    x, dy, wi, wo = mlp_data(rows, width, hidden, t)
    y0, saved = ops.gated_mlp_forward(x, wi, wo)
    g0 = ops.gated_mlp_backward(dy, x, wi, wo, saved)
    for pad, off in ((8, 0), (8, 8), (1, 0), (5, 3)):
        v = [padded(m, pad, off) for m in (x, dy, wi, wo)]
        y, s = ops.gated_mlp_forward(v[0], v[2], v[3])
        assert torch.equal(y, y0) and torch.equal(ops.gated_mlp(v[0], v[2], v[3]), ops.gated_mlp(x, wi, wo))
        for a, b in zip(ops.gated_mlp_backward(v[1], v[0], v[2], v[3], s), g0):
            assert torch.equal(a, b)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        got = ops.gated_mlp_backward(dy, x, wi, wo, saved, need=need)
        for n, a, b in zip(need, got, g0):
            assert torch.equal(a, b) if n else a is None
    x3 = x.reshape(1, rows, width)
    assert torch.equal(ops.gated_mlp(x3, wi, wo)[0], ops.gated_mlp(x, wi, wo))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,hidden", [(1023, 8, 16), (1985, 40, 31), (2048, 64, 128), (2049, 257, 96), (9999, 520, 1000), (16500, 33, 31),
                                               (20000, 100, 333), (40000, 512, 1280), (65537, 16, 8)])
def test_weight_gradients_of_many_rows(ops, rows, width, hidden, kind):
    """Sums over all rows with few outputs, which are cut into slices: each gradient, and its bits asked for alone and again."""
    t = TYPES[kind]
    x, dy, wi, wo = mlp_data(rows, width, hidden, t)
    want = mlp64(x, dy, wi, wo, "silu", t)
    _, saved = ops.gated_mlp_forward(x, wi, wo)
    got = ops.gated_mlp_backward(dy, x, wi, wo, saved)
    for name, g in zip(("dx", "dw_in", "dw_out"), got):
        within(g, *want[name], name)
    for _ in range(3):
        assert torch.equal(ops.gated_mlp_backward(dy, x, wi, wo, saved, need=(False, True, False))[1], got[1])
        assert torch.equal(ops.gated_mlp_backward(dy, x, wi, wo, saved, need=(False, False, True))[2], got[2])


def test_gated_mlp_gradient_against_differences(ops):
    """Directional derivatives of sum(dy * y) by central differences of the 64-bit definition; what 16 bits round in the
    analytic gradient is bounded by its units."""
    rows, width, hidden, t, act = 24, 40, 56, torch.float16, "gelu"
    x, dy, wi, wo = mlp_data(rows, width, hidden, t)
    _, saved = ops.gated_mlp_forward(x, wi, wo, act=act)
    grads = ops.gated_mlp_backward(dy, x, wi, wo, saved, act=act)
    bounds = mlp64(x, dy, wi, wo, act, t)

    def value(x, wi, wo):
        g, u = (x @ wi.T).chunk(2, -1)
        return (dy.to(F64) * ((act64(g, act)[0] * u) @ wo.T)).sum()

    at = [v.to(F64) for v in (x, wi, wo)]
    for i, name in enumerate(("dx", "dw_in", "dw_out")):
        p, h = rand(at[i].shape, 70 + i).to(F64), 1e-5
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * p, at[i] - h * p
        num = (value(*up) - value(*down)) / (2 * h)
        ana = (grads[i].to(F64) * p).sum()
        assert abs(num - ana) <= (bounds[name][1] * p.abs()).sum() + 1e-6 * abs(num)


def test_gated_mlp_infinities_stay_in_their_rows(ops):
    for rows in (4, 40, 300):
        x, dy, wi, wo = mlp_data(rows, 72, 100, torch.bfloat16)
        y0 = ops.gated_mlp(x, wi, wo)
        x[1, 3], x[2, 0] = float("inf"), float("nan")
        y, saved = ops.gated_mlp_forward(x, wi, wo)
        rest = [r for r in range(rows) if r not in (1, 2)]
        assert torch.equal(y[rest], ops.gated_mlp_forward(torch.where(torch.isfinite(x), x, torch.zeros_like(x)), wi, wo)[0][rest])
        assert not torch.isfinite(y[1]).any() and torch.isnan(y[2]).all() and torch.isfinite(y0).all()
        dx = ops.gated_mlp_backward(dy, x, wi, wo, saved, need=(True, False, False))[0]
        assert torch.isfinite(dx[rest]).all() and not torch.isfinite(dx[2]).any()


# ---- calls ----------------------------------------------------------------------------------------------

def test_zero_rows(ops):
    t = torch.bfloat16
    w, wi, wo = rand((64,), 1, t), rand((32, 64), 2, t), rand((64, 16), 3, t)
    x = torch.empty((0, 64), dtype=t, device="cuda")
    assert ops.add_rmsnorm(x, w, residual=x)[0].shape == (0, 64) and ops.add_rmsnorm_i8(x, w)[1].shape == (0,)
    dx, dw = ops.add_rmsnorm_backward(x, x, w)
    assert dx.shape == (0, 64) and dw.shape == (64,) and not dw.any()
    y, saved = ops.gated_mlp_forward(x, wi, wo)
    dx, dwi, dwo = ops.gated_mlp_backward(x, x, wi, wo, saved)
    assert y.shape == (0, 64) and not dwi.any() and not dwo.any() and dwi.shape == wi.shape
    e = torch.empty((0, 64), dtype=torch.int8, device="cuda")
    assert ops.matmul_i8(e, torch.empty(0, device="cuda"), eight((8, 64), 1), torch.ones(8, device="cuda")).shape == (0, 8)


def test_same_inputs_same_bits_on_any_stream_and_in_a_graph(ops):
    t = torch.bfloat16
    for rows in (4, 60, 400):
        x, dy, wi, wo = mlp_data(rows, 264, 520, t)
        w = rand((264,), 9, t)

        def step():
            n, s = ops.add_rmsnorm(x, w, residual=dy)
            y, saved = ops.gated_mlp_forward(n, wi, wo)
            g = ops.gated_mlp_backward(dy, n, wi, wo, saved)
            q, sc, _ = ops.add_rmsnorm_i8(x, w, residual=dy)
            i8 = ops.matmul_i8(q, sc, *ops.quantize_i8(wi))
            return [y, *g, *ops.add_rmsnorm_backward(g[0], s, w, ds=dy), i8, *ops.quantize_i8(i8, act="silu")]

        first = step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        for _ in range(2):
            graph.replay()
        for a, b, c in zip(first, other, held):
            assert torch.equal(a, b) and torch.equal(a, c)
        ops.check()


def test_refusals(ops):
    from paper_2505_03983_b200 import AsdError
    t = torch.bfloat16
    x, dy, wi, wo = mlp_data(4, 64, 32, t)
    w = rand((64,), 1, t)
    i8 = eight((4, 64), 1)
    one = torch.ones(4, device="cuda")
    _, saved = ops.gated_mlp_forward(x, wi, wo)
    cases = [
        (1, lambda: ops.add_rmsnorm(x.cpu(), w)), (1, lambda: ops.add_rmsnorm(x, w[:32])), (1, lambda: ops.add_rmsnorm(x, w.half())),
        (1, lambda: ops.add_rmsnorm(x, w, residual=x.float())), (1, lambda: ops.add_rmsnorm(x, w, residual=x[:2])),
        (1, lambda: ops.add_rmsnorm(x, w, eps=-1.0)), (1, lambda: ops.add_rmsnorm(x, w, eps=float("nan"))),
        (1, lambda: ops.add_rmsnorm(x.double(), w)), (1, lambda: ops.add_rmsnorm(x[0], w)), (1, lambda: ops.add_rmsnorm(x[:, :0], None)),
        (1, lambda: ops.add_rmsnorm_backward(dy[:2], x, w)), (1, lambda: ops.add_rmsnorm_backward(dy, x, w, ds=dy.float())),
        (1, lambda: ops.quantize_i8(x, act="relu")), (1, lambda: ops.quantize_i8(x[:, :63], act="silu")), (1, lambda: ops.quantize_i8(i8)),
        (1, lambda: ops.matmul_i8(x, one, i8, one)), (1, lambda: ops.matmul_i8(i8, one, i8[:, :32], one)),
        (1, lambda: ops.matmul_i8(i8, one[:3], i8, one)), (1, lambda: ops.matmul_i8(i8, one, i8, one.half())),
        (1, lambda: ops.matmul_i8(i8, one, i8, one, bias=one[:3])), (1, lambda: ops.matmul_i8(i8, one, i8, one, dtype=torch.int32)),
        (2, lambda: ops.matmul_i8(eight((1, 131072), 1), one[:1], eight((1, 131072), 1), one[:1])),
        (2, lambda: ops.gated_mlp(x.float(), wi.float(), wo.float())), (1, lambda: ops.gated_mlp(x, wi.half(), wo)),
        (1, lambda: ops.gated_mlp(x, wi[:63], wo)), (1, lambda: ops.gated_mlp(x, wi, wo.T)), (1, lambda: ops.gated_mlp(x, wi, wo, act=None)),
        (1, lambda: ops.gated_mlp_backward(dy[:2], x, wi, wo, saved)), (1, lambda: ops.gated_mlp_backward(dy, x, wi, wo, saved[:-1])),
    ]
    for k, (status, call) in enumerate(cases):
        with pytest.raises(AsdError) as e:
            call()
        assert e.value.status == status, (k, str(e.value))


def test_refusals_of_the_c_entry_points(ops):
    import ctypes as C
    from paper_2505_03983_b200 import operators as o
    lib, h = ops.lib, ops._handle
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    good = dict(rows=4, width=64, type=2, w_type=2, eps=1e-6, x=x.data_ptr(), ld_x=64, y=torch.zeros_like(x).data_ptr(), ld_y=64)
    for change in (dict(rows=-1), dict(width=0), dict(width=1 << 25), dict(type=3), dict(w_type=1), dict(reserved=1), dict(x=None),
                   dict(ld_x=63), dict(ld_x=1 << 40), dict(x=x.data_ptr() + 1), dict(y=None)):
        assert lib.asd_add_rmsnorm(h, C.byref(o._Norm(**{**good, **change})), st) == 1, change
        assert lib.asd_ops_last_error()
    # a workspace that is missing, too small, or off its boundary
    wi, wo = torch.zeros((66, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((64, 33), dtype=torch.bfloat16, device="cuda")
    space = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    a = o._GatedMlp(rows=4, width=64, hidden=33, type=2, act=1, x=x.data_ptr(), ld_x=64, w_in=wi.data_ptr(), ld_w_in=64, w_out=wo.data_ptr(),
                    ld_w_out=33, y=x.data_ptr(), ld_y=64)
    need = C.c_int64(0)
    assert lib.asd_gated_mlp_forward_workspace(h, C.byref(a), C.byref(need)) == 0 and need.value > 0
    assert lib.asd_gated_mlp_forward(h, C.byref(a), st) == 1 and b"workspace" in lib.asd_ops_last_error()
    a.workspace, a.workspace_bytes = space.data_ptr(), need.value - 1
    assert lib.asd_gated_mlp_forward(h, C.byref(a), st) == 1
    a.workspace, a.workspace_bytes = space.data_ptr() + 128, need.value
    assert lib.asd_gated_mlp_forward(h, C.byref(a), st) == 1
    ops.check()


# ---- gates far on the negative side ---------------------------------------------------------------------

def gate64(g, act):
    """act(g), and what of it 32 bits may lose: the header's bounds of the normal distribution function and the sigmoid, and a product."""
    if act == "silu":
        return g * torch.sigmoid(g), (4 + g.abs() + 1) * 2.0 ** -23
    return g * 0.5 * torch.erfc(-g / math.sqrt(2)), (8 + g * g + 1) * 2.0 ** -23


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(5, 64), (7, 100), (4, 1000), (1300, 264), (3, 1003), (2, 16390), (2, 17000)])
def test_quantize_of_gates_that_are_all_negative(ops, rows, width, kind, act):
    """A row whose largest value is itself far down the gate's tail: it is held to a relative error, not to one of 1."""
    g = torch.rand((rows, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * -2 - 4
    x = torch.cat([g, rand((rows, width), 2)], 1).to(TYPES[kind])
    q, scale = ops.quantize_i8(x, act=act)
    g, u = x[:, :width].to(F64), x[:, width:].to(F64)
    a, slack = gate64(g, act)
    check_q8(q, scale, a * u, slack=2 * (float(slack.max()) + 4 * 2.0 ** -24))


@pytest.mark.parametrize("rows", [4, 64, 2048])
def test_gated_mlp_of_gates_that_are_all_negative(ops, rows):
    """Rows of the identity through the weights, so that g and u are the weights' own values and y is h: rounded once to h, and
    exact from there on."""
    d, t = 64, torch.float16
    g = (torch.rand((d, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * -1 - 4).to(t)
    u = (torch.rand((d, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") * 4096 + 4096).to(t)
    one = torch.eye(d, device="cuda", dtype=t)
    x = one.repeat((rows + d - 1) // d, 1)[:rows]
    for act in ("silu", "gelu"):
        y = ops.gated_mlp(x, torch.cat([g, u]), one, act=act)
        a, slack = gate64(x.to(F64) @ g.to(F64).T, act)
        want = a * (x.to(F64) @ u.to(F64).T)
        within(y, want, want.abs() * (U[t] + slack + 2.0 ** -22), act)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(5, 64), (7, 33), (1300, 200), (4, 1000), (3, 1001), (2, 4096), (2, 5001), (2, 9000)])
def test_norm_gradient_of_very_small_rows(ops, rows, width, kind):
    """Rows whose rho is 10^19 with eps = 0: no factor of the gradient leaves the range of 32 bits while the gradient does not."""
    t = TYPES[kind]
    sign = torch.where(rand((rows, width), 1) < 0, -1.0, 1.0)
    s = ((1 + torch.rand((rows, width), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")) * 1e-19 * sign).to(t)
    dy, w = (100 * (sign + rand((rows, width), 3))).to(t), (1 + 0.1 * rand((width,), 4)).to(t)
    dx, dw = ops.add_rmsnorm_backward(dy, s, w, eps=0.0)
    _, f, rho, _ = norm64(s, None, w, 0.0)
    z, dz = f * rho, dy.to(F64) * w.to(F64)
    want = rho * (dz - z * (dz * z).mean(-1, keepdim=True))
    big = rho * (dz.abs() + z.abs() * (dz * z).abs().mean(-1, keepdim=True))
    within(dx, want, want.abs() * U[t] + big * 1e-5, "dx")
    terms = dy.to(F64) * z
    within(dw, terms.sum(0), terms.sum(0).abs() * U[t] + terms.abs().sum(0) * (GAMMA(rows) + 1e-5), "dw")


def test_first_call_of_a_thread(ops):
    """A thread on which nothing of CUDA has run yet: the first call there is the operator's."""
    import threading
    for rows in (4, 40, 300, 2048):
        x, dy, wi, wo = mlp_data(rows, 256, 512, torch.bfloat16)
        q, scale = ops.quantize_i8(x)
        w = ops.quantize_i8(wi)
        _, saved = ops.gated_mlp_forward(x, wi, wo)
        for f in (lambda: (ops.gated_mlp(x, wi, wo),), lambda: ops.gated_mlp_backward(dy, x, wi, wo, saved), lambda: (ops.matmul_i8(q, scale, *w),),
                  lambda: ops.quantize_i8(x, act="silu"), lambda: ops.add_rmsnorm(x, None, residual=dy)):
            want, got = f(), []
            del want  # its memory, so that none is asked for on the thread
            torch.cuda.synchronize()

            def work():
                try:
                    got.append(f())
                except BaseException as e:  # noqa: B902
                    got.append(e)

            thread = threading.Thread(target=work)
            thread.start()
            thread.join()
            assert not isinstance(got[0], BaseException), (rows, got[0])
            assert all(torch.equal(a, b) for a, b in zip(got[0], f()))


# ---- exact sums, several callers, and the error word ------------------------------------------------------

@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,width,hidden", [(1, 1030, 500), (8, 1030, 500), (40, 1030, 500), (300, 1030, 500), (2050, 1030, 516), (5000, 264, 300),
                                               (9000, 100, 333)])
def test_gated_mlp_is_exact(ops, rows, width, hidden, kind, act):
    """Whole numbers (w_out: 64ths) whose sums stay below 2^24 units, with every gate at 32 or more, where act(g) = g and act'(g) = 1
    in 32 bits: then only the roundings to 16 bits are left, and a product that is lost, doubled or out of place shows."""
    t = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(1)

    def whole(low, high, *shape):
        return torch.randint(low, high + 1, shape, generator=gen, device="cuda").to(F64)

    x, dy, wu, wo = whole(1, 2, rows, width), whole(-1, 1, rows, width), whole(-1, 1, hidden, width), whole(-1, 1, width, hidden) / 64
    wg = torch.zeros((hidden, width), dtype=F64, device="cuda")
    wg.scatter_(1, torch.rand((hidden, width), generator=gen, device="cuda").argsort(1)[:, :40], 1.0)

    def round16(v):
        return v.to(torch.float32).to(t).to(F64)

    g, u = x @ wg.T, x @ wu.T
    h, dh = round16(g * u), dy @ wo
    d = torch.cat([round16(dh * u), round16(dh * g)], 1)
    w_in = torch.cat([wg, wu])
    sums = {"y": (h, wo.T), "dx": (d, w_in), "dw_in": (d.T, x), "dw_out": (dy.T, h)}
    for name, (a, b) in sums.items():
        units = 1 if name == "dw_out" else 64
        assert float((a.abs() @ b.abs()).max()) * units < 2 ** 24, name
    assert float(g.min()) >= 32 and float(u.abs().max()) < 2 ** 15
    v = [m.to(t) for m in (x, w_in, wo)]
    y, saved = ops.gated_mlp_forward(*v, act=act)
    got = dict(zip(("dx", "dw_in", "dw_out"), ops.gated_mlp_backward(dy.to(t), *v, saved, act=act)), y=y)
    assert torch.equal(ops.gated_mlp(*v, act=act), y)
    for name, (a, b) in sums.items():
        assert torch.equal(got[name].to(F64), round16(a @ b)), name


def test_matmul_i8_is_exact_at_the_extremes(ops):
    """-128 times -128, where it is the longest sum below 2^24, beside other values by row, column and place in the sum."""
    one = torch.ones
    for rows, k, out in ((1, 1023, 300), (8, 1023, 300), (40, 1023, 300), (300, 1023, 300), (5000, 1023, 300)):
        a, b = (torch.full((n, k), -128, dtype=torch.int8, device="cuda") for n in (rows, out))
        r, c, i = (torch.arange(n, device="cuda") for n in (rows, out, k))
        a[r, (7 * r + 3) % k] = (r % 100).to(torch.int8)
        b[c, (11 * c + 5) % k] = (c % 90 - 127).to(torch.int8)
        b[:, i % 97 == 13] = 127
        want = a.to(F64) @ b.to(F64).T
        assert float((a.to(F64).abs() @ b.to(F64).abs().T).max()) < 2 ** 24
        y = ops.matmul_i8(a, one(rows, device="cuda"), b, one(out, device="cuda"), dtype=torch.float32)
        assert torch.equal(y.to(F64), want)


def step_of(ops, rows, seed):
    t = torch.bfloat16
    x, dy, wi, wo = mlp_data(rows, 264, 520, t)
    x, w = rand((rows, 264), seed, t), rand((264,), 9, t)

    def step():
        n, s = ops.add_rmsnorm(x, w, residual=dy)
        y, saved = ops.gated_mlp_forward(n, wi, wo)
        g = ops.gated_mlp_backward(dy, n, wi, wo, saved)
        q, sc, _ = ops.add_rmsnorm_i8(x, w, residual=dy)
        i8 = ops.matmul_i8(q, sc, *ops.quantize_i8(wi))
        return [y, *g, *ops.add_rmsnorm_backward(g[0], s, w, ds=dy), i8, *ops.quantize_i8(i8, act="silu")]

    return step


def test_several_streams_and_threads_at_once(ops):
    """One handle, four streams with work in flight together, from one thread and from four: the bits of each alone."""
    import threading
    steps = [step_of(ops, rows, 20 + i) for i, rows in enumerate((4, 60, 400, 1500))]
    alone = [s() for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = [[] for _ in steps]
    for _ in range(10):
        for i, s in enumerate(steps):
            with torch.cuda.stream(streams[i]):
                got[i].append(s())
    torch.cuda.synchronize()
    failed = []

    def work(i):
        try:
            with torch.cuda.stream(streams[i]):
                for _ in range(10):
                    got[i].append(steps[i]())
                streams[i].synchronize()
        except BaseException as e:  # noqa: B902
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(steps))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    for i, runs in enumerate(got):
        assert len(runs) == 20
        for run in runs:
            assert all(torch.equal(a, b) for a, b in zip(run, alone[i])), i
    ops.check()


ASD_ERR_TIMEOUT = 6


def test_check_reports_a_wait_that_ran_out(ops):
    """The word that a kernel sets when it gives up a wait, set here by the host: reported once, by its own status, and no obstacle
    to what comes after it."""
    import ctypes as C
    from paper_2505_03983_b200 import AsdError, AsdOps
    with AsdOps() as other:
        word = C.c_void_p.from_address(other._handle + 8).value  # behind the device's number and that of its SMs
        x = rand((4, 64), 1)
        want = other.quantize_i8(x)
        torch.cuda.synchronize()
        assert C.CDLL("libcuda.so.1").cuMemsetD32_v2(C.c_uint64(word), C.c_uint32(ASD_ERR_TIMEOUT), C.c_size_t(1)) == 0
        with pytest.raises(AsdError) as e:
            other.check()
        assert e.value.status == ASD_ERR_TIMEOUT and "limit" in str(e.value)
        other.check()
        ops.check()
        assert all(torch.equal(a, b) for a, b in zip(other.quantize_i8(x), want))


@pytest.mark.parametrize("rows,width", [(6, 64), (700, 33), (6, 1000), (1500, 1001), (6, 5000), (6, 9000), (6, 17003)])
def test_norm_gradient_parts(ops, rows, width):
    """Each gradient on its own has the bits that it has beside the other; neither is a valid call."""
    t = torch.bfloat16
    s, dy, ds, w = rand((rows, width), 1, t), rand((rows, width), 2, t), rand((rows, width), 4, t), rand((width,), 3, t)
    dx, dw = ops.add_rmsnorm_backward(dy, s, w, ds=ds)
    none, alone = ops.add_rmsnorm_backward(dy, s, w, need_dx=False)
    assert none is None and torch.equal(alone, dw)
    alone, none = ops.add_rmsnorm_backward(dy, s, w, ds=ds, need_dweight=False)
    assert none is None and torch.equal(alone, dx)
    assert ops.add_rmsnorm_backward(dy, s, w, need_dx=False, need_dweight=False) == (None, None)
