"""Cases for timing the operators of a gated residual block and for comparing their outputs.

The block is the one that a denoising network is made of where it is wider than this library's residual MLP: the stream is
added to and normalised, two projections make a gate and a value, their product is projected back.  It is trained in 16 bits
and served either in 16 bits or with 8-bit integers.  Four operators make it up:

  norm      s = x + r,  y = s / sqrt(mean(s^2) + eps) * w;  y in 16 bits with its gradients, or in 8 bits with a scale per row
  quantize  h = act(g) * u for a row [g | u], in 8 bits with a scale per row
  matmul    y = (a b^T) * a_scale * b_scale + bias for 8-bit integers a [rows, k] and b [out, k]
  mlp       y = (act(x Wg^T) * (x Wu^T)) Wo^T, with its gradients

`run` computes a case either in plain 32-bit torch operations or, where `own` is true, with this library's calls.  Values that
an operator holds in 8 bits are returned as the values they stand for, in the type of the operator's input.
"""
import math

import torch

own = False

EPS = 1e-6
TINY = 2.0 ** -100  # least magnitude that a row's scale is made from
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MOST_EXACT = 1e13   # operations of a case that are still done in 64 bits (well below a second)


def listed():
    return [
        # one chain's current point in a wide network: one row, where the launch is most of the time
        dict(name="norm_i8_1x4096", op="norm", form="i8", rows=1, width=4096, dtype="bf16"),
        # every drafted point of 512 chains with windows of 64, ahead of an 8-bit projection
        dict(name="norm_i8_32768x1024", op="norm", form="i8", rows=32768, width=1024, dtype="bf16"),
        # a training step's forward and backward at the wide network's width
        dict(name="norm_train_8192x4096", op="norm", form="train", rows=8192, width=4096, dtype="bf16"),
        # the drafted points of one chain with a window of 16, between the two 8-bit projections
        dict(name="quantize_16x4096", op="quantize", rows=16, hidden=4096, act="gelu", dtype="bf16"),
        # the same place in a large batch
        dict(name="quantize_8192x8192", op="quantize", rows=8192, hidden=8192, act="silu", dtype="bf16"),
        # one row through the wide network's gate and value projections: the weights' 8-bit stream is the time
        dict(name="matmul_i8_1x4096x8192", op="matmul", rows=1, k=4096, out=8192, bias=False, dtype="bf16"),
        # nothing a multiple of anything: an observation's features next to an action chunk
        dict(name="matmul_i8_777x1001x1003", op="matmul", rows=777, k=1001, out=1003, bias=True, dtype="f16"),
        # a full batch of drafted points
        dict(name="matmul_i8_8192x4096x8192", op="matmul", rows=8192, k=4096, out=8192, bias=False, dtype="bf16"),
        # one point of one chain in the small network
        dict(name="mlp_1x1024x4096", op="mlp", form="forward", rows=1, width=1024, hidden=4096, act="silu", dtype="bf16"),
        # one chain's window of 16 in the wide network, served in 16 bits
        dict(name="mlp_16x4096x8192", op="mlp", form="forward", rows=16, width=4096, hidden=8192, act="silu", dtype="f16"),
        # a small training step with a ragged batch and hidden size
        dict(name="mlp_train_1000x1000x2731", op="mlp", form="train", rows=1000, width=1000, hidden=2731, act="gelu", dtype="f16"),
        # a full training step
        dict(name="mlp_train_8192x2048x8192", op="mlp", form="train", rows=8192, width=2048, hidden=8192, act="silu", dtype="bf16"),
    ]


def _spread(rng, low, high, step=1):
    """A size between low and high, even over its logarithm; a multiple of `step` in most draws, any number in the others."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if step > 1 and rng.random() < 0.6:
        n = (n + step // 2) // step * step
    return max(low, min(high, n))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    op = rng.choice(["norm", "norm", "quantize", "matmul", "matmul", "mlp", "mlp"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    while True:
        if op == "norm":
            c = dict(op=op, form=rng.choice(["i8", "train"]), rows=_spread(rng, 1, 32768), width=_spread(rng, 64, 8192, 64), dtype=dtype)
            if c["rows"] * c["width"] > 8192 * 8192:
                continue
        elif op == "quantize":
            c = dict(op=op, rows=_spread(rng, 1, 32768), hidden=_spread(rng, 64, 16384, 64), act=rng.choice(["silu", "gelu"]), dtype=dtype)
            if c["rows"] * c["hidden"] > 8192 * 8192:
                continue
        elif op == "matmul":
            c = dict(op=op, rows=_spread(rng, 1, 8192), k=_spread(rng, 64, 8192, 64), out=_spread(rng, 64, 16384, 64),
                     bias=rng.random() < 0.5, dtype=dtype)
        else:
            c = dict(op=op, form=rng.choice(["forward", "train"]), rows=_spread(rng, 1, 8192), width=_spread(rng, 64, 4096, 64),
                     hidden=_spread(rng, 128, 11264, 64), act=rng.choice(["silu", "gelu"]), dtype=dtype)
        if 3072 not in c.values() and work(c)["flops"] <= most:
            return c


def work(case):
    op, n = case["op"], case["rows"]
    e = 2 if case["dtype"] != "f32" else 4
    if op == "norm":
        d = case["width"]
        if case["form"] == "i8":  # x, r in; s, the 8-bit values with their scales, and the values they stand for out
            return {"bytes": n * d * (3 * e + 1 + e) + 4 * n + d * e, "flops": 8.0 * n * d}
        return {"bytes": n * d * e * (4 + 4) + 2 * d * e, "flops": 18.0 * n * d}  # x, r, dy, ds in; s, y, dx out; s again for the backward
    if op == "quantize":
        h = case["hidden"]
        return {"bytes": n * h * (2 * e + 1 + e) + 4 * n, "flops": 10.0 * n * h}
    if op == "matmul":
        k, m = case["k"], case["out"]
        return {"bytes": n * k + m * k + 4 * (n + m) + (4 * m if case["bias"] else 0) + n * m * e, "flops": 2.0 * n * k * m}
    d, h = case["width"], case["hidden"]
    if case["form"] == "forward":
        return {"bytes": e * (3 * d * h + 2 * n * d), "flops": 6.0 * n * d * h}
    return {"bytes": e * (6 * d * h + 4 * n * d), "flops": 18.0 * n * d * h}


# ---- inputs --------------------------------------------------------------------------------------------

def _stream(gen, rows, width, dtype):
    """Rows of a residual stream: near normal, with channels of different size and a few that are much larger."""
    channel = torch.exp(0.4 * torch.randn(width, generator=gen, device="cuda"))
    channel[torch.randint(0, width, (max(1, width // 500),), generator=gen, device="cuda")] *= 8
    return (torch.randn(rows, width, generator=gen, device="cuda") * channel).to(dtype)


def _weights(gen, rows, width, dtype):
    return (torch.randn(rows, width, generator=gen, device="cuda") / math.sqrt(width)).to(dtype)


def _eight_bits(gen, rows, width):
    """Rows as a quantisation by the row's largest value leaves them, and scales."""
    v = torch.randn(rows, width, generator=gen, device="cuda")
    q = torch.round(v * (127 / v.abs().amax(dim=1, keepdim=True))).to(torch.int8)
    return q, torch.exp(0.5 * torch.randn(rows, generator=gen, device="cuda")) * 0.02


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t, n, op = TYPES[case["dtype"]], case["rows"], case["op"]
    s = {"case": case}
    if op == "norm":
        d = case["width"]
        s["x"], s["r"] = _stream(gen, n, d, t) * 0.25, _stream(gen, n, d, t)
        s["w"] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(t)
        if case["form"] == "train":
            s["dy"] = torch.randn(n, d, generator=gen, device="cuda").to(t)
            s["ds"] = (0.5 * torch.randn(n, d, generator=gen, device="cuda")).to(t)
    elif op == "quantize":
        s["x"] = _stream(gen, n, 2 * case["hidden"], t)
    elif op == "matmul":
        s["a"], s["a_scale"] = _eight_bits(gen, n, case["k"])
        s["b"], s["b_scale"] = _eight_bits(gen, case["out"], case["k"])
        s["bias"] = torch.randn(case["out"], generator=gen, device="cuda") if case["bias"] else None
    else:
        d, h = case["width"], case["hidden"]
        s["x"] = torch.randn(n, d, generator=gen, device="cuda").to(t)
        s["w_in"], s["w_out"] = _weights(gen, 2 * h, d, t), _weights(gen, d, h, t)
        if case["form"] == "train":
            s["dy"] = torch.randn(n, d, generator=gen, device="cuda").to(t)
    return s


# ---- the operators in plain 32-bit operations ----------------------------------------------------------

def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * (1 / math.sqrt(2))))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _rows_in_8_bits(y):
    most = y.abs().amax(dim=-1, keepdim=True).clamp_min(TINY)
    return torch.round(y * (127 / most)).to(torch.int8), (most / 127).squeeze(-1)


def _stands_for(q, scale, dtype):
    """The values of 8-bit rows, in `dtype`: one pass, rounded once."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=dtype, device=q.device))


def _plain(s):
    case = s["case"]
    t, op = TYPES[case["dtype"]], case["op"]
    if op == "norm":
        total = (s["x"].float() + s["r"].float()).to(t)  # what is stored is what is normalised
        f, w = total.float(), s["w"].float()
        root = torch.rsqrt(f.square().mean(dim=-1, keepdim=True) + EPS)
        z = f * root
        if case["form"] == "i8":
            q, scale = _rows_in_8_bits(z * w)
            return {"s": total, "y": _stands_for(q, scale, t), "scale": scale}
        dy = s["dy"].float()
        dz = dy * w
        dx = root * (dz - z * (dz * z).mean(dim=-1, keepdim=True)) + s["ds"].float()
        return {"s": total, "y": (z * w).to(t), "dx": dx.to(t), "dw": (dy * z).sum(dim=0).to(t)}
    if op == "quantize":
        g, u = s["x"].float().chunk(2, dim=-1)
        q, scale = _rows_in_8_bits(_act(g, case["act"])[0] * u)
        return {"y": _stands_for(q, scale, t), "scale": scale}
    if op == "matmul":
        y = (s["a"].float() @ s["b"].float().T) * s["a_scale"][:, None] * s["b_scale"]
        return (y if s["bias"] is None else y + s["bias"]).to(t)
    x, w_in, w_out = s["x"].float(), s["w_in"].float(), s["w_out"].float()
    g, u = (x @ w_in.T).chunk(2, dim=-1)
    a, da = _act(g, case["act"])
    h = a * u
    y = h @ w_out.T
    if case["form"] == "forward":
        return y.to(t)
    dy = s["dy"].float()
    dh = dy @ w_out
    both = torch.cat([dh * u * da, dh * a], dim=-1)
    return {"y": y.to(t), "dx": (both @ w_in).to(t), "dw_in": (both.T @ x).to(t), "dw_out": (dy.T @ h).to(t)}


# ---- the same with this library ------------------------------------------------------------------------

def _library(s):
    from paper_2505_03983_b200 import default_ops
    case, ops = s["case"], default_ops()  # this device's handle: it holds an error word, and nothing of the inputs
    t, op = TYPES[case["dtype"]], case["op"]
    if op == "norm":
        if case["form"] == "i8":
            q, scale, total = ops.add_rmsnorm_i8(s["x"], s["w"], residual=s["r"], eps=EPS)
            return {"s": total, "y": _stands_for(q, scale, t), "scale": scale}
        y, total = ops.add_rmsnorm(s["x"], s["w"], residual=s["r"], eps=EPS)
        dx, dw = ops.add_rmsnorm_backward(s["dy"], total, s["w"], ds=s["ds"], eps=EPS)
        return {"s": total, "y": y, "dx": dx, "dw": dw}
    if op == "quantize":
        q, scale = ops.quantize_i8(s["x"], act=case["act"])
        return {"y": _stands_for(q, scale, t), "scale": scale}
    if op == "matmul":
        return ops.matmul_i8(s["a"], s["a_scale"], s["b"], s["b_scale"], bias=s["bias"], dtype=t)
    if case["form"] == "forward":
        return ops.gated_mlp(s["x"], s["w_in"], s["w_out"], act=case["act"])
    y, saved = ops.gated_mlp_forward(s["x"], s["w_in"], s["w_out"], act=case["act"])
    dx, dw_in, dw_out = ops.gated_mlp_backward(s["dy"], s["x"], s["w_in"], s["w_out"], saved, act=case["act"])
    return {"y": y, "dx": dx, "dw_in": dw_in, "dw_out": dw_out}


def run(state):
    return _library(state) if own else _plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def _quantized64(y):
    scale = torch.maximum(torch.amax(torch.abs(y), 1), torch.tensor(TINY, dtype=torch.float64, device=y.device)) / 127.0
    return torch.round(y / scale[:, None]) * scale[:, None], scale


def exact(case, seed):
    if work(case)["flops"] > MOST_EXACT:
        return None
    s = prepare(case, seed)
    wide = {k: v.to(torch.float64) for k, v in s.items() if torch.is_tensor(v)}
    op = case["op"]
    if op == "norm":
        total = (wide["x"] + wide["r"]).to(TYPES[case["dtype"]]).to(torch.float64)
        length = torch.sqrt((total ** 2).sum(1) / case["width"] + EPS)
        y = wide["w"] * total / length[:, None]
        if case["form"] == "i8":
            value, scale = _quantized64(y)
            return {"s": total, "y": value, "scale": scale}
        inner = (wide["dy"] * wide["w"] * total).sum(1) / case["width"]
        dx = wide["ds"] + wide["dy"] * wide["w"] / length[:, None] - total * (inner / length ** 3)[:, None]
        return {"s": total, "y": y, "dx": dx, "dw": (wide["dy"] * total / length[:, None]).sum(0)}

    def gate(g):
        if case["act"] == "silu":
            value = g * torch.sigmoid(g)
            return value, torch.sigmoid(g) + value * torch.sigmoid(-g)
        normal = torch.erfc(-g / math.sqrt(2.0)) / 2.0
        return g * normal, normal + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)

    if op == "quantize":
        h = case["hidden"]
        value, scale = _quantized64(gate(wide["x"][:, :h])[0] * wide["x"][:, h:])
        return {"y": value, "scale": scale}
    if op == "matmul":
        y = torch.mm(wide["a"] * wide["a_scale"][:, None], (wide["b"] * wide["b_scale"][:, None]).t())
        return y + wide["bias"] if case["bias"] else y
    h = case["hidden"]
    w_g, w_u, w_o, x = wide["w_in"][:h], wide["w_in"][h:], wide["w_out"], wide["x"]
    g, u = torch.mm(x, w_g.t()), torch.mm(x, w_u.t())
    a, slope = gate(g)
    y = torch.mm(a * u, w_o.t())
    if case["form"] == "forward":
        return y
    dh = torch.mm(wide["dy"], w_o)
    dg, du = dh * u * slope, dh * a
    return {"y": y, "dx": torch.mm(dg, w_g) + torch.mm(du, w_u),
            "dw_in": torch.cat([torch.mm(dg.t(), x), torch.mm(du.t(), x)]), "dw_out": torch.mm(wide["dy"].t(), a * u)}
