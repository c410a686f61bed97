"""Cases for timing the operators of a denoiser's training step and for comparing their outputs.

A denoiser of this library is a residual MLP, h <- h + silu(W h + b) between an input and an output layer, or a stack of
gated blocks with norms between them.  Three operators train and serve it next to the gated MLP:

  linear  y = r + act(x W^T + b) with its gradients
  block   between two blocks: n = x / sqrt(mean(x^2) + eps) * w_post,  s = r + alpha * gate * n,
          y = s / sqrt(mean(s^2) + eps) * w;  y in 16 bits with its gradients, or in 8 bits with a scale per row.
          A row of the gate belongs to a run of rows, the points of one chain
  adamw   a step of AdamW over all parameters of a network, moments in 32 bits or in 8 with two scales to 256 of them

`run` computes a case either in plain 32-bit torch operations or, where `own` is true, with this library's calls.  Values that
an operator holds in 8 bits are returned as the values they stand for: y in the type of the operator's input, moments in
bfloat16, whose range holds a squared gradient.
"""
import math

import torch

own = False

EPS = 1e-6
TINY = 2.0 ** -100  # least magnitude that a scale is made from
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 256         # moments to a scale
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01
MOST_EXACT = 1e13   # operations of a case that are still done in 64 bits (well below a second)


def listed():
    return [
        # a hidden layer of the small policy network at one chain's current point: the launch is most of the time
        dict(name="linear_1x1024x1024", op="linear", form="forward", rows=1, width=1024, out=1024, act="silu", residual=True, bias="f32",
             dtype="bf16", out_dtype="bf16"),
        # a hidden layer of the wide network over one chain's window of 16: the weights' stream
        dict(name="linear_16x4096x4096", op="linear", form="forward", rows=16, width=4096, out=4096, act="silu", residual=True, bias="f32",
             dtype="bf16", out_dtype="bf16"),
        # nothing a multiple of anything: an observation's features into a small network, trained, with sums handed on in 32 bits
        dict(name="linear_train_1000x304x1001", op="linear", form="train", rows=1000, width=304, out=1001, act="gelu", residual=False, bias="f16",
             dtype="f16", out_dtype="f32"),
        # a hidden layer of the wide network in a training step
        dict(name="linear_train_8192x4096x4096", op="linear", form="train", rows=8192, width=4096, out=4096, act="silu", residual=True, bias="f32",
             dtype="bf16", out_dtype="bf16"),
        # one chain's current point between two blocks of a wide network
        dict(name="block_1x4096", op="block", form="forward", rows=1, width=4096, group=1, post=True, alpha=1.0, dtype="bf16"),
        # every drafted point of 512 chains with windows of 64 ahead of an 8-bit projection, a gate to each chain
        dict(name="block_i8_32768x1024", op="block", form="i8", rows=32768, width=1024, group=64, post=True, alpha=1.0, dtype="bf16"),
        # a small ragged training step with one learned gate and no norm behind the block
        dict(name="block_train_1001x1003", op="block", form="train", rows=1001, width=1003, group=1001, post=False, alpha=0.5, dtype="f16"),
        # a full training step, a gate to each chain
        dict(name="block_train_8192x4096", op="block", form="train", rows=8192, width=4096, group=64, post=True, alpha=1.0, dtype="bf16"),
        # the fitted network of the two-dimensional mixture: ten tensors, none of them large
        dict(name="adamw_32_3x64", op="adamw", bits=32, layers=3, width=64, inputs=18, out=2, dtype="f32", master=False),
        # the wide network: 16-bit parameters and gradients, moments and master values in 32 bits
        dict(name="adamw_32_6x4096", op="adamw", bits=32, layers=6, width=4096, inputs=3328, out=1024, dtype="bf16", master=True),
        # the same with moments in 8 bits
        dict(name="adamw_8_6x4096", op="adamw", bits=8, layers=6, width=4096, inputs=3328, out=1024, dtype="bf16", master=True),
        # many tensors of an odd size
        dict(name="adamw_8_24x1001", op="adamw", bits=8, layers=24, width=1001, inputs=333, out=113, dtype="f16", master=True),
    ]


def _spread(rng, low, high, step=1):
    """A size between low and high, even over its logarithm; a multiple of `step` in most draws, any number in the others."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if step > 1 and rng.random() < 0.6:
        n = (n + step // 2) // step * step
    return max(low, min(high, n))


def draw(rng):
    op = rng.choice(["linear", "linear", "block", "block", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    most = {m: max(work(c)[m] for c in listed() if c["op"] == op) for m in ("bytes", "flops")}
    while True:
        if op == "linear":
            c = dict(op=op, form=rng.choice(["forward", "train"]), rows=_spread(rng, 1, 16384), width=_spread(rng, 16, 8192, 64),
                     out=_spread(rng, 16, 8192, 64), act=rng.choice(["none", "silu", "gelu"]), residual=rng.random() < 0.5,
                     bias=rng.choice(["none", "f32", dtype]), dtype=dtype, out_dtype=rng.choice([dtype, dtype, "f32"]))
        elif op == "block":
            group = rng.choice([0, 1, 1, 2]) and _spread(rng, 1, 512)  # 0: one gate for all rows
            rows = _spread(rng, 1, 32768)
            if group:
                rows = max(1, rows // group) * group
            c = dict(op=op, form=rng.choice(["forward", "i8", "train", "train"]), rows=rows, width=_spread(rng, 64, 8192, 64), group=group or rows,
                     post=rng.random() < 0.7, alpha=rng.choice([1.0, 0.5]), dtype=dtype)
        else:
            bits = rng.choice([8, 32])
            dtype = rng.choice(["bf16", "f16", "f32"])
            c = dict(op=op, bits=bits, layers=_spread(rng, 1, 28), width=_spread(rng, 64, 4096, 64), inputs=_spread(rng, 18, 3328, 16),
                     out=_spread(rng, 2, 1024), dtype=dtype, master=dtype != "f32")
        if all(work(c)[m] <= most[m] for m in most):
            return c


def _sizes(case):
    """Elements of the network's weights and biases: the input layer, the hidden ones, the output layer."""
    w, n = case["width"], case["layers"]
    return [w * case["inputs"], w] + [w * w, w] * n + [case["out"] * w, case["out"]]


def _padded(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def work(case):
    op = case["op"]
    e = 4 if case["dtype"] == "f32" else 2
    if op == "linear":
        n, k, m = case["rows"], case["width"], case["out"]
        eo = 4 if case["out_dtype"] == "f32" else 2
        few = 0 if case["bias"] == "none" else m * (4 if case["bias"] == "f32" else 2)
        forward = e * (n * k + k * m) + few + n * m * eo * (2 if case["residual"] else 1)
        if case["form"] == "forward":
            return {"bytes": forward, "flops": 2.0 * n * k * m}
        return {"bytes": forward + n * m * eo + e * (n * k + k * m) + few, "flops": 6.0 * n * k * m}  # dy in; dx, dw, db out
    if op == "block":
        n, d, gates = case["rows"], case["width"], case["rows"] // case["group"]
        few = (gates + 1 + (1 if case["post"] else 0)) * d * e
        if case["form"] == "forward":
            return {"bytes": 4 * n * d * e + few, "flops": 12.0 * n * d}
        if case["form"] == "i8":  # as it is read back here: the 8-bit values, and the values they stand for
            return {"bytes": n * d * (3 * e + 1 + e) + 4 * n + few, "flops": 16.0 * n * d}
        return {"bytes": n * d * e * (4 + 4) + 2 * few, "flops": 40.0 * n * d}  # x, r, dy, ds in; s, y, dx, dr out
    n = sum(_sizes(case))
    p = n * (2 * e if not case["master"] else 2 * 4 + e)  # read and written; a master's 16-bit parameter is only written
    if case["bits"] == 32:
        return {"bytes": p + n * (e + 16), "flops": 16.0 * n}
    return {"bytes": p + n * (e + 4) + n * 4 + 16 * (n // BLOCK + 1), "flops": 40.0 * n}  # and both moments once more, in 16 bits


# ---- inputs --------------------------------------------------------------------------------------------

def _stream(gen, rows, width, dtype):
    """Rows of a residual stream: near normal, with channels of different size and a few that are much larger."""
    channel = torch.exp(0.4 * torch.randn(width, generator=gen, device="cuda"))
    channel[torch.randint(0, width, (max(1, width // 500),), generator=gen, device="cuda")] *= 8
    return (torch.randn(rows, width, generator=gen, device="cuda") * channel).to(dtype)


def _split(flat, case):
    """A network's tensors as views of one buffer, each at a multiple of 256 elements."""
    sizes = _sizes(case)
    starts = [sum(_padded(n) for n in sizes[:i]) for i in range(len(sizes))]
    return [flat[at:at + n] for at, n in zip(starts, sizes)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    t, op = TYPES[case["dtype"]], case["op"]
    s = {"case": case}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if op == "linear":
        n, k, m, to = case["rows"], case["width"], case["out"], TYPES[case["out_dtype"]]
        s["x"], s["w"] = normal(n, k).to(t), (normal(m, k) / math.sqrt(k)).to(t)
        s["b"] = None if case["bias"] == "none" else (0.3 * normal(m)).to(TYPES[case["bias"]])
        s["r"] = _stream(gen, n, m, to) if case["residual"] else None
        if case["form"] == "train":
            s["dy"] = normal(n, m).to(to)
    elif op == "block":
        n, d = case["rows"], case["width"]
        s["x"], s["r"] = _stream(gen, n, d, t) * 0.25, _stream(gen, n, d, t)
        s["w"] = (1 + 0.2 * normal(d)).to(t)
        s["w_post"] = (1 + 0.2 * normal(d)).to(t) if case["post"] else None
        s["gate"] = (0.4 + 0.3 * normal(n // case["group"], d)).to(t)
        if case["form"] == "train":
            s["dy"], s["ds"] = normal(n, d).to(t), (0.5 * normal(n, d)).to(t)
    else:
        sizes = _sizes(case)
        total = sum(_padded(n) for n in sizes)
        there = torch.zeros(total, device="cuda")
        for v in _split(there, case):
            v.fill_(1)
        there = there.to(torch.bool)

        def flat(v):  # nothing between one tensor's end and the next one's start
            return torch.where(there, v, torch.zeros((), dtype=v.dtype, device="cuda"))

        value = flat(0.02 * normal(total))
        s["p"], s["master"] = value.to(t), value if case["master"] else None
        size = 1e-3 * torch.exp(normal(total // BLOCK, 1))  # neighbouring gradients are alike in size
        s["g"] = flat((size * normal(total // BLOCK, BLOCK)).flatten()).to(t)
        if case["bits"] == 32:
            s["m"] = flat((0.3 * size * normal(total // BLOCK, BLOCK)).flatten())
            s["v"] = flat((size * (0.5 + 0.2 * normal(total // BLOCK, BLOCK))).square().flatten())
            s["scales"] = None
        else:
            s["m"] = flat(torch.clamp(torch.round(50 * normal(total)), -127, 127).to(torch.int8))
            s["v"] = flat(torch.clamp(torch.round(180 + 30 * normal(total)), 1, 255).to(torch.uint8))
            s["scales"] = torch.stack([size.flatten(), 2 * size.flatten()], dim=1).contiguous()
        s["step"] = torch.tensor([9 + int(seed) % 50, 0], device="cuda")  # the steps taken; the second word is the library's
    return s


# ---- the operators in plain 32-bit operations ----------------------------------------------------------

def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, 1.0
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    p = 0.5 * (1 + torch.erf(z * (1 / math.sqrt(2))))
    return z * p, p + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _rows_in_8_bits(y):
    most = y.abs().amax(dim=-1, keepdim=True).clamp_min(TINY)
    return torch.round(y * (127 / most)).to(torch.int8), (most / 127).squeeze(-1)


def _stands_for(q, scale, dtype):
    """The values of 8-bit rows, in `dtype`: one pass, rounded once."""
    return torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=dtype, device=q.device))


def _plain_linear(s):
    case = s["case"]
    t, to = TYPES[case["dtype"]], TYPES[case["out_dtype"]]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.T
    if s["b"] is not None:
        z = z + s["b"].float()
    y, slope = _act(z, case["act"])
    if s["r"] is not None:
        y = s["r"].float() + y
    if case["form"] == "forward":
        return y.to(to)
    dz = s["dy"].float() * slope
    out = {"y": y.to(to), "dx": (dz @ w).to(t), "dw": (dz.T @ x).to(t)}
    if s["b"] is not None:
        out["db"] = dz.sum(dim=0).to(s["b"].dtype)
    return out


def _plain_block(s):
    case = s["case"]
    t, n, d = TYPES[case["dtype"]], case["rows"], case["width"]
    gates = n // case["group"]
    x, w = s["x"].float(), s["w"].float()
    gate = s["gate"].float()[:, None] * case["alpha"]
    root_x = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) if case["post"] else 1.0
    w_post = s["w_post"].float() if case["post"] else 1.0
    norm = x * root_x
    total = (s["r"].float() + (gate * (norm * w_post).view(gates, -1, d)).view(n, d)).to(t)  # what is stored is what is normalised
    f = total.float()
    root = torch.rsqrt(f.square().mean(dim=-1, keepdim=True) + EPS)
    z = f * root
    if case["form"] == "i8":
        q, scale = _rows_in_8_bits(z * w)
        return {"s": total, "y": _stands_for(q, scale, t), "scale": scale}
    if case["form"] == "forward":
        return {"s": total, "y": (z * w).to(t)}
    dy = s["dy"].float()
    dz = dy * w
    dr = root * (dz - z * (dz * z).mean(dim=-1, keepdim=True)) + s["ds"].float()
    out = {"s": total, "y": (z * w).to(t), "dr": dr.to(t), "dw": (dy * z).sum(dim=0).to(t)}
    through = (dr * norm).view(gates, -1, d).sum(dim=1) * case["alpha"]  # the gradient of gate * w_post, by gate
    out["dgate"] = (through * w_post).to(t)
    dn = (gate * dr.view(gates, -1, d)).view(n, d) * w_post
    if case["post"]:
        out["dw_post"] = (through * s["gate"].float()).sum(dim=0).to(t)
        dn = root_x * (dn - norm * (dn * norm).mean(dim=-1, keepdim=True))
    out["dx"] = dn.to(t)
    return out


def _moments(m, v, scales):
    """The moments that 8-bit codes stand for: m = M (q / 127) |q / 127|, sqrt(v) = R (q / 255)^2."""
    a, b = m.view(-1, BLOCK).float() / 127, v.view(-1, BLOCK).float() / 255
    return (scales[:, :1] * (a * a.abs())).flatten(), (scales[:, 1:] * b.square()).square().flatten()


def _moments_in_8_bits(m, v):
    a, b = m.view(-1, BLOCK), v.view(-1, BLOCK).sqrt()
    scales = torch.stack([a.abs().amax(dim=1), b.amax(dim=1)], dim=1)
    scales = torch.where(scales < TINY, torch.zeros_like(scales), scales)
    low = scales.clamp_min(TINY)
    qm = torch.round(127 * (a.abs() / low[:, :1]).clamp_max(1).sqrt()) * a.sign() * (scales[:, :1] > 0)
    qv = torch.round(255 * (b / low[:, 1:]).clamp_max(1).sqrt()).clamp_min(1) * (b > 0) * (scales[:, 1:] > 0)
    return qm.to(torch.int8).flatten(), qv.to(torch.uint8).flatten(), scales


def _plain_adamw(s):
    case = s["case"]
    s["step"][0] += 1
    t = s["step"][0].double()
    correct1, correct2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).sqrt().float()
    g = s["g"].float()
    m, v = (s["m"], s["v"]) if case["bits"] == 32 else _moments(s["m"], s["v"], s["scales"])
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g.square()
    p = s["master"] if case["master"] else s["p"].float()
    p = p * (1 - LR * DECAY) - (LR / correct1) * m / (v.sqrt() / correct2 + ADAM_EPS)
    s["p"].copy_(p)
    out = {"p": s["p"]}
    if case["master"]:
        s["master"].copy_(p)
        out["master"] = s["master"]
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {**out, "m": s["m"], "v": s["v"]}
    for name, new in zip(("m", "v", "scales"), _moments_in_8_bits(m, v)):
        s[name].copy_(new)
    m, v = _moments(s["m"], s["v"], s["scales"])
    return {**out, "m": m.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain(s):
    return {"linear": _plain_linear, "block": _plain_block, "adamw": _plain_adamw}[s["case"]["op"]](s)


# ---- the same with this library ------------------------------------------------------------------------

def _library(s):
    from paper_2505_03983_b200 import default_ops
    case, ops = s["case"], default_ops()  # this device's handle: it holds an error word, and nothing of the inputs
    t, op = TYPES[case["dtype"]], case["op"]
    if op == "linear":
        act, to = None if case["act"] == "none" else case["act"], TYPES[case["out_dtype"]]
        if case["form"] == "forward":
            return ops.linear(s["x"], s["w"], s["b"], residual=s["r"], act=act, dtype=to)
        y, saved = ops.linear_forward(s["x"], s["w"], s["b"], residual=s["r"], act=act, dtype=to)
        dx, dw, db = ops.linear_backward(s["dy"], s["x"], s["w"], saved, s["b"], act=act)
        return {"y": y, "dx": dx, "dw": dw} if db is None else {"y": y, "dx": dx, "dw": dw, "db": db}
    if op == "block":
        gate = s["gate"][:, None]  # [gates, 1, width] beside [gates, group, width]
        x, r = (s[k].view(gate.shape[0], -1, gate.shape[2]) for k in ("x", "r"))
        how = dict(post_weight=s["w_post"], gate=gate, alpha=case["alpha"], eps=EPS, post_norm=case["post"])
        if case["form"] == "i8":
            q, scale, total = ops.block_rmsnorm_i8(x, r, s["w"], **how)
            q, scale = q.view(s["x"].shape), scale.flatten()
            return {"s": total.view(s["x"].shape), "y": _stands_for(q, scale, t), "scale": scale}
        y, total = ops.block_rmsnorm(x, r, s["w"], **how)
        out = {"s": total.view(s["x"].shape), "y": y.view(s["x"].shape)}
        if case["form"] == "forward":
            return out
        dy, ds = s["dy"].view(x.shape), s["ds"].view(x.shape)
        dx, dr, dw, dw_post, dgate = ops.block_rmsnorm_backward(dy, x, total, s["w"], ds=ds, **how)
        out |= {"dr": dr.view(s["x"].shape), "dw": dw, "dgate": dgate.view(s["gate"].shape), "dx": dx.view(s["x"].shape)}
        return {**out, "dw_post": dw_post} if case["post"] else out
    lists = {k: _split(s[k], case) for k in ("p", "g", "m", "v")}
    masters = _split(s["master"], case) if case["master"] else None
    scales = None
    if case["bits"] == 8:
        scales = [v.view(-1, 2) for v in s["scales"].flatten().split([_padded(n) // BLOCK * 2 for n in _sizes(case)])]
    ops.adamw(lists["p"], lists["g"], lists["m"], lists["v"], s["step"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
              masters=masters, scales=scales)
    out = {"p": s["p"], "master": s["master"]} if case["master"] else {"p": s["p"]}
    if case["bits"] == 32:
        return {**out, "m": s["m"], "v": s["v"]}
    m, v = ops.adamw_moments(s["m"], s["v"], s["scales"], dtype=torch.bfloat16)
    return {**out, "m": m, "v": v}


def run(state):
    return _library(state) if own else _plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------------------

def _exact_linear(case, wide):
    z = torch.mm(wide["x"], wide["w"].t())
    if case["bias"] != "none":
        z += wide["b"]
    if case["act"] == "silu":
        gate = torch.sigmoid(z)
        y, slope = z * gate, gate + z * gate * torch.sigmoid(-z)
    elif case["act"] == "gelu":
        normal = torch.erfc(-z / math.sqrt(2.0)) / 2.0
        y, slope = z * normal, normal + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    else:
        y, slope = z, torch.ones_like(z)
    if case["residual"]:
        y = y + wide["r"]
    if case["form"] == "forward":
        return y
    dz = slope * wide["dy"]
    grads = {"y": y, "dx": torch.mm(dz, wide["w"]), "dw": torch.mm(dz.t(), wide["x"])}
    return grads if case["bias"] == "none" else {**grads, "db": torch.mv(dz.t(), torch.ones_like(dz[:, 0]))}


def _exact_block(case, wide):
    d, group = case["width"], case["group"]
    gate = case["alpha"] * wide["gate"].repeat_interleave(group, 0)
    w_post = wide["w_post"] if case["post"] else torch.ones(d, dtype=torch.float64, device="cuda")
    x = wide["x"]
    length_x = torch.sqrt((x ** 2).sum(1, keepdim=True) / d + EPS) if case["post"] else torch.ones_like(x[:, :1])
    total = (wide["r"] + gate * w_post * x / length_x).to(TYPES[case["dtype"]]).to(torch.float64)
    length = torch.sqrt((total ** 2).sum(1, keepdim=True) / d + EPS)
    y = wide["w"] * total / length
    if case["form"] == "i8":
        scale = torch.maximum(torch.amax(torch.abs(y), 1), torch.tensor(TINY, dtype=torch.float64, device="cuda")) / 127.0
        return {"s": total, "y": torch.round(y / scale[:, None]) * scale[:, None], "scale": scale}
    if case["form"] == "forward":
        return {"s": total, "y": y}
    inner = (wide["dy"] * wide["w"] * total).sum(1, keepdim=True) / d
    dr = wide["ds"] + wide["dy"] * wide["w"] / length - total * inner / length ** 3
    by_gate = torch.stack([c.sum(0) for c in (dr * x / length_x).split(group)]) * case["alpha"] if group < case["rows"] \
        else (dr * x / length_x).sum(0, keepdim=True) * case["alpha"]
    d_in = dr * gate * w_post
    dx = d_in / length_x
    if case["post"]:
        dx = dx - x * ((d_in * x).sum(1, keepdim=True) / d) / length_x ** 3
    out = {"s": total, "y": y, "dr": dr, "dw": (wide["dy"] * total / length).sum(0), "dgate": by_gate * w_post, "dx": dx}
    return {**out, "dw_post": (by_gate * wide["gate"]).sum(0)} if case["post"] else out


def _exact_adamw(case, s, wide):
    t = int(s["step"][0]) + 1
    m, v = wide["m"], wide["v"]
    if case["bits"] == 8:
        scale = wide["scales"].repeat_interleave(BLOCK, 0)
        m = scale[:, 0] * torch.sign(m) * (m / 127.0) ** 2
        v = scale[:, 1] ** 2 * (v / 255.0) ** 4
    m = m + (1.0 - BETA1) * (wide["g"] - m)
    v = v + (1.0 - BETA2) * (wide["g"] ** 2 - v)
    p = wide["master"] if case["master"] else wide["p"]
    ratio = (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + ADAM_EPS)
    p = p - LR * (ratio + DECAY * p)
    out = {"p": p, "master": p} if case["master"] else {"p": p}
    if case["bits"] == 32:
        return {**out, "m": m, "v": v}
    root = torch.sqrt(v).view(-1, BLOCK)
    big_m, big_r = torch.amax(m.abs().view(-1, BLOCK), 1, keepdim=True), torch.amax(root, 1, keepdim=True)
    none_m, none_r = (torch.where(b > 0, b, torch.ones_like(b)) for b in (big_m, big_r))
    level = torch.round(127.0 * torch.sqrt(m.abs().view(-1, BLOCK) / none_m)) / 127.0
    m = big_m * level ** 2 * torch.sign(m.view(-1, BLOCK))
    level = torch.round(255.0 * torch.sqrt(root / none_r))
    level = torch.where((root > 0) & (level < 1), torch.ones_like(level), level) / 255.0
    return {**out, "m": m.flatten(), "v": (big_r * level ** 2).flatten() ** 2}


def exact(case, seed):
    if work(case)["flops"] > MOST_EXACT:
        return None
    s = prepare(case, seed)
    wide = {k: v.to(torch.float64) for k, v in s.items() if torch.is_tensor(v)}
    if case["op"] == "linear":
        return _exact_linear(case, wide)
    return _exact_block(case, wide) if case["op"] == "block" else _exact_adamw(case, s, wide)
