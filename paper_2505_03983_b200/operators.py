"""ctypes binding of the operators of a gated residual block (include/asd_ops.h).  Argument marshalling only: outputs and
workspaces are torch tensors allocated on the current stream, and the work is enqueued there.

There is no CPU fallback: if the shared library has not been built, or no CUDA device is present, the calls raise."""
from __future__ import annotations

import ctypes as C
from typing import Optional

from .binding import AsdError, load_library

OPS_SYMBOLS = [
    "asd_ops_create", "asd_ops_destroy", "asd_ops_last_error", "asd_ops_check",
    "asd_add_rmsnorm", "asd_add_rmsnorm_backward", "asd_add_rmsnorm_backward_workspace",
    "asd_quantize_i8", "asd_matmul_i8", "asd_matmul_i8_workspace",
    "asd_gated_mlp_saved", "asd_gated_mlp_forward", "asd_gated_mlp_forward_workspace",
    "asd_gated_mlp_backward", "asd_gated_mlp_backward_workspace",
]
ACT = {None: 0, "silu": 1, "gelu": 2}  # asd_act

_vp, _i32, _i64, _f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float


class _Norm(C.Structure):
    _fields_ = [("rows", _i32), ("width", _i32), ("type", _i32), ("w_type", _i32), ("eps", _f32), ("reserved", _i32),
                ("x", _vp), ("ld_x", _i64), ("residual", _vp), ("ld_residual", _i64), ("weight", _vp),
                ("sum", _vp), ("ld_sum", _i64), ("y", _vp), ("ld_y", _i64), ("scale", _vp)]


class _NormBackward(C.Structure):
    _fields_ = [("rows", _i32), ("width", _i32), ("type", _i32), ("w_type", _i32), ("eps", _f32), ("reserved", _i32),
                ("dy", _vp), ("ld_dy", _i64), ("s", _vp), ("ld_s", _i64), ("ds", _vp), ("ld_ds", _i64), ("weight", _vp),
                ("dx", _vp), ("ld_dx", _i64), ("dw", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class _Quantize(C.Structure):
    _fields_ = [("rows", _i32), ("width", _i32), ("type", _i32), ("act", _i32), ("x", _vp), ("ld_x", _i64),
                ("q", _vp), ("ld_q", _i64), ("scale", _vp)]


class _MatmulI8(C.Structure):
    _fields_ = [("rows", _i32), ("out", _i32), ("k", _i32), ("out_type", _i32), ("a", _vp), ("ld_a", _i64),
                ("b", _vp), ("ld_b", _i64), ("a_scale", _vp), ("b_scale", _vp), ("bias", _vp), ("y", _vp), ("ld_y", _i64),
                ("workspace", _vp), ("workspace_bytes", _i64)]


class _GatedMlp(C.Structure):
    _fields_ = [("rows", _i32), ("width", _i32), ("hidden", _i32), ("type", _i32), ("act", _i32), ("reserved", _i32),
                ("x", _vp), ("ld_x", _i64), ("w_in", _vp), ("ld_w_in", _i64), ("w_out", _vp), ("ld_w_out", _i64),
                ("y", _vp), ("ld_y", _i64), ("saved", _vp), ("workspace", _vp), ("workspace_bytes", _i64)]


class _GatedMlpBackward(C.Structure):
    _fields_ = [("rows", _i32), ("width", _i32), ("hidden", _i32), ("type", _i32), ("act", _i32), ("reserved", _i32),
                ("dy", _vp), ("ld_dy", _i64), ("x", _vp), ("ld_x", _i64), ("w_in", _vp), ("ld_w_in", _i64),
                ("w_out", _vp), ("ld_w_out", _i64), ("saved", _vp), ("dx", _vp), ("ld_dx", _i64),
                ("dw_in", _vp), ("ld_dw_in", _i64), ("dw_out", _vp), ("ld_dw_out", _i64),
                ("workspace", _vp), ("workspace_bytes", _i64)]


_LIB = None


def _library():
    """The shared library with the operators' prototypes declared."""
    global _LIB
    if _LIB is None:
        lib = load_library()
        lib.asd_ops_last_error.restype, lib.asd_ops_last_error.argtypes = C.c_char_p, []
        lib.asd_ops_destroy.restype, lib.asd_ops_destroy.argtypes = None, [_vp]
        lib.asd_ops_create.argtypes = [C.POINTER(_vp)]
        lib.asd_ops_check.argtypes = [_vp, _vp]
        for name, args in (("add_rmsnorm", _Norm), ("add_rmsnorm_backward", _NormBackward), ("quantize_i8", _Quantize),
                           ("matmul_i8", _MatmulI8), ("gated_mlp_forward", _GatedMlp),
                           ("gated_mlp_backward", _GatedMlpBackward)):
            getattr(lib, "asd_" + name).argtypes = [_vp, C.POINTER(args), _vp]
            if hasattr(lib, "asd_" + name + "_workspace"):
                getattr(lib, "asd_" + name + "_workspace").argtypes = [_vp, C.POINTER(args), C.POINTER(_i64)]
        lib.asd_gated_mlp_saved.argtypes = [_vp, C.POINTER(_GatedMlp), C.POINTER(_i64)]
        for name in OPS_SYMBOLS:
            if name not in ("asd_ops_last_error", "asd_ops_destroy"):
                getattr(lib, name).restype = C.c_int
        _LIB = lib
    return _LIB


def _require(ok, message: str):
    if not ok:
        raise AsdError(1, message)


def _gate(act):
    _require(act in ("silu", "gelu"), f'act must be "silu" or "gelu": {act!r}')
    return ACT[act]


class AsdOps:
    """A handle of the operators on one device (the current one): asd_ops_create on construction, asd_ops_destroy on
    close().  It keeps nothing of its inputs; calls may come from several streams.

    Tensors are CUDA tensors of two or more dimensions, whose last one is the row; leading dimensions are rows.  Rows may
    be strided; a tensor whose last dimension is not contiguous is copied first.  Results are new tensors."""

    def __init__(self):
        import torch
        if not torch.cuda.is_available():
            raise AsdError(4, "no CUDA device: the ASD library has no CPU path")
        self._torch = torch
        self._types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # asd_type
        self.lib = _library()
        torch.cuda.init()
        self.device = torch.cuda.current_device()
        torch.cuda.current_stream()  # the device's context exists before the library asks for it
        self._handle = _vp()
        self._check(self.lib.asd_ops_create(C.byref(self._handle)))

    # -- helpers -------------------------------------------------------------------------
    def _check(self, st: int):
        if st != 0:
            raise AsdError(st, self.lib.asd_ops_last_error().decode())

    def close(self):
        if getattr(self, "_handle", None):
            self.lib.asd_ops_destroy(self._handle)
            self._handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t, name, width=None, dtype=None):
        """(matrix of t's rows, distance of two rows)."""
        _require(isinstance(t, self._torch.Tensor) and t.is_cuda and t.device.index == self.device,
                 f"{name} must be a tensor on cuda:{self.device}")
        _require(t.dim() >= 2, f"{name} must have two or more dimensions: it has {t.dim()}")
        _require(width is None or t.shape[-1] == width, f"{name}: rows of {t.shape[-1]}, expected {width}")
        _require(dtype is None or t.dtype == dtype, f"{name}: {t.dtype}, expected {dtype}")
        _require(t.shape[-1] > 0, f"{name}: rows without elements")
        if t.dim() != 2:
            t = t.reshape(-1, t.shape[-1])
        n, w = t.shape
        if w > 1 and t.stride(1) != 1 or n > 1 and t.stride(0) < w:
            t = t.contiguous()
        return t, (t.stride(0) if n > 1 else w)

    def _vector(self, t, name, n, dtype=None):
        _require(isinstance(t, self._torch.Tensor) and t.is_cuda and t.device.index == self.device,
                 f"{name} must be a tensor on cuda:{self.device}")
        _require(t.dim() == 1 and t.shape[0] == n, f"{name} must have the shape ({n},): {tuple(t.shape)}")
        _require(dtype is None or t.dtype == dtype, f"{name}: {t.dtype}, expected {dtype}")
        return t.contiguous()

    def _type(self, t, name):
        _require(t.dtype in self._types, f"{name}: unsupported type {t.dtype}")
        return self._types[t.dtype]

    def _new(self, shape, dtype):
        return self._torch.empty(shape, dtype=dtype, device=self._torch.device("cuda", self.device))

    def _call(self, name, args):
        """asd_<name> on the current stream, with the workspace that it asks for."""
        query = getattr(self.lib, "asd_" + name + "_workspace", None)
        if query is not None:
            need = _i64(0)
            self._check(query(self._handle, C.byref(args), C.byref(need)))
            if need.value:
                space = self._new((need.value,), self._torch.uint8)
                args.workspace, args.workspace_bytes = space.data_ptr(), need.value
        self._check(getattr(self.lib, "asd_" + name)(self._handle, C.byref(args),
                                                     self._torch.cuda.current_stream(self.device).cuda_stream))

    def check(self):
        """Synchronises the current stream; raises ASD_ERR_TIMEOUT if a kernel of this handle gave up a wait."""
        self._check(self.lib.asd_ops_check(self._handle, self._torch.cuda.current_stream(self.device).cuda_stream))

    # -- norm ------------------------------------------------------------------------------
    def _norm(self, x, weight, residual, eps, q8):
        torch = self._torch
        kind = self._type(x, "x")
        shape, w = x.shape, x.shape[-1]
        a = _Norm()
        m, a.ld_x = self._rows(x, "x")
        a.rows, a.width, a.type, a.eps, a.x = m.shape[0], w, kind, eps, m.data_ptr()
        if residual is not None:
            _require(residual.shape == shape, f"residual: {tuple(residual.shape)}, expected {tuple(shape)}")
            r, a.ld_residual = self._rows(residual, "residual", dtype=x.dtype)
            a.residual = r.data_ptr()
        a.w_type = kind
        if weight is not None:
            weight = self._vector(weight, "weight", w)
            a.w_type, a.weight = self._type(weight, "weight"), weight.data_ptr()
        total = self._new(shape, x.dtype) if residual is not None else x
        if residual is not None:
            a.sum, a.ld_sum = total.data_ptr(), w
        y = self._new(shape, torch.int8 if q8 else x.dtype)
        a.y, a.ld_y = y.data_ptr(), w
        scale = self._new(shape[:-1], torch.float32) if q8 else None
        if q8 and a.rows:
            a.scale = scale.data_ptr()
        self._call("add_rmsnorm", a)
        return y, scale, total

    def add_rmsnorm(self, x, weight, residual=None, eps=1e-6):
        """(y, s): s = x + residual in the type of x (x itself without a residual), y its root-mean-square norm times
        weight ([width], of x's type or float32; None: 1)."""
        y, _, s = self._norm(x, weight, residual, eps, False)
        return y, s

    def add_rmsnorm_i8(self, x, weight, residual=None, eps=1e-6):
        """(q, scale, s): as add_rmsnorm, with y ~ q * scale[..., None] in int8 and a float32 scale per row."""
        return self._norm(x, weight, residual, eps, True)

    def add_rmsnorm_backward(self, dy, s, weight, ds=None, eps=1e-6, need_dweight=True):
        """(dx, dweight) of add_rmsnorm from the gradients dy of y and ds of s (None: 0); dx is the gradient of x and of
        the residual alike, dweight has weight's type (s's without a weight), or is None if it is not needed."""
        kind = self._type(s, "s")
        shape, w = s.shape, s.shape[-1]
        a = _NormBackward()
        _require(dy.shape == shape, f"dy: {tuple(dy.shape)}, expected {tuple(shape)}")
        m, a.ld_s = self._rows(s, "s")
        g, a.ld_dy = self._rows(dy, "dy", dtype=s.dtype)
        a.rows, a.width, a.type, a.eps, a.s, a.dy = m.shape[0], w, kind, eps, m.data_ptr(), g.data_ptr()
        if ds is not None:
            _require(ds.shape == shape, f"ds: {tuple(ds.shape)}, expected {tuple(shape)}")
            d, a.ld_ds = self._rows(ds, "ds", dtype=s.dtype)
            a.ds = d.data_ptr()
        a.w_type = kind
        if weight is not None:
            weight = self._vector(weight, "weight", w)
            a.w_type, a.weight = self._type(weight, "weight"), weight.data_ptr()
        dx = self._new(shape, s.dtype)
        a.dx, a.ld_dx = dx.data_ptr(), w
        dw = None
        if need_dweight:
            dw = self._new((w,), s.dtype if weight is None else weight.dtype)
            a.dw = dw.data_ptr()
        self._call("add_rmsnorm_backward", a)
        return dx, dw

    # -- 8 bits ----------------------------------------------------------------------------
    def quantize_i8(self, x, act: Optional[str] = None):
        """(q, scale) of the rows of x, or, with act "silu" or "gelu", of h = act(g) * u for rows [g | u]."""
        _require(act in ACT, f'act must be None, "silu" or "gelu": {act!r}')
        a = _Quantize()
        a.type, a.act = self._type(x, "x"), ACT[act]
        m, a.ld_x = self._rows(x, "x")
        w = m.shape[1]
        if act is not None:
            _require(w % 2 == 0, f"x: rows [g | u] of an even length, not {w}")
            w //= 2
        q = self._new(x.shape[:-1] + (w,), self._torch.int8)
        scale = self._new(x.shape[:-1], self._torch.float32)
        a.rows, a.width, a.x, a.q, a.ld_q, a.scale = m.shape[0], w, m.data_ptr(), q.data_ptr(), w, scale.data_ptr()
        self._call("quantize_i8", a)
        return q, scale

    def matmul_i8(self, a, a_scale, b, b_scale, bias=None, dtype=None):
        """(a b^T) * a_scale[..., None] * b_scale + bias in `dtype` (bfloat16): a [..., k] and b [out, k] int8, a_scale
        [...] a float32 per row (token), b_scale [out] one per row of b (channel), bias [out] float32 or None."""
        torch = self._torch
        dtype = torch.bfloat16 if dtype is None else dtype
        _require(dtype in self._types, f"unsupported type {dtype}")
        g = _MatmulI8()
        ma, g.ld_a = self._rows(a, "a", dtype=torch.int8)
        _require(b.dim() == 2, "b must be a matrix [out, k]")
        mb, g.ld_b = self._rows(b, "b", width=ma.shape[1], dtype=torch.int8)
        g.rows, g.out, g.k, g.out_type = ma.shape[0], mb.shape[0], ma.shape[1], self._types[dtype]
        _require(a_scale.shape == a.shape[:-1], f"a_scale: {tuple(a_scale.shape)}, expected {tuple(a.shape[:-1])}")
        sa = self._vector(a_scale.reshape(-1), "a_scale", g.rows, torch.float32)
        sb = self._vector(b_scale, "b_scale", g.out, torch.float32)
        g.a, g.b, g.a_scale, g.b_scale = ma.data_ptr(), mb.data_ptr(), sa.data_ptr(), sb.data_ptr()
        if bias is not None:
            bias = self._vector(bias, "bias", g.out, torch.float32)
            g.bias = bias.data_ptr()
        y = self._new(a.shape[:-1] + (g.out,), dtype)
        g.y, g.ld_y = y.data_ptr(), g.out
        self._call("matmul_i8", g)
        return y

    # -- gated MLP ---------------------------------------------------------------------------
    def _mlp_weights(self, a, dtype, w_in, w_out, width):
        _require(w_in.dim() == 2 and w_in.shape[0] % 2 == 0, f"w_in must be a matrix [2 hidden, width]: {tuple(w_in.shape)}")
        wi, a.ld_w_in = self._rows(w_in, "w_in", width=width, dtype=dtype)
        _require(w_out.dim() == 2 and w_out.shape[0] == width, f"w_out must be a matrix [width, hidden]: {tuple(w_out.shape)}")
        wo, a.ld_w_out = self._rows(w_out, "w_out", width=w_in.shape[0] // 2, dtype=dtype)
        a.width, a.hidden, a.w_in, a.w_out = width, w_in.shape[0] // 2, wi.data_ptr(), wo.data_ptr()
        return wi, wo

    def _mlp(self, x, w_in, w_out, act, keep):
        a = _GatedMlp()
        a.type, a.act = self._type(x, "x"), _gate(act)
        m, a.ld_x = self._rows(x, "x")
        a.rows, a.x = m.shape[0], m.data_ptr()
        held = self._mlp_weights(a, x.dtype, w_in, w_out, m.shape[1])  # noqa: F841  (copies live until the call is enqueued)
        y = self._new(x.shape, x.dtype)
        a.y, a.ld_y = y.data_ptr(), m.shape[1]
        saved = None
        if keep:
            need = _i64(0)
            self._check(self.lib.asd_gated_mlp_saved(self._handle, C.byref(a), C.byref(need)))
            saved = self._new((need.value,), self._torch.uint8)
            a.saved = saved.data_ptr() if need.value else None
        self._call("gated_mlp_forward", a)
        return y, saved

    def gated_mlp(self, x, w_in, w_out, act="silu"):
        """(act(x Wg^T) * (x Wu^T)) w_out^T with w_in = [Wg; Wu] [2 hidden, width], w_out [width, hidden]; float16 or
        bfloat16, act "silu" or "gelu"."""
        return self._mlp(x, w_in, w_out, act, False)[0]

    def gated_mlp_forward(self, x, w_in, w_out, act="silu"):
        """(y, saved): gated_mlp, and what gated_mlp_backward needs (opaque bytes)."""
        return self._mlp(x, w_in, w_out, act, True)

    def gated_mlp_backward(self, dy, x, w_in, w_out, saved, act="silu", need=(True, True, True)):
        """(dx, dw_in, dw_out); an entry of `need` that is false leaves out that gradient (None)."""
        a = _GatedMlpBackward()
        a.type, a.act = self._type(x, "x"), _gate(act)
        _require(dy.shape == x.shape, f"dy: {tuple(dy.shape)}, expected {tuple(x.shape)}")
        m, a.ld_x = self._rows(x, "x")
        g, a.ld_dy = self._rows(dy, "dy", dtype=x.dtype)
        a.rows, a.x, a.dy = m.shape[0], m.data_ptr(), g.data_ptr()
        held = self._mlp_weights(a, x.dtype, w_in, w_out, m.shape[1])  # noqa: F841
        f = _GatedMlp(rows=a.rows, width=a.width, hidden=a.hidden, type=a.type, act=a.act)
        size = _i64(0)
        self._check(self.lib.asd_gated_mlp_saved(self._handle, C.byref(f), C.byref(size)))
        _require(saved.numel() == size.value and saved.dtype == self._torch.uint8 and saved.is_cuda and saved.is_contiguous(),
                 f"saved must be what gated_mlp_forward returned: {size.value} bytes for these sizes")
        if size.value:
            a.saved = saved.data_ptr()
        dx = dw_in = dw_out = None
        if need[0]:
            dx = self._new(x.shape, x.dtype)
            a.dx, a.ld_dx = dx.data_ptr(), a.width
        if need[1]:
            dw_in = self._new(w_in.shape, x.dtype)
            a.dw_in, a.ld_dw_in = dw_in.data_ptr(), a.width
        if need[2]:
            dw_out = self._new(w_out.shape, x.dtype)
            a.dw_out, a.ld_dw_out = dw_out.data_ptr(), a.hidden
        self._call("gated_mlp_backward", a)
        return dx, dw_in, dw_out


_DEFAULT = {}


def default_ops() -> AsdOps:
    """The process's handle of the current device, made at its first use."""
    import torch
    if not torch.cuda.is_available():
        raise AsdError(4, "no CUDA device: the ASD library has no CPU path")
    device = torch.cuda.current_device()
    if device not in _DEFAULT:
        _DEFAULT[device] = AsdOps()
    return _DEFAULT[device]
