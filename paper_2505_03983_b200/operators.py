"""ctypes binding of the operators of a gated residual block (include/asd_ops.h).  Argument marshalling only: outputs and
workspaces are torch tensors allocated on the current stream, and the work is enqueued there.

There is no CPU fallback: if the shared library has not been built, or no CUDA device is present, the calls raise."""
from __future__ import annotations

import ctypes as C
import struct
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


def _packer(cls):
    """struct.pack of a structure's fields: the same bytes as the structure, in a fraction of its construction's time."""
    return struct.Struct("@" + "".join({_i32: "i", _f32: "f", _i64: "q", _vp: "P"}[f[1]] for f in cls._fields_)).pack


_pack_norm, _pack_norm_backward, _pack_quantize = _packer(_Norm), _packer(_NormBackward), _packer(_Quantize)
_pack_matmul, _pack_mlp, _pack_mlp_backward = _packer(_MatmulI8), _packer(_GatedMlp), _packer(_GatedMlpBackward)

_LIB = None


def _library():
    """The shared library with the operators' prototypes declared.  Argument structures are passed as their bytes."""
    global _LIB
    if _LIB is None:
        lib = load_library()
        lib.asd_ops_last_error.restype, lib.asd_ops_last_error.argtypes = C.c_char_p, []
        lib.asd_ops_destroy.restype, lib.asd_ops_destroy.argtypes = None, [_vp]
        lib.asd_ops_create.argtypes = [C.POINTER(_vp)]
        lib.asd_ops_check.argtypes = [_vp, _vp]
        for name in OPS_SYMBOLS:
            fn = getattr(lib, name)
            if name not in ("asd_ops_last_error", "asd_ops_destroy"):
                fn.restype = C.c_int
            if not name.startswith("asd_ops_"):
                query = name.endswith(("_workspace", "_saved"))
                fn.argtypes = [_vp, _vp, C.POINTER(_i64)] if query else [_vp, _vp, _vp]
        _LIB = lib
    return _LIB


def _fail(message: str):
    raise AsdError(1, message)


def _gate(act):
    return ACT[act] if act == "silu" or act == "gelu" else _fail(f'act must be "silu" or "gelu": {act!r}')


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
        self._i8, self._f32, self._u8 = torch.int8, torch.float32, torch.uint8
        self.lib = _library()
        self.device = torch.cuda.current_device()
        # the current stream's handle, by the shortest way that this torch has
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._stream = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)
        torch.cuda.current_stream().synchronize()  # the device's context exists before the library asks for it
        handle = _vp()
        self._check(self.lib.asd_ops_create(C.byref(handle)))
        self._handle = handle.value

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
        """(t as a matrix of rows, its rows, their length, the distance of two)."""
        if not isinstance(t, self._torch.Tensor) or t.get_device() != self.device:
            _fail(f"{name} must be a tensor on cuda:{self.device}")
        if dtype is not None and t.dtype is not dtype:
            _fail(f"{name}: {t.dtype}, expected {dtype}")
        if t.dim() != 2:
            if t.dim() < 2:
                _fail(f"{name} must have two or more dimensions: it has {t.dim()}")
            if t.shape[-1] == 0:
                _fail(f"{name}: rows without elements")
            t = t.reshape(-1, t.shape[-1])
        n, w = t.shape
        if width is not None and w != width:
            _fail(f"{name}: rows of {w}, expected {width}")
        if t.is_contiguous():
            return (t, n, w, w) if w else _fail(f"{name}: rows without elements")
        step, one = t.stride()
        if w > 1 and one != 1 or n > 1 and step < w:
            t, step = t.contiguous(), w
        return t, n, w, step if n > 1 else w

    def _vector(self, t, name, n, dtype):
        if not isinstance(t, self._torch.Tensor) or t.get_device() != self.device:
            _fail(f"{name} must be a tensor on cuda:{self.device}")
        if t.dim() != 1 or t.shape[0] != n:
            _fail(f"{name} must have the shape ({n},): {tuple(t.shape)}")
        if dtype is not None and t.dtype is not dtype:
            _fail(f"{name}: {t.dtype}, expected {dtype}")
        return t if t.is_contiguous() else t.contiguous()

    def _type(self, t, name):
        kind = self._types.get(getattr(t, "dtype", None))
        return _fail(f"{name} must be a tensor of float32, float16 or bfloat16") if kind is None else kind

    def _weight(self, weight, w, kind):
        """(w_type, weight, its address); without a weight that of the rows' type."""
        if weight is None:
            return kind, None, 0
        weight = self._vector(weight, "weight", w, None)
        return self._type(weight, "weight"), weight, weight.data_ptr()

    def _space(self, query, args):
        """The workspace that a call with these arguments asks for: (tensor or None, address, bytes)."""
        need = _i64()
        st = query(self._handle, args, need)
        if st != 0:
            self._check(st)
        n = need.value
        if not n:
            return None, 0, 0
        space = self._torch.empty(n, dtype=self._u8, device=self.device)
        return space, space.data_ptr(), n

    def check(self):
        """Synchronises the current stream; raises ASD_ERR_TIMEOUT if a kernel of this handle gave up a wait."""
        self._check(self.lib.asd_ops_check(self._handle, self._stream(self.device)))

    # -- norm ------------------------------------------------------------------------------
    def _norm(self, x, weight, residual, eps, q8):
        kind = self._type(x, "x")
        m, n, w, ld = self._rows(x, "x")
        r_ptr = r_ld = s_ptr = s_ld = 0
        total = x
        if residual is not None:
            r, _, _, r_ld = self._rows(residual, "residual", w, x.dtype)
            if residual.shape != x.shape:
                _fail(f"residual: {tuple(residual.shape)}, expected {tuple(x.shape)}")
            total = x.new_empty(x.shape)
            r_ptr, s_ptr, s_ld = r.data_ptr(), total.data_ptr(), w
        w_type, weight, w_ptr = self._weight(weight, w, kind)
        if q8:
            y, scale = x.new_empty(x.shape, dtype=self._i8), x.new_empty(x.shape[:-1], dtype=self._f32)
            sc_ptr = scale.data_ptr()
        else:
            y, scale, sc_ptr = x.new_empty(x.shape), None, 0
        st = self.lib.asd_add_rmsnorm(self._handle, _pack_norm(n, w, kind, w_type, eps, 0, m.data_ptr(), ld, r_ptr, r_ld, w_ptr, s_ptr, s_ld,
                                                               y.data_ptr(), w, sc_ptr), self._stream(self.device))
        if st != 0:
            self._check(st)
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
        m, n, w, ld = self._rows(s, "s")
        g, _, _, g_ld = self._rows(dy, "dy", w, s.dtype)
        d_ptr = d_ld = 0
        if ds is not None:
            d, _, _, d_ld = self._rows(ds, "ds", w, s.dtype)
            d_ptr = d.data_ptr()
        if dy.shape != s.shape or ds is not None and ds.shape != s.shape:
            _fail(f"dy and ds must have the shape of s, {tuple(s.shape)}")
        w_type, weight, w_ptr = self._weight(weight, w, kind)
        dx = s.new_empty(s.shape)
        dw, dw_ptr = None, 0
        if need_dweight:
            dw = s.new_empty(w, dtype=s.dtype if weight is None else weight.dtype)
            dw_ptr = dw.data_ptr()
        args = (n, w, kind, w_type, eps, 0, g.data_ptr(), g_ld, m.data_ptr(), ld, d_ptr, d_ld, w_ptr, dx.data_ptr(), w, dw_ptr)
        space, at, size = self._space(self.lib.asd_add_rmsnorm_backward_workspace, _pack_norm_backward(*args, 0, 0))
        st = self.lib.asd_add_rmsnorm_backward(self._handle, _pack_norm_backward(*args, at, size), self._stream(self.device))
        if st != 0:
            self._check(st)
        return dx, dw

    # -- 8 bits ----------------------------------------------------------------------------
    def quantize_i8(self, x, act: Optional[str] = None):
        """(q, scale) of the rows of x, or, with act "silu" or "gelu", of h = act(g) * u for rows [g | u]."""
        if act not in ACT:
            _fail(f'act must be None, "silu" or "gelu": {act!r}')
        kind = self._type(x, "x")
        m, n, w, ld = self._rows(x, "x")
        shape = x.shape
        if act is not None:
            if w % 2:
                _fail(f"x: rows [g | u] of an even length, not {w}")
            w //= 2
            shape = shape[:-1] + (w,)
        q, scale = x.new_empty(shape, dtype=self._i8), x.new_empty(shape[:-1], dtype=self._f32)
        st = self.lib.asd_quantize_i8(self._handle, _pack_quantize(n, w, kind, ACT[act], m.data_ptr(), ld, q.data_ptr(), w, scale.data_ptr()),
                                      self._stream(self.device))
        if st != 0:
            self._check(st)
        return q, scale

    def matmul_i8(self, a, a_scale, b, b_scale, bias=None, dtype=None):
        """(a b^T) * a_scale[..., None] * b_scale + bias in `dtype` (bfloat16): a [..., k] and b [out, k] int8, a_scale
        [...] a float32 per row (token), b_scale [out] one per row of b (channel), bias [out] float32 or None."""
        dtype = self._torch.bfloat16 if dtype is None else dtype
        if dtype not in self._types:
            _fail(f"unsupported type {dtype}")
        ma, n, k, ld_a = self._rows(a, "a", None, self._i8)
        mb, out, _, ld_b = self._rows(b, "b", k, self._i8)
        if b.dim() != 2:
            _fail("b must be a matrix [out, k]")
        shape = a.shape[:-1]
        if a_scale.shape != shape:
            _fail(f"a_scale: {tuple(a_scale.shape)}, expected {tuple(shape)}")
        sa = self._vector(a_scale if a_scale.dim() == 1 else a_scale.reshape(-1), "a_scale", n, self._f32)
        sb = self._vector(b_scale, "b_scale", out, self._f32)
        bias_ptr = 0
        if bias is not None:
            bias = self._vector(bias, "bias", out, self._f32)
            bias_ptr = bias.data_ptr()
        y = a.new_empty(shape + (out,), dtype=dtype)
        args = (n, out, k, self._types[dtype], ma.data_ptr(), ld_a, mb.data_ptr(), ld_b, sa.data_ptr(), sb.data_ptr(), bias_ptr,
                y.data_ptr(), out)
        space, at, size = self._space(self.lib.asd_matmul_i8_workspace, _pack_matmul(*args, 0, 0))
        st = self.lib.asd_matmul_i8(self._handle, _pack_matmul(*args, at, size), self._stream(self.device))
        if st != 0:
            self._check(st)
        return y

    # -- gated MLP ---------------------------------------------------------------------------
    def _mlp_weights(self, dtype, w_in, w_out, width):
        """(hidden, the two matrices, and their addresses with row distances)."""
        wi, two, _, ld_i = self._rows(w_in, "w_in", width, dtype)
        if w_in.dim() != 2 or two % 2 or two == 0:
            _fail(f"w_in must be a matrix [2 hidden, width]: {tuple(w_in.shape)}")
        wo, n, _, ld_o = self._rows(w_out, "w_out", two // 2, dtype)
        if w_out.dim() != 2 or n != width:
            _fail(f"w_out must be a matrix [width, hidden]: {tuple(w_out.shape)}")
        return two // 2, (wi, wo), (wi.data_ptr(), ld_i, wo.data_ptr(), ld_o)

    def _saved_bytes(self, n, w, hidden, kind, act):
        need = _i64()
        self._check(self.lib.asd_gated_mlp_saved(self._handle, _pack_mlp(n, w, hidden, kind, act, 0, *([0] * 11)), need))
        return need.value

    def _mlp(self, x, w_in, w_out, act, keep):
        kind, act = self._type(x, "x"), _gate(act)
        m, n, w, ld = self._rows(x, "x")
        hidden, held, weights = self._mlp_weights(x.dtype, w_in, w_out, w)  # `held`: copies live until the call is enqueued
        y = x.new_empty(x.shape)
        saved, saved_ptr = None, 0
        if keep:
            saved = x.new_empty(self._saved_bytes(n, w, hidden, kind, act), dtype=self._u8)
            saved_ptr = saved.data_ptr()
        args = (n, w, hidden, kind, act, 0, m.data_ptr(), ld, *weights, y.data_ptr(), w, saved_ptr)
        space, at, size = self._space(self.lib.asd_gated_mlp_forward_workspace, _pack_mlp(*args, 0, 0))
        st = self.lib.asd_gated_mlp_forward(self._handle, _pack_mlp(*args, at, size), self._stream(self.device))
        if st != 0:
            self._check(st)
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
        kind, act = self._type(x, "x"), _gate(act)
        m, n, w, ld = self._rows(x, "x")
        g, _, _, g_ld = self._rows(dy, "dy", w, x.dtype)
        if dy.shape != x.shape:
            _fail(f"dy: {tuple(dy.shape)}, expected {tuple(x.shape)}")
        hidden, held, weights = self._mlp_weights(x.dtype, w_in, w_out, w)
        size = self._saved_bytes(n, w, hidden, kind, act)
        if saved.dtype is not self._u8 or saved.numel() != size or saved.get_device() != self.device or not saved.is_contiguous():
            _fail(f"saved must be what gated_mlp_forward returned: {size} bytes for these sizes")
        dx = x.new_empty(x.shape) if need[0] else None
        dw_in = x.new_empty(w_in.shape) if need[1] else None
        dw_out = x.new_empty(w_out.shape) if need[2] else None
        out = [0 if t is None else t.data_ptr() for t in (dx, dw_in, dw_out)]
        args = (n, w, hidden, kind, act, 0, g.data_ptr(), g_ld, m.data_ptr(), ld, *weights, saved.data_ptr(), out[0], w, out[1], w, out[2], hidden)
        space, at, size = self._space(self.lib.asd_gated_mlp_backward_workspace, _pack_mlp_backward(*args, 0, 0))
        st = self.lib.asd_gated_mlp_backward(self._handle, _pack_mlp_backward(*args, at, size), self._stream(self.device))
        if st != 0:
            self._check(st)
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
