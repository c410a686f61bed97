"""The operators of a gated residual block (include/asd_ops.h) for torch tensors.  Argument marshalling only, done by a small
native module (csrc/asd_torch.cpp); the structures and prototypes of the C entry points are declared here for ctypes.

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
_EXT = None


def _library():
    """The shared library with the operators' prototypes declared, for callers of the C entry points."""
    global _LIB
    if _LIB is None:
        lib = load_library()
        lib.asd_ops_last_error.restype, lib.asd_ops_last_error.argtypes = C.c_char_p, []
        lib.asd_ops_destroy.restype, lib.asd_ops_destroy.argtypes = None, [_vp]
        lib.asd_ops_create.argtypes = [C.POINTER(_vp)]
        lib.asd_ops_check.argtypes = [_vp, _vp]
        for name, args in (("add_rmsnorm", _Norm), ("add_rmsnorm_backward", _NormBackward), ("quantize_i8", _Quantize),
                           ("matmul_i8", _MatmulI8), ("gated_mlp_forward", _GatedMlp), ("gated_mlp_backward", _GatedMlpBackward)):
            getattr(lib, "asd_" + name).argtypes = [_vp, C.POINTER(args), _vp]
            if "asd_" + name + "_workspace" in OPS_SYMBOLS:
                getattr(lib, "asd_" + name + "_workspace").argtypes = [_vp, C.POINTER(args), C.POINTER(_i64)]
        lib.asd_gated_mlp_saved.argtypes = [_vp, C.POINTER(_GatedMlp), C.POINTER(_i64)]
        for name in OPS_SYMBOLS:
            if name not in ("asd_ops_last_error", "asd_ops_destroy"):
                getattr(lib, name).restype = C.c_int
        _LIB = lib
    return _LIB


def _extension():
    """The binding for torch tensors (csrc/asd_torch.cpp).  Raises if it has not been built."""
    global _EXT
    if _EXT is None:
        load_library()  # says how to build what is missing
        import torch  # noqa: F401  (its libraries, before those that need them)
        try:
            from . import _asd_torch
        except ImportError as e:
            raise ImportError(f"the operators' torch binding does not load ({e}): run `python -m paper_2505_03983_b200.build "
                              "--force` (or __graft_entry__.build()); there is no fallback path") from e
        _EXT = _asd_torch
    return _EXT


def _gate(act):
    if act != "silu" and act != "gelu":
        raise AsdError(1, f'act must be "silu" or "gelu": {act!r}')
    return ACT[act]


class AsdOps:
    """A handle of the operators on one device (the current one): asd_ops_create on construction, asd_ops_destroy on
    close().  It keeps nothing of its inputs; calls may come from several streams.

    Tensors are CUDA tensors of two or more dimensions, whose last one is the row; leading dimensions are rows.  Rows may
    be strided; a tensor whose last dimension is not contiguous is copied first.  Results are new tensors.  The work is
    enqueued on the current stream."""

    def __init__(self):
        import torch
        if not torch.cuda.is_available():
            raise AsdError(4, "no CUDA device: the ASD library has no CPU path")
        self.lib = _library()
        self._ext = _extension()
        self._types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # asd_type
        self._bf16 = torch.bfloat16
        self.device = torch.cuda.current_device()
        torch.cuda.current_stream().synchronize()  # the device's context exists before the library asks for it
        self._handle = self._ext.create()

    def close(self):
        if getattr(self, "_handle", None):
            self._ext.destroy(self._handle)
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

    def check(self):
        """Synchronises the current stream; raises ASD_ERR_TIMEOUT if a kernel of this handle gave up a wait."""
        self._ext.check(self._handle, self.device)

    # -- norm ------------------------------------------------------------------------------
    def add_rmsnorm(self, x, weight, residual=None, eps=1e-6):
        """(y, s): s = x + residual in the type of x (x itself without a residual), y its root-mean-square norm times
        weight ([width], of x's type or float32; None: 1)."""
        y, _, s = self._ext.add_rmsnorm(self._handle, self.device, x, weight, residual, eps, False)
        return y, s

    def add_rmsnorm_i8(self, x, weight, residual=None, eps=1e-6):
        """(q, scale, s): as add_rmsnorm, with y ~ q * scale[..., None] in int8 and a float32 scale per row."""
        return self._ext.add_rmsnorm(self._handle, self.device, x, weight, residual, eps, True)

    def add_rmsnorm_backward(self, dy, s, weight, ds=None, eps=1e-6, need_dweight=True, need_dx=True):
        """(dx, dweight) of add_rmsnorm from the gradients dy of y and ds of s (None: 0); dx is the gradient of x and of
        the residual alike, dweight has weight's type (s's without a weight); one that is not needed is None."""
        return self._ext.add_rmsnorm_backward(self._handle, self.device, dy, s, weight, ds, eps, need_dweight, need_dx)

    # -- 8 bits ----------------------------------------------------------------------------
    def quantize_i8(self, x, act: Optional[str] = None):
        """(q, scale) of the rows of x, or, with act "silu" or "gelu", of h = act(g) * u for rows [g | u]."""
        if act not in ACT:
            raise AsdError(1, f'act must be None, "silu" or "gelu": {act!r}')
        return self._ext.quantize_i8(self._handle, self.device, x, ACT[act])

    def matmul_i8(self, a, a_scale, b, b_scale, bias=None, dtype=None):
        """(a b^T) * a_scale[..., None] * b_scale + bias in `dtype` (bfloat16): a [..., k] and b [out, k] int8, a_scale
        [...] a float32 per row (token), b_scale [out] one per row of b (channel), bias [out] float32 or None."""
        kind = self._types.get(self._bf16 if dtype is None else dtype)
        if kind is None:
            raise AsdError(1, f"unsupported type {dtype}")
        return self._ext.matmul_i8(self._handle, self.device, a, a_scale, b, b_scale, bias, kind)

    # -- gated MLP ---------------------------------------------------------------------------
    def gated_mlp(self, x, w_in, w_out, act="silu"):
        """(act(x Wg^T) * (x Wu^T)) w_out^T with w_in = [Wg; Wu] [2 hidden, width], w_out [width, hidden]; float16 or
        bfloat16, act "silu" or "gelu"."""
        return self._ext.gated_mlp(self._handle, self.device, x, w_in, w_out, _gate(act), False)[0]

    def gated_mlp_forward(self, x, w_in, w_out, act="silu"):
        """(y, saved): gated_mlp, and what gated_mlp_backward needs (opaque bytes)."""
        return self._ext.gated_mlp(self._handle, self.device, x, w_in, w_out, _gate(act), True)

    def gated_mlp_backward(self, dy, x, w_in, w_out, saved, act="silu", need=(True, True, True)):
        """(dx, dw_in, dw_out); an entry of `need` that is false leaves out that gradient (None)."""
        return self._ext.gated_mlp_backward(self._handle, self.device, dy, x, w_in, w_out, saved, _gate(act), *need)


_DEFAULT = {}
_current_device = None


def default_ops() -> AsdOps:
    """The process's handle of the current device, made at its first use."""
    global _current_device
    if _current_device is None:
        import torch
        if not torch.cuda.is_available():
            raise AsdError(4, "no CUDA device: the ASD library has no CPU path")
        _current_device = torch.cuda.current_device
    device = _current_device()
    ops = _DEFAULT.get(device)
    if ops is None:
        ops = _DEFAULT[device] = AsdOps()
    return ops
