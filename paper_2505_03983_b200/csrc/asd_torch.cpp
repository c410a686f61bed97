// The operators of include/asd_ops.h for torch tensors: checks of shapes, types and devices, outputs and workspaces from
// torch's allocator on the current stream, and the C entry points.  A call with few rows is over on the GPU in a few
// microseconds; marshalled in Python, its arguments alone took longer (10 to 35 us).
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/utils/pybind.h>
#include <torch/extension.h>

#include <string>

#include "asd_ops.h"

namespace {

using at::Tensor;
using OptTensor = std::optional<Tensor>;

PyObject* g_error = nullptr;  // binding.AsdError

[[noreturn]] void fail(int status, const std::string& message) {
  PyObject* e = PyObject_CallFunction(g_error, "is", status, message.c_str());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw py::error_already_set();
}
void require(bool ok, const std::string& message) {
  if (!ok) fail(ASD_ERR_INVALID_ARG, message);
}
void check(asd_status st) {
  if (st != ASD_OK) fail(st, asd_ops_last_error());
}

std::string shape_text(at::IntArrayRef s) {
  std::string t = "(";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + ")";
}
int type_of(const Tensor& t, const char* name) {
  switch (t.scalar_type()) {
    case at::kFloat: return ASD_TYPE_F32;
    case at::kHalf: return ASD_TYPE_F16;
    case at::kBFloat16: return ASD_TYPE_BF16;
    default: fail(ASD_ERR_INVALID_ARG, std::string(name) + " must be a tensor of float32, float16 or bfloat16");
  }
}
at::ScalarType scalar_of(int type) { return type == ASD_TYPE_F32 ? at::kFloat : type == ASD_TYPE_F16 ? at::kHalf : at::kBFloat16; }

struct Call {
  asd_ops* ops;
  int device;
  void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
  Tensor empty(at::IntArrayRef shape, at::ScalarType type) const {
    return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (c10::DeviceIndex)device), std::nullopt);
  }
  void on_device(const Tensor& t, const char* name) const {
    if (!t.is_cuda() || t.get_device() != device)
      fail(ASD_ERR_INVALID_ARG, std::string(name) + " must be a tensor on cuda:" + std::to_string(device));
  }
};

// A tensor as rows of its last dimension.
struct Rows {
  Tensor t;  // keeps a copy alive until the call is enqueued
  int64_t n, w, ld;
  void* p() const { return t.data_ptr(); }
};
Rows rows_of(const Call& c, const Tensor& t, const char* name, int64_t width = -1, std::optional<at::ScalarType> type = std::nullopt) {
  c.on_device(t, name);
  if (type && t.scalar_type() != *type)
    fail(ASD_ERR_INVALID_ARG, std::string(name) + ": " + c10::toString(t.scalar_type()) + ", expected " + c10::toString(*type));
  const int64_t dims = t.dim();
  if (dims < 2) fail(ASD_ERR_INVALID_ARG, std::string(name) + " must have two or more dimensions: it has " + std::to_string(dims));
  const int64_t w = t.size(-1);
  if (w == 0) fail(ASD_ERR_INVALID_ARG, std::string(name) + ": rows without elements");
  if (width >= 0 && w != width)
    fail(ASD_ERR_INVALID_ARG, std::string(name) + ": rows of " + std::to_string(w) + ", expected " + std::to_string(width));
  Rows r{t, t.numel() / w, w, w};
  if (!t.is_contiguous()) {
    if (dims != 2) r.t = t.reshape({-1, w});
    const int64_t step = r.t.stride(0), one = r.t.stride(1);
    if ((w > 1 && one != 1) || (r.n > 1 && step < w))
      r.t = r.t.contiguous();
    else if (r.n > 1)
      r.ld = step;
  }
  if (r.n > INT32_MAX) fail(ASD_ERR_UNSUPPORTED, std::string(name) + ": more than 2^31 - 1 rows");
  return r;
}
Tensor vector_of(const Call& c, const Tensor& t, const char* name, int64_t n, std::optional<at::ScalarType> type) {
  c.on_device(t, name);
  if (t.dim() != 1 || t.size(0) != n)
    fail(ASD_ERR_INVALID_ARG, std::string(name) + " must have the shape (" + std::to_string(n) + ",): " + shape_text(t.sizes()));
  if (type && t.scalar_type() != *type)
    fail(ASD_ERR_INVALID_ARG, std::string(name) + ": " + c10::toString(t.scalar_type()) + ", expected " + c10::toString(*type));
  return t.is_contiguous() ? t : t.contiguous();
}
void same_shape(const Tensor& t, const char* name, const Tensor& as) {
  if (t.sizes() != as.sizes())
    fail(ASD_ERR_INVALID_ARG, std::string(name) + ": " + shape_text(t.sizes()) + ", expected " + shape_text(as.sizes()));
}
// The shape of t with another last dimension, or (last < 0) without it.
c10::SmallVector<int64_t, 6> shape_with(const Tensor& t, int64_t last) {
  c10::SmallVector<int64_t, 6> s(t.sizes().begin(), t.sizes().end() - 1);
  if (last >= 0) s.push_back(last);
  return s;
}
// The workspace of a call: asked for, allocated, entered in its arguments.
template <typename A>
Tensor workspace(const Call& c, A* a, asd_status (*query)(asd_ops*, const A*, int64_t*)) {
  int64_t bytes = 0;
  check(query(c.ops, a, &bytes));
  if (!bytes) return Tensor();
  Tensor t = c.empty({bytes}, at::kByte);
  a->workspace = t.data_ptr();
  a->workspace_bytes = bytes;
  return t;
}

// (y, scale or None, s)
py::tuple add_rmsnorm(int64_t ops, int device, const Tensor& x, const OptTensor& weight, const OptTensor& residual, double eps, bool q8) {
  const Call c{(asd_ops*)ops, device};
  asd_rmsnorm_args a{};
  a.type = a.w_type = type_of(x, "x");
  const Rows m = rows_of(c, x, "x");
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX), a.eps = (float)eps;
  a.x = m.p(), a.ld_x = m.ld;
  Rows r;
  Tensor total = x, w;
  if (residual) {
    r = rows_of(c, *residual, "residual", m.w, x.scalar_type());
    same_shape(*residual, "residual", x);
    total = c.empty(x.sizes(), x.scalar_type());
    a.residual = r.p(), a.ld_residual = r.ld, a.sum = total.data_ptr(), a.ld_sum = m.w;
  }
  if (weight) {
    w = vector_of(c, *weight, "weight", m.w, std::nullopt);
    a.w_type = type_of(w, "weight");
    a.weight = w.data_ptr();
  }
  Tensor y = c.empty(x.sizes(), q8 ? at::kChar : x.scalar_type()), scale;
  a.y = y.data_ptr(), a.ld_y = m.w;
  if (q8) {
    scale = c.empty(shape_with(x, -1), at::kFloat);
    a.scale = scale.data_ptr<float>();
  }
  check(asd_add_rmsnorm(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(y), q8 ? py::cast(std::move(scale)) : py::none(), std::move(total));
}

py::tuple add_rmsnorm_backward(int64_t ops, int device, const Tensor& dy, const Tensor& s, const OptTensor& weight, const OptTensor& ds, double eps,
                               bool need_dw, bool need_dx) {
  const Call c{(asd_ops*)ops, device};
  asd_rmsnorm_backward_args a{};
  a.type = a.w_type = type_of(s, "s");
  const Rows m = rows_of(c, s, "s"), g = rows_of(c, dy, "dy", m.w, s.scalar_type());
  same_shape(dy, "dy", s);
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX), a.eps = (float)eps;
  a.s = m.p(), a.ld_s = m.ld, a.dy = g.p(), a.ld_dy = g.ld;
  Rows d;
  if (ds) {
    d = rows_of(c, *ds, "ds", m.w, s.scalar_type());
    same_shape(*ds, "ds", s);
    a.ds = d.p(), a.ld_ds = d.ld;
  }
  Tensor w, dw, dx;
  if (weight) {
    w = vector_of(c, *weight, "weight", m.w, std::nullopt);
    a.w_type = type_of(w, "weight");
    a.weight = w.data_ptr();
  }
  if (need_dx) {
    dx = c.empty(s.sizes(), s.scalar_type());
    a.dx = dx.data_ptr(), a.ld_dx = m.w;
  }
  if (need_dw) {
    dw = c.empty({m.w}, scalar_of(a.w_type));
    a.dw = dw.data_ptr();
  }
  const Tensor space = workspace(c, &a, asd_add_rmsnorm_backward_workspace);
  check(asd_add_rmsnorm_backward(c.ops, &a, c.stream()));
  return py::make_tuple(need_dx ? py::cast(std::move(dx)) : py::none(), need_dw ? py::cast(std::move(dw)) : py::none());
}

py::tuple quantize_i8(int64_t ops, int device, const Tensor& x, int act) {
  const Call c{(asd_ops*)ops, device};
  asd_quantize_args a{};
  a.type = type_of(x, "x"), a.act = act;
  const Rows m = rows_of(c, x, "x");
  int64_t w = m.w;
  if (act != ASD_ACT_NONE) {
    if (w % 2) fail(ASD_ERR_INVALID_ARG, "x: rows [g | u] of an even length, not " + std::to_string(w));
    w /= 2;
  }
  Tensor q = c.empty(shape_with(x, w), at::kChar), scale = c.empty(shape_with(x, -1), at::kFloat);
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(w, INT32_MAX);
  a.x = m.p(), a.ld_x = m.ld, a.q = (int8_t*)q.data_ptr(), a.ld_q = w, a.scale = scale.data_ptr<float>();
  check(asd_quantize_i8(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(q), std::move(scale));
}

Tensor matmul_i8(int64_t ops, int device, const Tensor& x, const Tensor& a_scale, const Tensor& b, const Tensor& b_scale, const OptTensor& bias,
                 int out_type) {
  const Call c{(asd_ops*)ops, device};
  asd_matmul_i8_args a{};
  const Rows ma = rows_of(c, x, "a", -1, at::kChar), mb = rows_of(c, b, "b", ma.w, at::kChar);
  require(b.dim() == 2, "b must be a matrix [out, k]");
  const auto lead = shape_with(x, -1);
  if (a_scale.sizes() != at::IntArrayRef(lead))
    fail(ASD_ERR_INVALID_ARG, "a_scale: " + shape_text(a_scale.sizes()) + ", expected " + shape_text(lead));
  const Tensor sa = vector_of(c, a_scale.dim() == 1 ? a_scale : a_scale.reshape({-1}), "a_scale", ma.n, at::kFloat);
  const Tensor sb = vector_of(c, b_scale, "b_scale", mb.n, at::kFloat);
  a.rows = (int32_t)ma.n, a.out = (int32_t)mb.n, a.k = (int32_t)std::min<int64_t>(ma.w, INT32_MAX), a.out_type = out_type;
  a.a = (const int8_t*)ma.p(), a.ld_a = ma.ld, a.b = (const int8_t*)mb.p(), a.ld_b = mb.ld;
  a.a_scale = sa.data_ptr<float>(), a.b_scale = sb.data_ptr<float>();
  Tensor bb;
  if (bias) {
    bb = vector_of(c, *bias, "bias", mb.n, at::kFloat);
    a.bias = bb.data_ptr<float>();
  }
  Tensor y = c.empty(shape_with(x, mb.n), scalar_of(out_type));
  a.y = y.data_ptr(), a.ld_y = mb.n;
  const Tensor space = workspace(c, &a, asd_matmul_i8_workspace);
  check(asd_matmul_i8(c.ops, &a, c.stream()));
  return y;
}

// Both matrices of the gated MLP, entered in the arguments.
struct Weights {
  Rows in, out;
};
template <typename A>
Weights mlp_weights(const Call& c, A* a, const Tensor& w_in, const Tensor& w_out, int64_t width, at::ScalarType type) {
  if (w_in.dim() != 2 || w_in.size(0) % 2 || w_in.size(0) == 0)
    fail(ASD_ERR_INVALID_ARG, "w_in must be a matrix [2 hidden, width]: " + shape_text(w_in.sizes()));
  if (w_out.dim() != 2 || w_out.size(0) != width)
    fail(ASD_ERR_INVALID_ARG, "w_out must be a matrix [width, hidden]: " + shape_text(w_out.sizes()));
  Weights w{rows_of(c, w_in, "w_in", width, type), rows_of(c, w_out, "w_out", w_in.size(0) / 2, type)};
  a->hidden = (int32_t)(w_in.size(0) / 2);
  a->w_in = w.in.p(), a->ld_w_in = w.in.ld, a->w_out = w.out.p(), a->ld_w_out = w.out.ld;
  return w;
}

// (y, saved or None)
py::tuple gated_mlp(int64_t ops, int device, const Tensor& x, const Tensor& w_in, const Tensor& w_out, int act, bool keep) {
  const Call c{(asd_ops*)ops, device};
  asd_gated_mlp_args a{};
  a.type = type_of(x, "x"), a.act = act;
  const Rows m = rows_of(c, x, "x");
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX), a.x = m.p(), a.ld_x = m.ld;
  const Weights w = mlp_weights(c, &a, w_in, w_out, m.w, x.scalar_type());
  Tensor y = c.empty(x.sizes(), x.scalar_type()), saved;
  a.y = y.data_ptr(), a.ld_y = m.w;
  if (keep) {
    int64_t bytes = 0;
    check(asd_gated_mlp_saved(c.ops, &a, &bytes));
    saved = c.empty({bytes}, at::kByte);
    a.saved = saved.data_ptr();
  }
  const Tensor space = workspace(c, &a, asd_gated_mlp_forward_workspace);
  check(asd_gated_mlp_forward(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(y), keep ? py::cast(std::move(saved)) : py::none());
}

py::tuple gated_mlp_backward(int64_t ops, int device, const Tensor& dy, const Tensor& x, const Tensor& w_in, const Tensor& w_out, const Tensor& saved,
                             int act, bool need_dx, bool need_dw_in, bool need_dw_out) {
  const Call c{(asd_ops*)ops, device};
  asd_gated_mlp_backward_args a{};
  a.type = type_of(x, "x"), a.act = act;
  const Rows m = rows_of(c, x, "x"), g = rows_of(c, dy, "dy", m.w, x.scalar_type());
  same_shape(dy, "dy", x);
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX);
  a.x = m.p(), a.ld_x = m.ld, a.dy = g.p(), a.ld_dy = g.ld;
  const Weights w = mlp_weights(c, &a, w_in, w_out, m.w, x.scalar_type());
  asd_gated_mlp_args f{};
  f.rows = a.rows, f.width = a.width, f.hidden = a.hidden, f.type = a.type, f.act = a.act;
  int64_t bytes = 0;
  check(asd_gated_mlp_saved(c.ops, &f, &bytes));
  c.on_device(saved, "saved");
  require(saved.scalar_type() == at::kByte && saved.numel() == bytes && saved.is_contiguous(),
          "saved must be what gated_mlp_forward returned: " + std::to_string(bytes) + " bytes for these sizes");
  a.saved = saved.data_ptr();
  Tensor dx, dw_in, dw_out;
  if (need_dx) {
    dx = c.empty(x.sizes(), x.scalar_type());
    a.dx = dx.data_ptr(), a.ld_dx = m.w;
  }
  if (need_dw_in) {
    dw_in = c.empty(w_in.sizes(), x.scalar_type());
    a.dw_in = dw_in.data_ptr(), a.ld_dw_in = m.w;
  }
  if (need_dw_out) {
    dw_out = c.empty(w_out.sizes(), x.scalar_type());
    a.dw_out = dw_out.data_ptr(), a.ld_dw_out = a.hidden;
  }
  const Tensor space = workspace(c, &a, asd_gated_mlp_backward_workspace);
  check(asd_gated_mlp_backward(c.ops, &a, c.stream()));
  auto out = [](bool need, Tensor& t) -> py::object { return need ? py::cast(std::move(t)) : py::none(); };
  return py::make_tuple(out(need_dx, dx), out(need_dw_in, dw_in), out(need_dw_out, dw_out));
}

// w [out, width] of a linear layer, entered in the arguments.
template <typename A>
Rows layer_weight(const Call& c, A* a, const Tensor& w, int64_t width, at::ScalarType type) {
  if (w.dim() != 2) fail(ASD_ERR_INVALID_ARG, "w must be a matrix [out, width]: " + shape_text(w.sizes()));
  if (w.size(0) == 0) fail(ASD_ERR_INVALID_ARG, "w: no rows");
  const Rows r = rows_of(c, w, "w", width, type);
  a->out = (int32_t)r.n, a->w = r.p(), a->ld_w = r.ld;
  return r;
}

// (y, saved or None)
py::tuple linear(int64_t ops, int device, const Tensor& x, const Tensor& w, const OptTensor& bias, const OptTensor& residual, int act, int out_type,
                 bool keep) {
  const Call c{(asd_ops*)ops, device};
  asd_linear_args a{};
  a.type = type_of(x, "x"), a.act = act;
  a.out_type = out_type < 0 ? a.type : out_type, a.bias_type = ASD_TYPE_F32;
  const Rows m = rows_of(c, x, "x");
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX), a.x = m.p(), a.ld_x = m.ld;
  const Rows mw = layer_weight(c, &a, w, m.w, x.scalar_type());
  Tensor b, saved;
  if (bias) {
    b = vector_of(c, *bias, "bias", mw.n, std::nullopt);
    a.bias_type = type_of(b, "bias");
    a.bias = b.data_ptr();
  }
  Tensor y = c.empty(shape_with(x, mw.n), scalar_of(a.out_type));
  a.y = y.data_ptr(), a.ld_y = mw.n;
  Rows r;
  if (residual) {
    r = rows_of(c, *residual, "residual", mw.n, scalar_of(a.out_type));
    same_shape(*residual, "residual", y);
    a.residual = r.p(), a.ld_residual = r.ld;
  }
  if (keep && act != ASD_ACT_NONE) {
    int64_t bytes = 0;
    check(asd_linear_saved(c.ops, &a, &bytes));
    saved = c.empty({bytes}, at::kByte);
    a.saved = saved.data_ptr();
  }
  const Tensor space = workspace(c, &a, asd_linear_forward_workspace);
  check(asd_linear_forward(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(y), saved.defined() ? py::cast(std::move(saved)) : py::none());
}

py::tuple linear_backward(int64_t ops, int device, const Tensor& dy, const Tensor& x, const Tensor& w, const OptTensor& saved, const OptTensor& bias,
                          int act, bool need_dx, bool need_dw, bool need_db) {
  const Call c{(asd_ops*)ops, device};
  asd_linear_backward_args a{};
  a.type = type_of(x, "x"), a.act = act, a.bias_type = ASD_TYPE_F32;
  a.dy_type = type_of(dy, "dy");
  const Rows m = rows_of(c, x, "x");
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX), a.x = m.p(), a.ld_x = m.ld;
  const Rows mw = layer_weight(c, &a, w, m.w, x.scalar_type()), g = rows_of(c, dy, "dy", mw.n);
  const auto shape = shape_with(x, mw.n);
  if (dy.sizes() != at::IntArrayRef(shape)) fail(ASD_ERR_INVALID_ARG, "dy: " + shape_text(dy.sizes()) + ", expected " + shape_text(shape));
  a.dy = g.p(), a.ld_dy = g.ld;
  Tensor b, dx, dw, db;
  if (bias) {
    b = vector_of(c, *bias, "bias", mw.n, std::nullopt);
    a.bias_type = type_of(b, "bias");
  }
  if (act != ASD_ACT_NONE) {
    asd_linear_args f{};
    f.rows = a.rows, f.width = a.width, f.out = a.out, f.type = f.out_type = f.bias_type = a.type, f.act = act;
    int64_t bytes = 0;
    check(asd_linear_saved(c.ops, &f, &bytes));
    require(saved.has_value(), "saved must be what linear_forward returned, not None");
    c.on_device(*saved, "saved");
    require(saved->scalar_type() == at::kByte && saved->numel() == bytes && saved->is_contiguous(),
            "saved must be what linear_forward returned: " + std::to_string(bytes) + " bytes for these sizes");
    a.saved = saved->data_ptr();
  }
  if (need_dx) {
    dx = c.empty(x.sizes(), x.scalar_type());
    a.dx = dx.data_ptr(), a.ld_dx = m.w;
  }
  if (need_dw) {
    dw = c.empty(w.sizes(), x.scalar_type());
    a.dw = dw.data_ptr(), a.ld_dw = m.w;
  }
  if (need_db && bias) {
    db = c.empty({mw.n}, scalar_of(a.bias_type));
    a.dbias = db.data_ptr();
  }
  const Tensor space = workspace(c, &a, asd_linear_backward_workspace);
  check(asd_linear_backward(c.ops, &a, c.stream()));
  auto out = [](Tensor& t) -> py::object { return t.defined() ? py::cast(std::move(t)) : py::none(); };
  return py::make_tuple(out(dx), out(dw), out(db));
}

// The gate of block_rmsnorm, entered in the arguments with the weights: a row for each run of x's rows.
struct BlockWeights {
  Tensor w, post;
  Rows gate;
};
template <typename A>
BlockWeights block_weights(const Call& c, A* a, const Tensor& x, int64_t rows, int64_t width, const OptTensor& weight, const OptTensor& post,
                           const OptTensor& gate, double alpha, double eps, bool post_norm) {
  BlockWeights b;
  a->w_type = a->post_type = a->gate_type = a->type, a->group = 1;
  a->alpha = (float)alpha, a->eps = (float)eps, a->post_norm = post_norm;
  if (weight) {
    b.w = vector_of(c, *weight, "weight", width, std::nullopt);
    a->w_type = type_of(b.w, "weight"), a->weight = b.w.data_ptr();
  }
  if (post) {
    b.post = vector_of(c, *post, "post_weight", width, std::nullopt);
    a->post_type = type_of(b.post, "post_weight"), a->post_weight = b.post.data_ptr();
  }
  if (gate) {
    const Tensor& t = *gate;
    bool fits = t.dim() == 1 || t.dim() == x.dim();
    if (fits && t.dim() > 1) {
      int64_t i = 0;
      while (i < t.dim() - 1 && t.size(i) == x.size(i)) ++i;
      while (i < t.dim() - 1 && t.size(i) == 1) ++i;
      fits = i == t.dim() - 1;
    }
    if (!fits)
      fail(ASD_ERR_INVALID_ARG, "gate: " + shape_text(t.sizes()) + ", expected (width,), or the leading dimensions of x " + shape_text(x.sizes()) +
                                    " up to some point and 1 from there on");
    b.gate = rows_of(c, t.dim() == 1 ? t.unsqueeze(0) : t, "gate", width);
    a->gate_type = type_of(t, "gate"), a->gate = b.gate.p(), a->ld_gate = b.gate.ld;
    a->group = (int32_t)(b.gate.n ? std::max<int64_t>(1, rows / b.gate.n) : 1);
  }
  return b;
}

// (y, scale or None, s)
py::tuple block_rmsnorm(int64_t ops, int device, const Tensor& x, const Tensor& residual, const OptTensor& weight, const OptTensor& post,
                        const OptTensor& gate, double alpha, double eps, bool post_norm, bool q8) {
  const Call c{(asd_ops*)ops, device};
  asd_block_rmsnorm_args a{};
  a.type = type_of(x, "x");
  const Rows m = rows_of(c, x, "x"), r = rows_of(c, residual, "residual", m.w, x.scalar_type());
  same_shape(residual, "residual", x);
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX);
  a.x = m.p(), a.ld_x = m.ld, a.residual = r.p(), a.ld_residual = r.ld;
  const BlockWeights b = block_weights(c, &a, x, m.n, m.w, weight, post, gate, alpha, eps, post_norm);
  Tensor s = c.empty(x.sizes(), x.scalar_type()), y = c.empty(x.sizes(), q8 ? at::kChar : x.scalar_type()), scale;
  a.s = s.data_ptr(), a.ld_s = m.w, a.y = y.data_ptr(), a.ld_y = m.w;
  if (q8) {
    scale = c.empty(shape_with(x, -1), at::kFloat);
    a.scale = scale.data_ptr<float>();
  }
  check(asd_block_rmsnorm(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(y), q8 ? py::cast(std::move(scale)) : py::none(), std::move(s));
}

py::tuple block_rmsnorm_backward(int64_t ops, int device, const Tensor& dy, const Tensor& x, const Tensor& s, const OptTensor& weight,
                                 const OptTensor& post, const OptTensor& gate, const OptTensor& ds, double alpha, double eps, bool post_norm,
                                 bool need_dx, bool need_dr, bool need_dw, bool need_dp, bool need_dg) {
  const Call c{(asd_ops*)ops, device};
  asd_block_rmsnorm_backward_args a{};
  a.type = type_of(x, "x");
  const Rows m = rows_of(c, x, "x"), ms = rows_of(c, s, "s", m.w, x.scalar_type()), g = rows_of(c, dy, "dy", m.w, x.scalar_type());
  same_shape(s, "s", x);
  same_shape(dy, "dy", x);
  a.rows = (int32_t)m.n, a.width = (int32_t)std::min<int64_t>(m.w, INT32_MAX);
  a.x = m.p(), a.ld_x = m.ld, a.s = ms.p(), a.ld_s = ms.ld, a.dy = g.p(), a.ld_dy = g.ld;
  Rows d;
  if (ds) {
    d = rows_of(c, *ds, "ds", m.w, x.scalar_type());
    same_shape(*ds, "ds", x);
    a.ds = d.p(), a.ld_ds = d.ld;
  }
  const BlockWeights b = block_weights(c, &a, x, m.n, m.w, weight, post, gate, alpha, eps, post_norm);
  Tensor dx, dr, dw, dp, dg;
  if (need_dx) {
    dx = c.empty(x.sizes(), x.scalar_type());
    a.dx = dx.data_ptr(), a.ld_dx = m.w;
  }
  if (need_dr) {
    dr = c.empty(x.sizes(), x.scalar_type());
    a.dresidual = dr.data_ptr(), a.ld_dresidual = m.w;
  }
  if (need_dw && weight) {
    dw = c.empty({m.w}, scalar_of(a.w_type));
    a.dweight = dw.data_ptr();
  }
  if (need_dp && post) {
    dp = c.empty({m.w}, scalar_of(a.post_type));
    a.dpost_weight = dp.data_ptr();
  }
  if (need_dg && gate) {
    // without rows nothing is summed up
    dg = m.n ? c.empty(gate->sizes(), scalar_of(a.gate_type)) : at::zeros(gate->sizes(), gate->options());
    a.dgate = dg.data_ptr(), a.ld_dgate = m.w;
  }
  const Tensor space = workspace(c, &a, asd_block_rmsnorm_backward_workspace);
  check(asd_block_rmsnorm_backward(c.ops, &a, c.stream()));
  auto out = [](Tensor& t) -> py::object { return t.defined() ? py::cast(std::move(t)) : py::none(); };
  return py::make_tuple(out(dx), out(dr), out(dw), out(dp), out(dg));
}

// A dense tensor of n elements in its own order, entered as an address.
void* dense(const Call& c, const Tensor& t, const char* name, int64_t n, std::optional<at::ScalarType> type) {
  c.on_device(t, name);
  if (type && t.scalar_type() != *type)
    fail(ASD_ERR_INVALID_ARG, std::string(name) + ": " + c10::toString(t.scalar_type()) + ", expected " + c10::toString(*type));
  if (t.numel() != n) fail(ASD_ERR_INVALID_ARG, std::string(name) + ": " + std::to_string(t.numel()) + " elements, expected " + std::to_string(n));
  if (!t.is_contiguous()) fail(ASD_ERR_INVALID_ARG, std::string(name) + " must be contiguous");
  return t.data_ptr();
}
// A float32 tensor of one element on the device, or NULL.
const float* device_scalar(const Call& c, const OptTensor& t, const char* name) {
  return t ? (const float*)dense(c, *t, name, 1, at::kFloat) : nullptr;
}
// A list of tensors, as Python has it: no tensor is copied to look at it.
struct TensorList {
  py::object held;
  PyObject** items = nullptr;
  size_t n = 0;
  TensorList(const py::object& list, const char* name) {
    if (list.is_none()) return;
    held = py::reinterpret_steal<py::object>(PySequence_Fast(list.ptr(), "a list of tensors is expected"));
    if (!held) throw py::error_already_set();
    items = PySequence_Fast_ITEMS(held.ptr());
    n = (size_t)PySequence_Fast_GET_SIZE(held.ptr());
    for (size_t i = 0; i < n; ++i)
      if (items[i] != Py_None && !THPVariable_Check(items[i])) fail(ASD_ERR_INVALID_ARG, std::string(name) + ": not a tensor");
  }
  bool given() const { return (bool)held; }
  bool has(size_t i) const { return held && items[i] != Py_None; }
  const Tensor& at(size_t i, const char* name) const {
    if (items[i] == Py_None) fail(ASD_ERR_INVALID_ARG, std::string(name) + ": not a tensor");
    return THPVariable_Unpack(items[i]);
  }
};

void adamw(int64_t ops, int device, const py::object& params_, const py::object& grads_, const py::object& m_, const py::object& v_, const Tensor& step, py::object lr,
           double beta1, double beta2, double eps, double weight_decay, const py::object& masters_, const py::object& scales_,
           const OptTensor& grad_scale, const OptTensor& skip, bool unbiased) {
  const Call c{(asd_ops*)ops, device};
  const TensorList params(params_, "params"), grads(grads_, "grads"), m(m_, "exp_avgs"), v(v_, "exp_avg_sqs"), masters(masters_, "masters"),
      scales(scales_, "scales");
  const size_t n = params.n;
  require(grads.n == n && m.n == n && v.n == n && (!masters.given() || masters.n == n) && (!scales.given() || scales.n == n),
          "adamw: lists of different lengths");
  require(n <= (size_t)INT32_MAX, "adamw: more than 2^31 - 1 tensors");
  std::vector<asd_adamw_tensor> list(n);
  std::vector<Tensor> held;  // gradients that had to be copied, until the call is enqueued
  const bool q8 = scales.given();
  require(q8 || !unbiased, "adamw: unbiased is a rounding of moments in 8 bits, which have scales");
  for (size_t i = 0; i < n; ++i) {
    asd_adamw_tensor& t = list[i];
    const Tensor &p = params.at(i, "params"), &g = grads.at(i, "grads");
    t.n = p.numel();
    t.type = type_of(p, "params"), t.grad_type = type_of(g, "grads");
    t.param = dense(c, p, "params", t.n, std::nullopt);
    if (g.sizes() != p.sizes()) fail(ASD_ERR_INVALID_ARG, "grads: " + shape_text(g.sizes()) + ", expected " + shape_text(p.sizes()));
    c.on_device(g, "grads");
    if (!g.is_contiguous()) {
      held.push_back(g.contiguous());
      t.grad = held.back().data_ptr();
    } else {
      t.grad = g.data_ptr();
    }
    t.master = masters.has(i) ? (float*)dense(c, masters.at(i, "masters"), "masters", t.n, at::kFloat) : nullptr;
    t.m = dense(c, m.at(i, "exp_avgs"), "exp_avgs", t.n, q8 ? at::kChar : at::kFloat);
    t.v = dense(c, v.at(i, "exp_avg_sqs"), "exp_avg_sqs", t.n, q8 ? at::kByte : at::kFloat);
    t.scales = q8 ? (float*)dense(c, scales.at(i, "scales"), "scales", (t.n + 255) / 256 * 2, at::kFloat) : nullptr;
  }
  asd_adamw_args a{};
  a.count = (int32_t)n, a.bits = !q8 ? 32 : unbiased ? 8 | ASD_ADAMW_UNBIASED : 8, a.tensors = list.data();
  a.beta1 = beta1, a.beta2 = beta2, a.eps = eps, a.weight_decay = weight_decay;
  Tensor rate;
  if (THPVariable_Check(lr.ptr())) {
    rate = THPVariable_Unpack(lr.ptr());
    a.lr_device = device_scalar(c, rate, "lr");
  } else {
    a.lr = lr.cast<double>();
  }
  a.grad_scale = device_scalar(c, grad_scale, "grad_scale"), a.skip = device_scalar(c, skip, "skip");
  a.step = (int64_t*)dense(c, step, "step", 2, at::kLong);
  check(asd_adamw(c.ops, &a, c.stream()));
  // autograd sees that they have changed
  auto changed = [](const Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  };
  for (size_t i = 0; i < n; ++i) {
    changed(params.at(i, "params")), changed(m.at(i, "exp_avgs")), changed(v.at(i, "exp_avg_sqs"));
    if (masters.has(i)) changed(masters.at(i, "masters"));
    if (q8) changed(scales.at(i, "scales"));
  }
  changed(step);
}

py::tuple adamw_moments(int64_t ops, int device, const Tensor& m, const Tensor& v, const Tensor& scales, int type) {
  const Call c{(asd_ops*)ops, device};
  asd_adamw_moments_args a{};
  a.n = m.numel(), a.type = type;
  a.m = dense(c, m, "exp_avg", a.n, at::kChar), a.v = dense(c, v, "exp_avg_sq", a.n, at::kByte);
  a.scales = (const float*)dense(c, scales, "scales", (a.n + 255) / 256 * 2, at::kFloat);
  Tensor fm = c.empty(m.sizes(), scalar_of(type)), fv = c.empty(m.sizes(), scalar_of(type));
  a.m_out = fm.data_ptr(), a.v_out = fv.data_ptr();
  check(asd_adamw_moments(c.ops, &a, c.stream()));
  return py::make_tuple(std::move(fm), std::move(fv));
}

int64_t create() {
  asd_ops* o = nullptr;
  check(asd_ops_create(&o));
  return (int64_t)o;
}
void destroy(int64_t ops) { asd_ops_destroy((asd_ops*)ops); }
void check_handle(int64_t ops, int device) { check(asd_ops_check((asd_ops*)ops, Call{(asd_ops*)ops, device}.stream())); }

}  // namespace

PYBIND11_MODULE(_asd_torch, m) {
  g_error = py::object(py::module_::import("paper_2505_03983_b200.binding").attr("AsdError")).release().ptr();
  m.def("create", &create);
  m.def("destroy", &destroy);
  m.def("check", &check_handle);
  m.def("add_rmsnorm", &add_rmsnorm);
  m.def("add_rmsnorm_backward", &add_rmsnorm_backward);
  m.def("quantize_i8", &quantize_i8);
  m.def("matmul_i8", &matmul_i8);
  m.def("gated_mlp", &gated_mlp);
  m.def("gated_mlp_backward", &gated_mlp_backward);
  m.def("block_rmsnorm", &block_rmsnorm);
  m.def("block_rmsnorm_backward", &block_rmsnorm_backward);
  m.def("adamw", &adamw);
  m.def("adamw_moments", &adamw_moments);
  m.def("linear", &linear);
  m.def("linear_backward", &linear_backward);
}
