// C entry points of the operators (include/asd_ops.h): checks of the arguments, the layout of the workspaces, and the
// sequence of kernels of each call.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "asd_ops_internal.h"

namespace asd {
namespace {

constexpr int kMsgBytes = 256;
thread_local char g_msg[kMsgBytes] = "";
thread_local cudaError_t g_launch = cudaSuccess;

bool is_type(int t) { return t == ASD_TYPE_F32 || t == ASD_TYPE_F16 || t == ASD_TYPE_BF16; }
bool off_element(const void* p, int es) { return (uintptr_t)p % (uintptr_t)es != 0; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The pieces of a workspace, one after the other on 256-byte boundaries; with a NULL base it only adds up sizes.
struct Cut {
  uint8_t* base;
  int64_t used = 0;
  void* take(int64_t bytes) {
    void* p = base ? base + used : nullptr;
    used += round_up(bytes, 256);
    return p;
  }
};

// An operand of a matrix product as the TMA can read it: itself, or a copy in the workspace with rows of a multiple of
// 16 bytes, which is added to the list of copies to be made.
Mat aligned_operand(Mat m, Cut* cut, Packs* packs) {
  if (mat_aligned(m)) return m;
  const int64_t ld = round_up(m.cols * m.es, 16) / m.es;
  void* p = cut->take(m.rows * ld * m.es);
  packs->src[packs->n] = m;
  packs->dst[packs->n] = p;
  packs->ld[packs->n++] = ld;
  return Mat{p, m.rows, m.cols, ld, m.es};
}

#define REQUIRE(cond, status, ...)                          \
  do {                                                      \
    if (!(cond)) return asd::ops_fail(status, __VA_ARGS__); \
  } while (0)

asd_status check_handle(const asd_ops* o, const void* args) {
  REQUIRE(o && args, ASD_ERR_INVALID_ARG, "the handle and the arguments must not be NULL");
  return ASD_OK;
}
asd_status check_device(const asd_ops* o) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(cudaGetLastError()));
  REQUIRE(dev == o->device, ASD_ERR_STATE, "the handle belongs to device %d, but device %d is current", o->device, dev);
  return ASD_OK;
}
// A matrix argument: `name`, rows of `cols` elements of `es` bytes.
asd_status check_mat(const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols, int es) {
  if (rows == 0) return ASD_OK;
  REQUIRE(p, ASD_ERR_INVALID_ARG, "%s must not be NULL", name);
  REQUIRE(ld >= cols, ASD_ERR_INVALID_ARG, "%s: the distance of two rows (%lld) is less than a row (%lld)", name, (long long)ld, (long long)cols);
  REQUIRE(ld <= (int64_t)1 << 36, ASD_ERR_INVALID_ARG, "%s: the distance of two rows (%lld) is over 2^36", name, (long long)ld);
  REQUIRE(!off_element(p, es), ASD_ERR_INVALID_ARG, "%s: the address is not a multiple of its element's %d bytes", name, es);
  return ASD_OK;
}
asd_status check_sizes(int32_t rows, int32_t a, const char* name) {
  REQUIRE(rows >= 0, ASD_ERR_INVALID_ARG, "rows must be >= 0: %d", rows);
  REQUIRE(a >= 1 && a <= kOpsMaxDim, ASD_ERR_INVALID_ARG, "%s must be 1..%d: %d", name, kOpsMaxDim, a);
  return ASD_OK;
}
asd_status check_workspace(const void* p, int64_t have, int64_t need) {
  if (need == 0) return ASD_OK;
  REQUIRE(p && ((uintptr_t)p & 255) == 0, ASD_ERR_INVALID_ARG, "a workspace of %lld bytes on a 256-byte boundary is needed", (long long)need);
  REQUIRE(have >= need, ASD_ERR_INVALID_ARG, "the workspace has %lld bytes, %lld are needed", (long long)have, (long long)need);
  return ASD_OK;
}
#define CHECK(call)                          \
  do {                                       \
    const asd_status st_ = (call);           \
    if (st_ != ASD_OK) return st_;           \
  } while (0)

// ---- matmul_i8 ----------------------------------------------------------------------------------------
asd_status check_matmul(const asd_ops* o, const asd_matmul_i8_args* a) {
  CHECK(check_handle(o, a));
  CHECK(check_sizes(a->rows, a->out, "out"));
  REQUIRE(a->k >= 1, ASD_ERR_INVALID_ARG, "k must be >= 1: %d", a->k);
  REQUIRE(a->k <= kOpsMaxK8, ASD_ERR_UNSUPPORTED, "a sum of more than %d 8-bit products can leave int32: k = %d", kOpsMaxK8, a->k);
  REQUIRE(is_type(a->out_type), ASD_ERR_INVALID_ARG, "unknown out_type %d", a->out_type);
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("a", a->a, a->ld_a, a->rows, a->k, 1));
  CHECK(check_mat("b", a->b, a->ld_b, a->out, a->k, 1));
  CHECK(check_mat("y", a->y, a->ld_y, a->rows, a->out, ops_type_size(a->out_type)));
  REQUIRE(a->a_scale && a->b_scale, ASD_ERR_INVALID_ARG, "a_scale and b_scale must not be NULL");
  REQUIRE(!off_element(a->a_scale, 4) && !off_element(a->b_scale, 4) && !off_element(a->bias, 4), ASD_ERR_INVALID_ARG,
          "scales and bias must be on 4-byte boundaries");
  return ASD_OK;
}
asd_status run_matmul(const asd_ops* o, const asd_matmul_i8_args* a, Cut* cut, bool launch, cudaStream_t st) {
  OpsGemm g{};
  Packs packs;
  g.epi = OPS_I8, g.type = a->out_type, g.m = a->rows, g.n = a->out, g.k[0] = a->k, g.parts = 1;
  g.a[0] = {aligned_operand(Mat{a->a, a->rows, a->k, a->ld_a, 1}, cut, &packs), false};
  g.b[0] = {aligned_operand(Mat{a->b, a->out, a->k, a->ld_b, 1}, cut, &packs), false};
  if (!launch) return ASD_OK;
  launch_packs(o, packs, st);
  g.c[0] = a->y, g.ldc = a->ld_y;
  g.scale_a = a->a_scale, g.scale_b = a->b_scale, g.bias = a->bias;
  return ops_gemm(o, g, false, st);
}

// ---- gated_mlp ----------------------------------------------------------------------------------------
// What is common to the forward and the backward arguments.
asd_status check_mlp(int32_t rows, int32_t width, int32_t hidden, int32_t type, int32_t act) {
  CHECK(check_sizes(rows, width, "width"));
  REQUIRE(hidden >= 1 && hidden <= kOpsMaxDim / 2, ASD_ERR_INVALID_ARG, "hidden must be 1..%d: %d", kOpsMaxDim / 2, hidden);
  REQUIRE(is_type(type), ASD_ERR_INVALID_ARG, "unknown type %d", type);
  REQUIRE(type != ASD_TYPE_F32, ASD_ERR_UNSUPPORTED, "the gated MLP takes F16 or BF16");
  REQUIRE(act == ASD_ACT_SILU || act == ASD_ACT_GELU, ASD_ERR_INVALID_ARG, "act must be SILU or GELU: %d", act);
  return ASD_OK;
}
int64_t padded_hidden(int64_t hidden) { return round_up(hidden, 8); }
// saved: h [rows, padded hidden], then the gate's two factors
int64_t saved_h_bytes(int64_t rows, int64_t hidden) { return round_up(rows * padded_hidden(hidden) * 2, 256); }

asd_status run_forward(const asd_ops* o, const asd_gated_mlp_args* a, Cut* cut, bool launch, cudaStream_t st) {
  const int64_t hp = padded_hidden(a->hidden);
  Packs packs;
  const Mat x = aligned_operand(Mat{a->x, a->rows, a->width, a->ld_x, 2}, cut, &packs);
  const Mat w = aligned_operand(Mat{a->w_in, 2 * (int64_t)a->hidden, a->width, a->ld_w_in, 2}, cut, &packs);
  const Mat wo = aligned_operand(Mat{a->w_out, a->width, a->hidden, a->ld_w_out, 2}, cut, &packs);
  void* h = a->saved ? a->saved : cut->take(a->rows * hp * 2);
  if (!launch) return ASD_OK;
  launch_packs(o, packs, st);
  OpsGemm g{};
  g.epi = OPS_GATE, g.type = a->type, g.act = a->act, g.m = a->rows, g.n = a->hidden, g.k[0] = a->width, g.parts = 1;
  g.a[0] = {x, false};
  g.b[0] = {Mat{w.p, a->hidden, w.cols, w.ld, 2}, false};
  g.b[1] = {Mat{(const uint8_t*)w.p + 2 * w.ld * a->hidden, a->hidden, w.cols, w.ld, 2}, false};
  g.c[0] = h, g.ldc = hp;
  g.kept = a->saved ? (uint8_t*)a->saved + saved_h_bytes(a->rows, a->hidden) : nullptr;
  CHECK(ops_gemm(o, g, false, st));
  OpsGemm y{};
  y.epi = OPS_STORE, y.type = a->type, y.m = a->rows, y.n = a->width, y.k[0] = a->hidden, y.parts = 1;
  y.a[0] = {Mat{h, a->rows, a->hidden, hp, 2}, false};
  y.b[0] = {wo, false};
  y.c[0] = a->y, y.ldc = a->ld_y;
  return ops_gemm(o, y, true, st);
}

asd_status run_backward(const asd_ops* o, const asd_gated_mlp_backward_args* a, Cut* cut, bool launch, cudaStream_t st) {
  const int64_t hp = padded_hidden(a->hidden), rows = a->rows;
  const bool inner = a->dx || a->dw_in;
  Packs packs;
  const Mat dy = aligned_operand(Mat{a->dy, rows, a->width, a->ld_dy, 2}, cut, &packs);
  Mat x{}, w{}, wo{};
  if (a->dw_in) x = aligned_operand(Mat{a->x, rows, a->width, a->ld_x, 2}, cut, &packs);
  if (a->dx) w = aligned_operand(Mat{a->w_in, 2 * (int64_t)a->hidden, a->width, a->ld_w_in, 2}, cut, &packs);
  if (inner) wo = aligned_operand(Mat{a->w_out, a->width, a->hidden, a->ld_w_out, 2}, cut, &packs);
  uint8_t* dgu = inner ? (uint8_t*)cut->take(rows * 2 * hp * 2) : nullptr;  // [rows, dg | du], each padded
  // the weights' gradients are sums over all rows: few outputs in slices
  const int s_in = a->dw_in ? sum_slices(o, a->hidden, a->width, rows, 6) : 1, s_out = a->dw_out ? sum_slices(o, a->width, a->hidden, rows, 6) : 1;
  float* part_in[2];
  for (float*& p : part_in) p = (float*)cut->take(part_bytes(a->hidden, a->width, s_in));
  float* part_out = (float*)cut->take(part_bytes(a->width, a->hidden, s_out));
  if (!launch) return ASD_OK;
  launch_packs(o, packs, st);
  const Mat dg{dgu, rows, a->hidden, 2 * hp, 2}, du{dgu + 2 * hp, rows, a->hidden, 2 * hp, 2};
  if (inner) {  // dh = dy w_out, and from it dg and du
    OpsGemm g{};
    g.epi = OPS_GATE_GRAD, g.type = a->type, g.m = rows, g.n = a->hidden, g.k[0] = a->width, g.parts = 1;
    g.a[0] = {dy, false};
    g.b[0] = {wo, true};
    g.c[0] = dgu, g.c[1] = dgu + 2 * hp, g.ldc = 2 * hp;
    g.kept = (uint8_t*)a->saved + saved_h_bytes(rows, a->hidden);
    CHECK(ops_gemm(o, g, false, st));
  }
  OpsGemm list[kMostProducts];
  int n = 0;
  auto product = [&](const Operand& p, const Operand& q, void* c, int64_t ldc, int64_t m, int64_t cols, int64_t k) -> OpsGemm& {
    OpsGemm g{};
    g.epi = OPS_STORE, g.type = a->type, g.m = m, g.n = cols, g.k[0] = k, g.parts = 1;
    g.a[0] = p, g.b[0] = q, g.c[0] = c, g.ldc = ldc;
    return list[n++] = g;
  };
  if (a->dx) {  // dg Wg + du Wu
    OpsGemm& g = product({dg, false}, {Mat{w.p, a->hidden, w.cols, w.ld, 2}, true}, a->dx, a->ld_dx, rows, a->width, a->hidden);
    g.parts = 2, g.k[1] = a->hidden;
    g.a[1] = {du, false};
    g.b[1] = {Mat{(const uint8_t*)w.p + 2 * w.ld * a->hidden, a->hidden, w.cols, w.ld, 2}, true};
  }
  if (a->dw_in) {  // dg^T x, du^T x
    for (int i = 0; i < 2; ++i) {
      uint8_t* c = (uint8_t*)a->dw_in + i * 2 * a->ld_dw_in * a->hidden;
      OpsGemm& g = product({i ? du : dg, true}, {x, true}, c, a->ld_dw_in, a->hidden, a->width, rows);
      g.slices = s_in, g.part = part_in[i];
    }
  }
  if (a->dw_out) {  // dy^T h
    OpsGemm& g = product({dy, true}, {Mat{a->saved, rows, a->hidden, hp, 2}, true}, a->dw_out, a->ld_dw_out, a->width, a->hidden, rows);
    g.slices = s_out, g.part = part_out;
  }
  return ops_gemm_list(o, list, n, st);
}

asd_status check_forward(const asd_ops* o, const asd_gated_mlp_args* a) {
  CHECK(check_handle(o, a));
  CHECK(check_mlp(a->rows, a->width, a->hidden, a->type, a->act));
  REQUIRE(a->reserved == 0, ASD_ERR_INVALID_ARG, "reserved must be 0");
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, 2));
  CHECK(check_mat("w_in", a->w_in, a->ld_w_in, 2 * (int64_t)a->hidden, a->width, 2));
  CHECK(check_mat("w_out", a->w_out, a->ld_w_out, a->width, a->hidden, 2));
  CHECK(check_mat("y", a->y, a->ld_y, a->rows, a->width, 2));
  REQUIRE(((uintptr_t)a->saved & 255) == 0, ASD_ERR_INVALID_ARG, "saved must be on a 256-byte boundary");
  return ASD_OK;
}
asd_status check_backward(const asd_ops* o, const asd_gated_mlp_backward_args* a) {
  CHECK(check_handle(o, a));
  CHECK(check_mlp(a->rows, a->width, a->hidden, a->type, a->act));
  REQUIRE(a->reserved == 0, ASD_ERR_INVALID_ARG, "reserved must be 0");
  if (a->dw_in) CHECK(check_mat("dw_in", a->dw_in, a->ld_dw_in, 2 * (int64_t)a->hidden, a->width, 2));
  if (a->dw_out) CHECK(check_mat("dw_out", a->dw_out, a->ld_dw_out, a->width, a->hidden, 2));
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("dy", a->dy, a->ld_dy, a->rows, a->width, 2));
  if (a->dw_in) CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, 2));
  if (a->dx) CHECK(check_mat("w_in", a->w_in, a->ld_w_in, 2 * (int64_t)a->hidden, a->width, 2));
  if (a->dx || a->dw_in) CHECK(check_mat("w_out", a->w_out, a->ld_w_out, a->width, a->hidden, 2));
  if (a->dx) CHECK(check_mat("dx", a->dx, a->ld_dx, a->rows, a->width, 2));
  REQUIRE(a->saved && ((uintptr_t)a->saved & 255) == 0, ASD_ERR_INVALID_ARG, "saved must be the forward call's buffer");
  return ASD_OK;
}

// ---- linear -------------------------------------------------------------------------------------------
// What is common to the forward and the backward arguments; `o_type` is that of y and the residual, or of dy.
asd_status check_layer(int32_t rows, int32_t width, int32_t out, int32_t type, int32_t o_type, const char* o_name, int32_t bias_type, int32_t act,
                       int32_t reserved) {
  CHECK(check_sizes(rows, width, "width"));
  REQUIRE(out >= 1 && out <= kOpsMaxDim, ASD_ERR_INVALID_ARG, "out must be 1..%d: %d", kOpsMaxDim, out);
  REQUIRE(is_type(type), ASD_ERR_INVALID_ARG, "unknown type %d", type);
  REQUIRE(type != ASD_TYPE_F32, ASD_ERR_UNSUPPORTED, "the linear layer takes F16 or BF16");
  REQUIRE(o_type == type || o_type == ASD_TYPE_F32, ASD_ERR_INVALID_ARG, "%s must be the type of x, or F32: %d", o_name, o_type);
  REQUIRE(bias_type == type || bias_type == ASD_TYPE_F32, ASD_ERR_INVALID_ARG, "bias_type must be the type of x, or F32: %d", bias_type);
  REQUIRE(act == ASD_ACT_NONE || act == ASD_ACT_SILU || act == ASD_ACT_GELU, ASD_ERR_INVALID_ARG, "unknown act %d", act);
  REQUIRE(reserved == 0, ASD_ERR_INVALID_ARG, "reserved must be 0");
  return ASD_OK;
}
asd_status check_linear_sizes(const asd_ops* o, const asd_linear_args* a) {
  CHECK(check_handle(o, a));
  return check_layer(a->rows, a->width, a->out, a->type, a->out_type, "out_type", a->bias_type, a->act, a->reserved);
}
asd_status check_linear(const asd_ops* o, const asd_linear_args* a) {
  CHECK(check_linear_sizes(o, a));
  if (a->rows == 0) return ASD_OK;
  const int es = ops_type_size(a->out_type);
  CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, 2));
  CHECK(check_mat("w", a->w, a->ld_w, a->out, a->width, 2));
  CHECK(check_mat("y", a->y, a->ld_y, a->rows, a->out, es));
  if (a->residual) CHECK(check_mat("residual", a->residual, a->ld_residual, a->rows, a->out, es));
  REQUIRE(!off_element(a->bias, ops_type_size(a->bias_type)), ASD_ERR_INVALID_ARG, "bias: the address is not a multiple of its element");
  REQUIRE(((uintptr_t)a->saved & 255) == 0, ASD_ERR_INVALID_ARG, "saved must be on a 256-byte boundary");
  return ASD_OK;
}
asd_status check_linear_backward(const asd_ops* o, const asd_linear_backward_args* a) {
  CHECK(check_handle(o, a));
  CHECK(check_layer(a->rows, a->width, a->out, a->type, a->dy_type, "dy_type", a->bias_type, a->act, a->reserved));
  REQUIRE(!off_element(a->dbias, ops_type_size(a->bias_type)), ASD_ERR_INVALID_ARG, "dbias: the address is not a multiple of its element");
  if (a->dw) CHECK(check_mat("dw", a->dw, a->ld_dw, a->out, a->width, 2));
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("dy", a->dy, a->ld_dy, a->rows, a->out, ops_type_size(a->dy_type)));
  if (a->dw) CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, 2));
  if (a->dx) CHECK(check_mat("w", a->w, a->ld_w, a->out, a->width, 2));
  if (a->dx) CHECK(check_mat("dx", a->dx, a->ld_dx, a->rows, a->width, 2));
  if (a->act != ASD_ACT_NONE)
    REQUIRE(a->saved && ((uintptr_t)a->saved & 255) == 0, ASD_ERR_INVALID_ARG, "saved must be the forward call's buffer");
  return ASD_OK;
}
asd_status run_linear(const asd_ops* o, const asd_linear_args* a, Cut* cut, bool launch, cudaStream_t st) {
  Packs packs;
  OpsGemm g{};
  const bool plain = !a->bias && !a->residual && a->act == ASD_ACT_NONE && a->out_type == a->type;
  g.epi = plain ? OPS_STORE : OPS_LINEAR, g.type = a->type, g.out_type = a->out_type, g.act = a->act;
  g.m = a->rows, g.n = a->out, g.k[0] = a->width, g.parts = 1;
  g.a[0] = {aligned_operand(Mat{a->x, a->rows, a->width, a->ld_x, 2}, cut, &packs), false};
  g.b[0] = {aligned_operand(Mat{a->w, a->out, a->width, a->ld_w, 2}, cut, &packs), false};
  if (!launch) return ASD_OK;
  launch_packs(o, packs, st);
  g.c[0] = a->y, g.ldc = a->ld_y;
  g.kept = a->act == ASD_ACT_NONE ? nullptr : (uint8_t*)a->saved;
  g.b1 = a->bias, g.b1_f32 = a->bias_type == ASD_TYPE_F32;
  g.res = a->residual, g.ldr = a->ld_residual;
  return ops_gemm(o, g, false, st);
}
asd_status run_linear_backward(const asd_ops* o, const asd_linear_backward_args* a, Cut* cut, bool launch, cudaStream_t st) {
  const int64_t rows = a->rows;
  const int es = ops_type_size(a->dy_type);
  const bool products = a->dx || a->dw, acts = a->act != ASD_ACT_NONE;
  Packs packs;
  const Mat dy{a->dy, rows, a->out, a->ld_dy, es};
  Mat x{}, w{}, dz = dy;  // dz is dy itself where there is nothing to change in it
  if (a->dw) x = aligned_operand(Mat{a->x, rows, a->width, a->ld_x, 2}, cut, &packs);
  if (a->dx) w = aligned_operand(Mat{a->w, a->out, a->width, a->ld_w, 2}, cut, &packs);
  LinearRows r{};
  if (products && (acts || es == 4 || !mat_aligned(dy))) {
    dz = Mat{nullptr, rows, a->out, round_up(a->out, 8), 2};
    dz.p = r.dz = cut->take(rows * dz.ld * 2);
    if (a->type == ASD_TYPE_F16 && es == 4) {  // what 32 bits hold may be far beyond the range of these 16
      r.peaks = (uint32_t*)cut->take(4 * linear_peaks(o, rows, a->out));
      r.unscale = (float*)cut->take(4);
    }
  }
  if (a->dbias) r.part = (float*)cut->take(linear_part_bytes(o, rows, a->out));
  const int slices = a->dw ? sum_slices(o, a->out, a->width, rows, 2) : 1;  // dw is a sum over all rows: few outputs in slices
  float* part = (float*)cut->take(part_bytes(a->out, a->width, slices));
  if (!launch) return ASD_OK;
  launch_packs(o, packs, st);
  if (r.dz || a->dbias) {
    r.rows = a->rows, r.out = a->out, r.type = a->type, r.dy_f32 = es == 4, r.bias_type = a->bias_type;
    r.dy = dy.p, r.ld_dy = dy.ld, r.kept = acts ? (const float*)a->saved : nullptr, r.ld_dz = dz.ld, r.dbias = a->dbias;
    CHECK(launch_linear_rows(o, r, st));
  }
  OpsGemm list[kMostProducts];
  int n = 0;
  if (a->dx) {  // dz w
    OpsGemm& g = list[n++] = OpsGemm{};
    g.epi = OPS_STORE, g.type = a->type, g.m = rows, g.n = a->width, g.k[0] = a->out, g.parts = 1;
    g.a[0] = {dz, false}, g.b[0] = {w, true}, g.c[0] = a->dx, g.ldc = a->ld_dx, g.unscale = r.unscale;
  }
  if (a->dw) {  // dz^T x
    OpsGemm& g = list[n++] = OpsGemm{};
    g.epi = OPS_STORE, g.type = a->type, g.m = a->out, g.n = a->width, g.k[0] = rows, g.parts = 1;
    g.a[0] = {dz, true}, g.b[0] = {x, true}, g.c[0] = a->dw, g.ldc = a->ld_dw, g.unscale = r.unscale;
    g.slices = slices, g.part = part;
  }
  return ops_gemm_list(o, list, n, st);
}

asd_status check_norm(int32_t rows, int32_t width, int32_t type, int32_t w_type, float eps, int32_t reserved, const void* weight) {
  CHECK(check_sizes(rows, width, "width"));
  REQUIRE(is_type(type), ASD_ERR_INVALID_ARG, "unknown type %d", type);
  REQUIRE(w_type == type || w_type == ASD_TYPE_F32, ASD_ERR_INVALID_ARG, "w_type must be that of x, or F32: %d", w_type);
  REQUIRE(eps >= 0.f && isfinite(eps), ASD_ERR_INVALID_ARG, "eps must be finite and >= 0");
  REQUIRE(reserved == 0, ASD_ERR_INVALID_ARG, "reserved must be 0");
  REQUIRE(!off_element(weight, ops_type_size(w_type)), ASD_ERR_INVALID_ARG, "weight: the address is not a multiple of its element");
  return ASD_OK;
}
asd_status check_norm_backward(const asd_ops* o, const asd_rmsnorm_backward_args* a) {
  CHECK(check_handle(o, a));
  CHECK(check_norm(a->rows, a->width, a->type, a->w_type, a->eps, a->reserved, a->weight));
  REQUIRE(!off_element(a->dw, ops_type_size(a->w_type)), ASD_ERR_INVALID_ARG, "dw: the address is not a multiple of its element");
  const int es = ops_type_size(a->type);
  CHECK(check_mat("dy", a->dy, a->ld_dy, a->rows, a->width, es));
  CHECK(check_mat("s", a->s, a->ld_s, a->rows, a->width, es));
  if (a->ds) CHECK(check_mat("ds", a->ds, a->ld_ds, a->rows, a->width, es));
  if (a->dx) CHECK(check_mat("dx", a->dx, a->ld_dx, a->rows, a->width, es));
  return ASD_OK;
}

// ---- block_rmsnorm --------------------------------------------------------------------------------------
// What is common to the forward and the backward arguments.
template <typename A>
asd_status check_block(const asd_ops* o, const A* a) {
  CHECK(check_handle(o, a));
  CHECK(check_norm(a->rows, a->width, a->type, a->w_type, a->eps, 0, a->weight));
  REQUIRE(a->post_type == a->type || a->post_type == ASD_TYPE_F32, ASD_ERR_INVALID_ARG, "post_type must be that of x, or F32: %d", a->post_type);
  REQUIRE(a->gate_type == a->type || a->gate_type == ASD_TYPE_F32, ASD_ERR_INVALID_ARG, "gate_type must be that of x, or F32: %d", a->gate_type);
  REQUIRE(!off_element(a->post_weight, ops_type_size(a->post_type)), ASD_ERR_INVALID_ARG, "post_weight: the address is not a multiple of its element");
  REQUIRE(a->post_norm == 0 || a->post_norm == 1, ASD_ERR_INVALID_ARG, "post_norm must be 0 or 1: %d", a->post_norm);
  REQUIRE(isfinite(a->alpha), ASD_ERR_INVALID_ARG, "alpha must be finite");
  if (a->rows == 0) return ASD_OK;
  const int es = ops_type_size(a->type);
  CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, es));
  CHECK(check_mat("s", a->s, a->ld_s, a->rows, a->width, es));
  if (a->gate) {
    REQUIRE(a->group >= 1 && a->rows % a->group == 0, ASD_ERR_INVALID_ARG, "group must be 1 or more, and rows (%d) a multiple of it: %d", a->rows, a->group);
    CHECK(check_mat("gate", a->gate, a->ld_gate, a->rows / a->group, a->width, ops_type_size(a->gate_type)));
  }
  return ASD_OK;
}
asd_status check_block_backward(const asd_ops* o, const asd_block_rmsnorm_backward_args* a) {
  CHECK(check_block(o, a));
  REQUIRE(!off_element(a->dweight, ops_type_size(a->w_type)) && !off_element(a->dpost_weight, ops_type_size(a->post_type)), ASD_ERR_INVALID_ARG,
          "dweight, dpost_weight: the address is not a multiple of its element");
  REQUIRE(!a->dgate || a->gate || a->rows == 0, ASD_ERR_INVALID_ARG, "dgate without a gate");
  if (a->rows == 0) return ASD_OK;
  const int es = ops_type_size(a->type);
  CHECK(check_mat("dy", a->dy, a->ld_dy, a->rows, a->width, es));
  if (a->ds) CHECK(check_mat("ds", a->ds, a->ld_ds, a->rows, a->width, es));
  if (a->dx) CHECK(check_mat("dx", a->dx, a->ld_dx, a->rows, a->width, es));
  if (a->dresidual) CHECK(check_mat("dresidual", a->dresidual, a->ld_dresidual, a->rows, a->width, es));
  if (a->dgate) CHECK(check_mat("dgate", a->dgate, a->ld_dgate, a->rows / a->group, a->width, ops_type_size(a->gate_type)));
  return ASD_OK;
}

// ---- adamw ----------------------------------------------------------------------------------------------
// Whether an address of a param stands in the list twice: its threads would then change it in an order of their own.  No memory is asked
// for: all that come after a batch of the list are looked up among it, in a table on the stack that is at most half full.
asd_status check_params(const asd_adamw_args* a) {
  constexpr int kBatch = 2048;
  const void* slots[2 * kBatch];
  for (int from = 0; from < a->count; from += std::min(kBatch, a->count - from)) {
    const int n = std::min(kBatch, a->count - from);
    size_t size = 64;
    while (size < 2 * (size_t)n) size *= 2;
    memset(slots, 0, size * sizeof(*slots));
    for (int i = from; i < a->count; ++i) {
      if (a->tensors[i].n == 0) continue;
      const void* p = a->tensors[i].param;
      size_t at = (((uintptr_t)p >> 1) * 0x9e3779b97f4a7c15ull >> 32) & (size - 1);
      while (slots[at] && slots[at] != p) at = (at + 1) & (size - 1);
      REQUIRE(!slots[at], ASD_ERR_INVALID_ARG, "tensor %d: its param stands in the list twice", i);
      if (i - from < n) slots[at] = p;
    }
  }
  return ASD_OK;
}
asd_status check_adamw(const asd_ops* o, const asd_adamw_args* a) {
  CHECK(check_handle(o, a));
  REQUIRE(a->bits == 32 || a->bits == 8 || a->bits == (8 | ASD_ADAMW_UNBIASED), ASD_ERR_INVALID_ARG, "bits must be 32, 8 or 8 | ASD_ADAMW_UNBIASED: %d", a->bits);
  REQUIRE(a->count >= 0 && (a->count == 0 || a->tensors), ASD_ERR_INVALID_ARG, "%d tensors, and no list of them", a->count);
  REQUIRE(a->lr >= 0 && isfinite(a->lr) && a->eps >= 0 && isfinite(a->eps) && a->weight_decay >= 0 && isfinite(a->weight_decay), ASD_ERR_INVALID_ARG,
          "lr, eps and weight_decay must be finite and >= 0");
  REQUIRE(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1, ASD_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  REQUIRE(a->step && !off_element(a->step, 8), ASD_ERR_INVALID_ARG, "step must not be NULL, and on an 8-byte boundary");
  REQUIRE(!off_element(a->lr_device, 4) && !off_element(a->grad_scale, 4) && !off_element(a->skip, 4), ASD_ERR_INVALID_ARG,
          "lr_device, grad_scale and skip must be on 4-byte boundaries");
  int64_t all = 0;
  for (int i = 0; i < a->count; ++i) {
    const asd_adamw_tensor& t = a->tensors[i];
    REQUIRE(t.n >= 0 && t.n <= kAdamMost, ASD_ERR_INVALID_ARG, "tensor %d: %lld elements", i, (long long)t.n);
    REQUIRE(is_type(t.type) && is_type(t.grad_type), ASD_ERR_INVALID_ARG, "tensor %d: unknown type %d or %d", i, t.type, t.grad_type);
    if (t.n == 0) continue;
    all += t.n + 1024;
    REQUIRE(all <= kAdamMost, ASD_ERR_UNSUPPORTED, "more than 2^36 elements in a call");
    REQUIRE(t.param && t.grad && t.m && t.v, ASD_ERR_INVALID_ARG, "tensor %d: param, grad, m and v must not be NULL", i);
    REQUIRE(!off_element(t.param, ops_type_size(t.type)) && !off_element(t.grad, ops_type_size(t.grad_type)) && !off_element(t.master, 4) &&
                (a->bits != 32 || (!off_element(t.m, 4) && !off_element(t.v, 4))),
            ASD_ERR_INVALID_ARG, "tensor %d: an address is not a multiple of its element", i);
    REQUIRE(a->bits == 32 || (t.scales && !off_element(t.scales, 8)), ASD_ERR_INVALID_ARG, "tensor %d: scales must not be NULL, and on an 8-byte boundary", i);
  }
  return check_params(a);
}

asd_status zero(void* p, int64_t ld, int64_t rows, int64_t cols, int es, cudaStream_t st) {
  if (cudaMemset2DAsync(p, (size_t)(ld * es), 0, (size_t)(cols * es), (size_t)rows, st) != cudaSuccess)
    return ops_fail(ASD_ERR_CUDA, "cudaMemset2DAsync: %s", cudaGetErrorString(cudaGetLastError()));
  return ASD_OK;
}

}  // namespace

asd_status ops_fail(asd_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_msg, kMsgBytes, fmt, ap);
  va_end(ap);
  return st;
}
void ops_note_launch(cudaError_t e) {
  if (e == cudaSuccess) return;
  cudaGetLastError();
  if (g_launch == cudaSuccess) g_launch = e;
}
asd_status ops_launched(const char* what) {
  const cudaError_t e = g_launch;
  g_launch = cudaSuccess;
  return e == cudaSuccess ? ASD_OK : ops_fail(ASD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
int ops_type_size(int type) { return type == ASD_TYPE_F32 ? 4 : is_type(type) ? 2 : 0; }

}  // namespace asd

using namespace asd;

extern "C" {

const char* asd_ops_last_error(void) { return g_msg; }

asd_status asd_ops_create(asd_ops** out) {
  REQUIRE(out, ASD_ERR_INVALID_ARG, "out must not be NULL");
  *out = nullptr;
  int dev = 0, major = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return ops_fail(ASD_ERR_CUDA, "no CUDA device");
  }
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return ops_fail(ASD_ERR_CUDA, "cudaDeviceGetAttribute: %s", cudaGetErrorString(cudaGetLastError()));
  REQUIRE(major == 10, ASD_ERR_UNSUPPORTED, "the library is built for sm_100a; device %d has compute capability %d.x", dev, major);
  CHECK(ops_rows_prepare());
  CHECK(ops_gemm_prepare());
  CHECK(ops_stream_prepare());
  CHECK(ops_split_prepare());
  CHECK(ops_block_prepare());
  asd_ops* o = new (std::nothrow) asd_ops();
  REQUIRE(o, ASD_ERR_OOM, "out of host memory");
  o->device = dev;
  o->num_sms = sms;
  if (cudaMalloc(reinterpret_cast<void**>(&o->err), 256) != cudaSuccess) {
    cudaGetLastError();
    delete o;
    return ops_fail(ASD_ERR_OOM, "out of device memory");
  }
  if (cudaMemset(o->err, 0, 256) != cudaSuccess) {
    cudaFree(o->err);
    delete o;
    return ops_fail(ASD_ERR_CUDA, "cudaMemset: %s", cudaGetErrorString(cudaGetLastError()));
  }
  *out = o;
  return ASD_OK;
}

void asd_ops_destroy(asd_ops* o) {
  if (!o) return;
  cudaFree(o->err);
  delete o;
}

asd_status asd_ops_check(asd_ops* o, void* stream) {
  REQUIRE(o, ASD_ERR_INVALID_ARG, "the handle must not be NULL");
  CHECK(check_device(o));
  cudaStream_t st = (cudaStream_t)stream;
  int word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, o->err, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return ops_fail(ASD_ERR_CUDA, "%s", cudaGetErrorString(e));
  }
  if (word == 0) return ASD_OK;
  e = cudaMemsetAsync(o->err, 0, sizeof(int), st);
  if (e != cudaSuccess) cudaGetLastError();
  return ops_fail(ASD_ERR_TIMEOUT, "a wait inside a kernel ran out of its limit: outputs since the last check are undefined");
}

asd_status asd_add_rmsnorm(asd_ops* o, const asd_rmsnorm_args* a, void* stream) {
  CHECK(check_handle(o, a));
  CHECK(check_norm(a->rows, a->width, a->type, a->w_type, a->eps, a->reserved, a->weight));
  if (a->rows == 0) return ASD_OK;
  const int es = ops_type_size(a->type);
  CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->width, es));
  if (a->residual) CHECK(check_mat("residual", a->residual, a->ld_residual, a->rows, a->width, es));
  if (a->sum) CHECK(check_mat("sum", a->sum, a->ld_sum, a->rows, a->width, es));
  CHECK(check_mat("y", a->y, a->ld_y, a->rows, a->width, a->scale ? 1 : es));
  REQUIRE(!off_element(a->scale, 4), ASD_ERR_INVALID_ARG, "scale must be on a 4-byte boundary");
  CHECK(check_device(o));
  launch_rmsnorm(o, a, (cudaStream_t)stream);
  return ops_launched("add_rmsnorm");
}

asd_status asd_add_rmsnorm_backward_workspace(asd_ops* o, const asd_rmsnorm_backward_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_handle(o, a));
  CHECK(check_norm(a->rows, a->width, a->type, a->w_type, a->eps, a->reserved, nullptr));
  *bytes = rmsnorm_backward_bytes(o, a);
  return ASD_OK;
}
asd_status asd_add_rmsnorm_backward(asd_ops* o, const asd_rmsnorm_backward_args* a, void* stream) {
  CHECK(check_norm_backward(o, a));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, rmsnorm_backward_bytes(o, a)));
  CHECK(check_device(o));
  cudaStream_t st = (cudaStream_t)stream;
  if (a->rows == 0) return a->dw ? zero(a->dw, a->width, 1, a->width, ops_type_size(a->w_type), st) : ASD_OK;
  if (!a->dx && !a->dw) return ASD_OK;
  launch_rmsnorm_backward(o, a, st);
  return ops_launched("add_rmsnorm_backward");
}

asd_status asd_quantize_i8(asd_ops* o, const asd_quantize_args* a, void* stream) {
  CHECK(check_handle(o, a));
  CHECK(check_sizes(a->rows, a->width, "width"));
  REQUIRE(is_type(a->type), ASD_ERR_INVALID_ARG, "unknown type %d", a->type);
  REQUIRE(a->act == ASD_ACT_NONE || a->act == ASD_ACT_SILU || a->act == ASD_ACT_GELU, ASD_ERR_INVALID_ARG, "unknown act %d", a->act);
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("x", a->x, a->ld_x, a->rows, a->act == ASD_ACT_NONE ? a->width : 2 * (int64_t)a->width, ops_type_size(a->type)));
  CHECK(check_mat("q", a->q, a->ld_q, a->rows, a->width, 1));
  REQUIRE(a->scale && !off_element(a->scale, 4), ASD_ERR_INVALID_ARG, "scale must not be NULL, and on a 4-byte boundary");
  CHECK(check_device(o));
  launch_quantize(o, a, (cudaStream_t)stream);
  return ops_launched("quantize_i8");
}

asd_status asd_matmul_i8_workspace(asd_ops* o, const asd_matmul_i8_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_matmul(o, a));
  Cut cut{nullptr};
  *bytes = 0;
  if (a->rows) CHECK(run_matmul(o, a, &cut, false, nullptr));
  *bytes = cut.used;
  return ASD_OK;
}
asd_status asd_matmul_i8(asd_ops* o, const asd_matmul_i8_args* a, void* stream) {
  CHECK(check_matmul(o, a));
  if (a->rows == 0) return ASD_OK;
  Cut need{nullptr}, cut{(uint8_t*)a->workspace};
  CHECK(run_matmul(o, a, &need, false, nullptr));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, need.used));
  CHECK(check_device(o));
  return run_matmul(o, a, &cut, true, (cudaStream_t)stream);
}

asd_status asd_gated_mlp_saved(asd_ops* o, const asd_gated_mlp_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_handle(o, a));
  CHECK(check_mlp(a->rows, a->width, a->hidden, a->type, a->act));
  *bytes = saved_h_bytes(a->rows, a->hidden) + gated_kept_bytes(a->rows, a->hidden);
  return ASD_OK;
}
asd_status asd_gated_mlp_forward_workspace(asd_ops* o, const asd_gated_mlp_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_forward(o, a));
  Cut cut{nullptr};
  *bytes = 0;
  if (a->rows) CHECK(run_forward(o, a, &cut, false, nullptr));
  *bytes = cut.used;
  return ASD_OK;
}
asd_status asd_gated_mlp_forward(asd_ops* o, const asd_gated_mlp_args* a, void* stream) {
  CHECK(check_forward(o, a));
  if (a->rows == 0) return ASD_OK;
  Cut need{nullptr}, cut{(uint8_t*)a->workspace};
  CHECK(run_forward(o, a, &need, false, nullptr));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, need.used));
  CHECK(check_device(o));
  return run_forward(o, a, &cut, true, (cudaStream_t)stream);
}

asd_status asd_gated_mlp_backward_workspace(asd_ops* o, const asd_gated_mlp_backward_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_backward(o, a));
  Cut cut{nullptr};
  *bytes = 0;
  if (a->rows) CHECK(run_backward(o, a, &cut, false, nullptr));
  *bytes = cut.used;
  return ASD_OK;
}
asd_status asd_gated_mlp_backward(asd_ops* o, const asd_gated_mlp_backward_args* a, void* stream) {
  CHECK(check_backward(o, a));
  cudaStream_t st = (cudaStream_t)stream;
  if (a->rows == 0) {
    CHECK(check_device(o));
    if (a->dw_in) CHECK(zero(a->dw_in, a->ld_dw_in, 2 * (int64_t)a->hidden, a->width, 2, st));
    if (a->dw_out) CHECK(zero(a->dw_out, a->ld_dw_out, a->width, a->hidden, 2, st));
    return ASD_OK;
  }
  Cut need{nullptr}, cut{(uint8_t*)a->workspace};
  CHECK(run_backward(o, a, &need, false, nullptr));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, need.used));
  CHECK(check_device(o));
  return run_backward(o, a, &cut, true, st);
}

asd_status asd_linear_saved(asd_ops* o, const asd_linear_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_linear_sizes(o, a));
  *bytes = a->act == ASD_ACT_NONE ? 0 : linear_kept_bytes(a->rows, a->out);
  return ASD_OK;
}
asd_status asd_linear_forward_workspace(asd_ops* o, const asd_linear_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_linear(o, a));
  Cut cut{nullptr};
  *bytes = 0;
  if (a->rows) CHECK(run_linear(o, a, &cut, false, nullptr));
  *bytes = cut.used;
  return ASD_OK;
}
asd_status asd_linear_forward(asd_ops* o, const asd_linear_args* a, void* stream) {
  CHECK(check_linear(o, a));
  if (a->rows == 0) return ASD_OK;
  Cut need{nullptr}, cut{(uint8_t*)a->workspace};
  CHECK(run_linear(o, a, &need, false, nullptr));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, need.used));
  CHECK(check_device(o));
  return run_linear(o, a, &cut, true, (cudaStream_t)stream);
}
asd_status asd_linear_backward_workspace(asd_ops* o, const asd_linear_backward_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_linear_backward(o, a));
  Cut cut{nullptr};
  *bytes = 0;
  if (a->rows) CHECK(run_linear_backward(o, a, &cut, false, nullptr));
  *bytes = cut.used;
  return ASD_OK;
}
asd_status asd_linear_backward(asd_ops* o, const asd_linear_backward_args* a, void* stream) {
  CHECK(check_linear_backward(o, a));
  cudaStream_t st = (cudaStream_t)stream;
  if (a->rows == 0) {
    CHECK(check_device(o));
    if (a->dw) CHECK(zero(a->dw, a->ld_dw, a->out, a->width, 2, st));
    if (a->dbias) CHECK(zero(a->dbias, a->out, 1, a->out, ops_type_size(a->bias_type), st));
    return ASD_OK;
  }
  Cut need{nullptr}, cut{(uint8_t*)a->workspace};
  CHECK(run_linear_backward(o, a, &need, false, nullptr));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, need.used));
  CHECK(check_device(o));
  return run_linear_backward(o, a, &cut, true, st);
}

asd_status asd_block_rmsnorm(asd_ops* o, const asd_block_rmsnorm_args* a, void* stream) {
  CHECK(check_block(o, a));
  if (a->rows == 0) return ASD_OK;
  CHECK(check_mat("residual", a->residual, a->ld_residual, a->rows, a->width, ops_type_size(a->type)));
  CHECK(check_mat("y", a->y, a->ld_y, a->rows, a->width, a->scale ? 1 : ops_type_size(a->type)));
  REQUIRE(!off_element(a->scale, 4), ASD_ERR_INVALID_ARG, "scale must be on a 4-byte boundary");
  CHECK(check_device(o));
  launch_block_rmsnorm(o, a, (cudaStream_t)stream);
  return ops_launched("block_rmsnorm");
}
asd_status asd_block_rmsnorm_backward_workspace(asd_ops* o, const asd_block_rmsnorm_backward_args* a, int64_t* bytes) {
  REQUIRE(bytes, ASD_ERR_INVALID_ARG, "bytes must not be NULL");
  CHECK(check_block_backward(o, a));
  *bytes = block_rmsnorm_backward_bytes(o, a);
  return ASD_OK;
}
asd_status asd_block_rmsnorm_backward(asd_ops* o, const asd_block_rmsnorm_backward_args* a, void* stream) {
  CHECK(check_block_backward(o, a));
  CHECK(check_workspace(a->workspace, a->workspace_bytes, block_rmsnorm_backward_bytes(o, a)));
  CHECK(check_device(o));
  cudaStream_t st = (cudaStream_t)stream;
  if (a->rows == 0) {
    if (a->dweight) CHECK(zero(a->dweight, a->width, 1, a->width, ops_type_size(a->w_type), st));
    if (a->dpost_weight) CHECK(zero(a->dpost_weight, a->width, 1, a->width, ops_type_size(a->post_type), st));
    return ASD_OK;
  }
  if (!a->dx && !a->dresidual && !a->dweight && !a->dpost_weight && !a->dgate) return ASD_OK;
  launch_block_rmsnorm_backward(o, a, st);
  return ops_launched("block_rmsnorm_backward");
}

asd_status asd_adamw(asd_ops* o, const asd_adamw_args* a, void* stream) {
  CHECK(check_adamw(o, a));
  CHECK(check_device(o));
  launch_adamw(o, a, (cudaStream_t)stream);
  return ops_launched("adamw");
}
asd_status asd_adamw_moments(asd_ops* o, const asd_adamw_moments_args* a, void* stream) {
  CHECK(check_handle(o, a));
  REQUIRE(a->n >= 0 && a->n <= kAdamMost, ASD_ERR_INVALID_ARG, "%lld elements", (long long)a->n);
  REQUIRE(is_type(a->type), ASD_ERR_INVALID_ARG, "unknown type %d", a->type);
  REQUIRE(a->reserved == 0, ASD_ERR_INVALID_ARG, "reserved must be 0");
  if (a->n == 0) return ASD_OK;
  REQUIRE(a->m && a->v && a->m_out && a->v_out, ASD_ERR_INVALID_ARG, "m, v, m_out and v_out must not be NULL");
  REQUIRE(a->scales && !off_element(a->scales, 8), ASD_ERR_INVALID_ARG, "scales must not be NULL, and on an 8-byte boundary");
  REQUIRE(!off_element(a->m_out, ops_type_size(a->type)) && !off_element(a->v_out, ops_type_size(a->type)), ASD_ERR_INVALID_ARG,
          "m_out, v_out: an address is not a multiple of its element");
  CHECK(check_device(o));
  launch_moments(o, a, (cudaStream_t)stream);
  return ops_launched("adamw_moments");
}

}  // extern "C"
