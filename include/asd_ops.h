/*
 * asd_ops.h - C ABI of the operators that a denoiser is trained and served with, next to the sampler of asd.h.
 *
 * A denoiser that is wider or deeper than the residual MLP of asd.h is usually made of blocks
 *     s = x + r                                  the residual stream
 *     n = s / sqrt(mean(s^2) + eps) * w          its root-mean-square norm
 *     y = (act(n Wg^T) * (n Wu^T)) Wo^T          two projections, their gated product, and the way back
 * trained in 16 bits and served in 16 bits or with 8-bit integers.  These entry points are the block's parts:
 * the norm (16 / 32 bits with its gradients, or 8 bits with a scale per row), the row quantisation with or
 * without the gate, the 8-bit matrix product, and the gated MLP with its gradients.  Beside them stand the linear layer
 * with bias, activation and residual (a layer of the residual MLP of asd.h), the norms between two blocks with the branch's
 * gate and scale, and the optimizer's step.
 *
 * Conventions
 *  - Those of asd.h: plain C, every function returns an asd_status and never throws, aborts or exits; the caller
 *    owns every buffer; there is no CPU fallback.
 *  - Pointers are device memory of the device that was current in asd_ops_create, which must be current in the
 *    call; matrices are row-major with contiguous rows, ld_* is the distance of two rows in ELEMENTS
 *    (>= the row's length).  Any length, distance and element-aligned address is accepted: operands of the matrix
 *    products whose address or distance is not a multiple of 16 bytes are copied to the workspace first; such rows of
 *    the other operators come through shared memory in aligned pieces (up to 256 elements, and over 16384 or, in
 *    the gradients of the norms, 8192: element by element).
 *  - Work is enqueued on the stream given in the call (a cudaStream_t as void*; NULL = the default stream) and the
 *    call returns.  No call synchronises, allocates or keeps anything of its inputs, so calls may be captured in
 *    a CUDA graph, and one handle may serve several streams and threads.
 *  - Workspaces are the caller's: asd_*_workspace returns the bytes that the call with the same arguments needs
 *    (their address 256-byte aligned; 0 when none).  A workspace may be reused by the next call on the same stream.
 *  - No output may overlap an input or another output, except that asd_add_rmsnorm's sum and asd_block_rmsnorm's s may be
 *    its x or its residual, asd_linear_forward's y its residual, and asd_add_rmsnorm_backward's dx its dy or ds, with
 *    the same row distance.
 *  - Zero rows is a valid call that does nothing (gradients of weights are then set to zero).
 *  - Sums, statistics and the activation are in 32 bits (the norm of a row whose sum of squares is beyond them is 0).  Results do not depend on the order in which blocks of a
 *    kernel run: the same inputs give the same bits.
 *  - A call that returns an error has enqueued nothing, except for CUDA: a launch failed after others may have been
 *    enqueued, and the outputs are undefined.
 */
#ifndef ASD_OPS_H
#define ASD_OPS_H

#include <stdint.h>

#include "asd.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct asd_ops asd_ops; /* opaque: the device, and an error word on it */

typedef enum { ASD_TYPE_F32 = 0, ASD_TYPE_F16 = 1, ASD_TYPE_BF16 = 2 } asd_type;

/*
 * SILU: g / (1 + exp(-g)).  GELU: g Phi(g) with the normal distribution function (not the tanh form).  Both are computed in 32 bits
 * with the approximate exponential and reciprocal, for every type: off by at most (4 + |g|) 2^-23 and (8 + g^2) 2^-23 of their
 * value, as long as that is above 2^-119 (below, they may be 0).
 */
typedef enum { ASD_ACT_NONE = 0, ASD_ACT_SILU = 1, ASD_ACT_GELU = 2 } asd_act;

asd_status asd_ops_create(asd_ops** out);
void asd_ops_destroy(asd_ops* ops);
/* Message of the calling thread's last failed operator call ("" if none); never NULL. */
const char* asd_ops_last_error(void);
/*
 * Every wait inside the matrix kernels is bounded; when its limit (about 0.2 s) runs out the kernel records that
 * and finishes with undefined outputs.  This call synchronises the stream, returns ASD_ERR_TIMEOUT if that has
 * happened on this handle since the last check (and clears it), CUDA if the stream has failed, OK otherwise.  Not to be
 * called while the stream is being captured.
 */
asd_status asd_ops_check(asd_ops* ops, void* cuda_stream);

/*
 * s = x + r, rounded to the type of x, and y = s / sqrt(mean(s^2) + eps) * w of every row of the rounded s.
 *   scale == NULL: y has the type of x.
 *   scale != NULL: y is int8 and scale [rows] fp32:  m = max(max_j |y_j|, 2^-100),  scale = m / 127,
 *                  q_j = round-to-nearest-even(y_j * (127 / m)), |q_j| <= 127, y computed and kept in fp32.
 *                  A row with a NaN or an infinity among its y has q = 0 and scale = NaN.
 * residual may be NULL (s = x); sum may be NULL (s is not stored).  weight [width] has type w_type: that of x,
 * or F32; NULL means 1.
 */
typedef struct {
  int32_t rows, width;
  int32_t type, w_type; /* asd_type */
  float eps;            /* >= 0 */
  int32_t reserved;     /* 0 */
  const void* x;        int64_t ld_x;
  const void* residual; int64_t ld_residual;
  const void* weight;
  void* sum;            int64_t ld_sum;
  void* y;              int64_t ld_y;
  float* scale;
} asd_rmsnorm_args;
asd_status asd_add_rmsnorm(asd_ops* ops, const asd_rmsnorm_args* args, void* cuda_stream);

/*
 * Gradients of the form without scale: with z = s rho, rho = 1 / sqrt(mean(s^2) + eps),
 *   dx = rho (dy w - z mean(dy w z)) + ds        (the gradient of x and of the residual alike)
 *   dw = sum over rows of dy z                   (w_type)
 * ds, the gradient that reaches s itself, may be NULL (0).  dx and dw may each be NULL (not computed); weight NULL
 * means 1, with dw in F32 unless w_type says otherwise.
 */
typedef struct {
  int32_t rows, width;
  int32_t type, w_type;
  float eps;
  int32_t reserved;
  const void* dy; int64_t ld_dy;
  const void* s;  int64_t ld_s;
  const void* ds; int64_t ld_ds;
  const void* weight;
  void* dx;       int64_t ld_dx;
  void* dw;
  void* workspace; int64_t workspace_bytes;
} asd_rmsnorm_backward_args;
asd_status asd_add_rmsnorm_backward_workspace(asd_ops* ops, const asd_rmsnorm_backward_args* args, int64_t* bytes);
asd_status asd_add_rmsnorm_backward(asd_ops* ops, const asd_rmsnorm_backward_args* args, void* cuda_stream);

/*
 * Rows in 8 bits, q and scale as in asd_add_rmsnorm.  act NONE: of x [rows, width].  SILU / GELU: of
 * h_j = act(x_j) x_{width + j}, x [rows, 2 width] with the gate first; h is computed and kept in fp32.
 */
typedef struct {
  int32_t rows, width;
  int32_t type, act;
  const void* x; int64_t ld_x;
  int8_t* q;     int64_t ld_q;
  float* scale; /* [rows] */
} asd_quantize_args;
asd_status asd_quantize_i8(asd_ops* ops, const asd_quantize_args* args, void* cuda_stream);

/*
 * y[i, j] = (sum_k a[i, k] b[j, k]) a_scale[i] b_scale[j] + bias[j], the sum exact in int32 (k <= 131071, otherwise
 * UNSUPPORTED), the rest in fp32, rounded once to out_type.  a [rows, k] (a scale per token), b [out, k] (a scale
 * per channel) int8; bias [out] fp32 or NULL.
 */
typedef struct {
  int32_t rows, out, k;
  int32_t out_type;
  const int8_t* a; int64_t ld_a;
  const int8_t* b; int64_t ld_b;
  const float* a_scale;
  const float* b_scale;
  const float* bias;
  void* y; int64_t ld_y;
  void* workspace; int64_t workspace_bytes;
} asd_matmul_i8_args;
asd_status asd_matmul_i8_workspace(asd_ops* ops, const asd_matmul_i8_args* args, int64_t* bytes);
asd_status asd_matmul_i8(asd_ops* ops, const asd_matmul_i8_args* args, void* cuda_stream);

/*
 * y = h w_out^T,  h = act(g) u,  [g | u] = x w_in^T.   x [rows, width], w_in [2 hidden, width] with the gate's rows
 * first, w_out [width, hidden], y [rows, width]; F16 or BF16 throughout (UNSUPPORTED otherwise), sums in fp32, h
 * rounded to the type, act SILU or GELU.
 * saved != NULL: what asd_gated_mlp_backward needs is kept there (asd_gated_mlp_saved gives its bytes; address
 * 256-byte aligned, layout private to the library): h, and the gate's two factors u act'(g) and act(g) in the upper 24
 * of their 32 bits, truncated (off by less than 2^-15 of themselves, towards zero).
 */
typedef struct {
  int32_t rows, width, hidden;
  int32_t type, act;
  int32_t reserved;
  const void* x;     int64_t ld_x;
  const void* w_in;  int64_t ld_w_in;
  const void* w_out; int64_t ld_w_out;
  void* y;           int64_t ld_y;
  void* saved;
  void* workspace;   int64_t workspace_bytes;
} asd_gated_mlp_args;
asd_status asd_gated_mlp_saved(asd_ops* ops, const asd_gated_mlp_args* args, int64_t* bytes);
asd_status asd_gated_mlp_forward_workspace(asd_ops* ops, const asd_gated_mlp_args* args, int64_t* bytes);
asd_status asd_gated_mlp_forward(asd_ops* ops, const asd_gated_mlp_args* args, void* cuda_stream);

/*
 * Gradients:  dh = dy w_out,  dg = dh u act'(g),  du = dh act(g)  (rounded to the type),
 *   dx = [dg | du] w_in,   dw_in = [dg | du]^T x,   dw_out = dy^T h.
 * x, w_in, w_out and `saved` as in the forward call; dx, dw_in, dw_out may each be NULL (not computed).
 */
typedef struct {
  int32_t rows, width, hidden;
  int32_t type, act;
  int32_t reserved;
  const void* dy;    int64_t ld_dy;
  const void* x;     int64_t ld_x;
  const void* w_in;  int64_t ld_w_in;
  const void* w_out; int64_t ld_w_out;
  const void* saved;
  void* dx;          int64_t ld_dx;
  void* dw_in;       int64_t ld_dw_in;
  void* dw_out;      int64_t ld_dw_out;
  void* workspace;   int64_t workspace_bytes;
} asd_gated_mlp_backward_args;
asd_status asd_gated_mlp_backward_workspace(asd_ops* ops, const asd_gated_mlp_backward_args* args, int64_t* bytes);
asd_status asd_gated_mlp_backward(asd_ops* ops, const asd_gated_mlp_backward_args* args, void* cuda_stream);

/*
 * y = r + act(z),  z = x w^T + bias: a layer of the residual MLP that the sampler runs, and any other projection.
 * x [rows, width], w [out, width] F16 or BF16 (UNSUPPORTED otherwise), sums, bias, activation and residual in fp32, rounded
 * once.  (The tensor cores' fp32 sums are truncated: one of `width` products is off by up to (width + 8) 2^-23 of the sum of
 * their magnitudes; measured 4.4e-6 of z at a width of 4096, 1e-6 at 1024.)  y and residual [rows, out] have
 * out_type: type, or F32; bias [out] has bias_type: type, or F32.  bias and residual may be NULL (0), act NONE, SILU or GELU.  y
 * may be the residual itself, with the same row distance.
 * saved != NULL (with an activation): act'(z) for asd_linear_backward, in fp32 (asd_linear_saved gives the bytes, 0 for act
 * NONE; address 256-byte aligned, layout private to the library).
 */
typedef struct {
  int32_t rows, width, out;
  int32_t type, out_type, bias_type;
  int32_t act;
  int32_t reserved;
  const void* x;        int64_t ld_x;
  const void* w;        int64_t ld_w;
  const void* bias;
  const void* residual; int64_t ld_residual;
  void* y;              int64_t ld_y;
  void* saved;
  void* workspace;      int64_t workspace_bytes;
} asd_linear_args;
asd_status asd_linear_saved(asd_ops* ops, const asd_linear_args* args, int64_t* bytes);
asd_status asd_linear_forward_workspace(asd_ops* ops, const asd_linear_args* args, int64_t* bytes);
asd_status asd_linear_forward(asd_ops* ops, const asd_linear_args* args, void* cuda_stream);

/*
 * Gradients:  dz = dy act'(z)  (rounded to the type for the products; F16 with a dy in F32: times a power of two that goes by dy's
 * largest finite magnitude and is taken off their sums, so that a dz of 2^-28 of that still has all bits of F16),
 *   dx = dz w,   dw = dz^T x,   dbias = sum over rows of dz before that rounding  (bias_type);
 * the residual's is dy.  dy has dy_type: type, or F32.  x, w and `saved` as in the forward call (saved is not read for act
 * NONE); dx, dw, dbias may each be NULL (not computed).
 */
typedef struct {
  int32_t rows, width, out;
  int32_t type, dy_type, bias_type;
  int32_t act;
  int32_t reserved;
  const void* dy; int64_t ld_dy;
  const void* x;  int64_t ld_x;
  const void* w;  int64_t ld_w;
  const void* saved;
  void* dx;       int64_t ld_dx;
  void* dw;       int64_t ld_dw;
  void* dbias;
  void* workspace; int64_t workspace_bytes;
} asd_linear_backward_args;
asd_status asd_linear_backward_workspace(asd_ops* ops, const asd_linear_backward_args* args, int64_t* bytes);
asd_status asd_linear_backward(asd_ops* ops, const asd_linear_backward_args* args, void* cuda_stream);

/*
 * Between two blocks, for an x that the first has made and the residual r that went around it:
 *   n = x / sqrt(mean(x^2) + eps)   (post_norm 1; post_norm 0: n = x)
 *   s = r + alpha gate w_post n     rounded to the type of x
 *   y = s / sqrt(mean(s^2) + eps) w of every row of the rounded s, the next block's input; int8 with scale != NULL, as in
 *                                   asd_add_rmsnorm
 * Row i takes row i / group of gate [rows / group, width] (a gate for each chain; group = rows: one for all).  weight (w),
 * post_weight (w_post) [width] and gate have types of their own: that of x, or F32; each may be NULL (1).  s may be x or the
 * residual itself, with the same row distance.
 */
typedef struct {
  int32_t rows, width;
  int32_t type, w_type, post_type, gate_type; /* asd_type */
  int32_t post_norm;
  int32_t group; /* with a gate: 1.., rows a multiple of it */
  float eps;     /* >= 0 */
  float alpha;
  const void* x;        int64_t ld_x;
  const void* residual; int64_t ld_residual;
  const void* weight;
  const void* post_weight;
  const void* gate;     int64_t ld_gate;
  void* s;              int64_t ld_s;
  void* y;              int64_t ld_y;
  float* scale;
} asd_block_rmsnorm_args;
asd_status asd_block_rmsnorm(asd_ops* ops, const asd_block_rmsnorm_args* args, void* cuda_stream);

/*
 * Gradients of the form without scale: with z = s rho, rho = 1 / sqrt(mean(s^2) + eps), rho_x that of x (post_norm 0: 1),
 *   dS = ds + rho (dy w - z mean(dy w z))             dresidual = dS
 *   c = alpha gate w_post,  dx = rho_x (c dS - n mean(c dS n))      (post_norm 0: dx = c dS)
 *   dweight = sum over rows of dy z,  dpost_weight = sum over rows of alpha gate dS n,
 *   dgate[k] = sum over the rows of gate row k of alpha w_post dS n
 * each rounded once.  ds, the gradient that reaches s itself, may be NULL (0).  The outputs may each be NULL (not computed);
 * those of weights have the weights' types, dgate asks for a gate.
 */
typedef struct {
  int32_t rows, width;
  int32_t type, w_type, post_type, gate_type;
  int32_t post_norm;
  int32_t group;
  float eps;
  float alpha;
  const void* dy; int64_t ld_dy;
  const void* ds; int64_t ld_ds;
  const void* x;  int64_t ld_x;
  const void* s;  int64_t ld_s;
  const void* weight;
  const void* post_weight;
  const void* gate; int64_t ld_gate;
  void* dx;        int64_t ld_dx;
  void* dresidual; int64_t ld_dresidual;
  void* dweight;
  void* dpost_weight;
  void* dgate;     int64_t ld_dgate;
  void* workspace; int64_t workspace_bytes;
} asd_block_rmsnorm_backward_args;
asd_status asd_block_rmsnorm_backward_workspace(asd_ops* ops, const asd_block_rmsnorm_backward_args* args, int64_t* bytes);
asd_status asd_block_rmsnorm_backward(asd_ops* ops, const asd_block_rmsnorm_backward_args* args, void* cuda_stream);

/*
 * A step of AdamW over `count` tensors (any number of them, of any size):
 *   g = grad grad_scale,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in fp32 (an eps between 0 and 2^-126 is 2^-126), with t the number of steps after this one.  p is the master value where there is one, which is then rounded to
 * the parameter; otherwise the parameter itself, rounded to its type.
 * bits 32: m and v are fp32.  bits 8: m int8 and v uint8 with two scales (M, R) to each 256 neighbouring elements of a
 * tensor, all zero at first:
 *   m = M (q / 127) |q / 127|,   M = max |m|,           q rounded to nearest
 *   v = (R (q / 255)^2)^2,       R = max sqrt(v),       q rounded to nearest, and 1 at least where v > 0
 * a scale below 2^-100 is 0, with q = 0; a NaN or an infinity among a block's moments makes its scale NaN and its q 0.  The
 * step itself is taken with the moments before they are rounded.  Rounded to the nearest, a q follows no decay that is smaller than
 * half a step, (1 - beta1) q < 1 or (1 - beta2) q < 2: with a beta2 of 0.999 sqrt(v) grows beside its true value over the steps, by
 * 4 % in 1000 and a third in 10000 where a block's gradients are of one size.
 * bits 8 | ASD_ADAMW_UNBIASED: the same codes, with q rounded up with the probability of its fraction, or down, so that its mean follows.
 * Whether it is comes from the number of the step and the element's place in its tensor: the same in every run.
 * step: two words on the device, the number of steps taken and one that the library uses (0 at first, and between calls); the
 * call moves the first on by one, so that a captured call may be replayed.  lr_device (in place of lr), grad_scale (NULL: 1)
 * and skip (nonzero: nothing is written and the step is not counted; NULL: never) are read on the device.  No two tensors
 * and no two calls in flight may share memory or `step` (a param that stands twice in the list is refused).
 */
enum { ASD_ADAMW_UNBIASED = 256 };
typedef struct {
  int64_t n;
  int32_t type, grad_type; /* asd_type */
  void* param;             /* of `type` */
  const void* grad;        /* of `grad_type` */
  float* master;           /* or NULL */
  void* m;
  void* v;
  float* scales;           /* bits 8: [(n + 255) / 256][2], on 8 bytes */
} asd_adamw_tensor;
typedef struct {
  int32_t count, bits;
  const asd_adamw_tensor* tensors; /* host */
  double lr, beta1, beta2, eps, weight_decay; /* lr, eps, weight_decay >= 0, 0 <= beta < 1 */
  const float* lr_device;
  const float* grad_scale;
  const float* skip;
  int64_t* step;
} asd_adamw_args;
asd_status asd_adamw(asd_ops* ops, const asd_adamw_args* args, void* cuda_stream);

/* The moments that 8-bit codes stand for, m_out and v_out [n] of `type` (fp16 does not hold the v of small gradients). */
typedef struct {
  int64_t n;
  const void* m;
  const void* v;
  const float* scales;
  int32_t type, reserved;
  void* m_out;
  void* v_out;
} asd_adamw_moments_args;
asd_status asd_adamw_moments(asd_ops* ops, const asd_adamw_moments_args* args, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* ASD_OPS_H */
