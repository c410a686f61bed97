// Internal declarations shared by the translation units of the operators (include/asd_ops.h): the handle, the
// message of a failed call, and the launchers of the kernels.  Nothing here crosses the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "asd_ops.h"

struct asd_ops {
  int device;
  int num_sms;
  int* err;  // device word: 0, or ASD_ERR_TIMEOUT
};

namespace asd {

constexpr int kOpsMaxDim = 1 << 24;  // rows' lengths; keeps a row's products of sizes inside 32 bits
constexpr int kOpsMaxK8 = 131071;    // 2^31 / 128^2: the longest sum of 8-bit products that int32 holds

asd_status ops_fail(asd_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void ops_note_launch(cudaError_t e);        // what a launch returned, kept until ops_launched
asd_status ops_launched(const char* what);  // OK, or CUDA with the first error of this thread's launches since the last call
int ops_type_size(int type);                // bytes of an asd_type, 0 if it is none

// Launch with programmatic stream serialization: the kernel may start while its predecessor in the stream ends.  Every kernel of the
// operators waits for it (griddepcontrol.wait) before it touches global memory, and lets its own successor start
// (griddepcontrol.launch_dependents) only after that wait.  The split and the stream kernel with `early` read their weights
// before the wait: that the kernel before them was let in only after its own wait is what makes it safe, for then everything
// further back has ended, and the kernel before them is of the same call and does not write the weights.
template <typename... P, typename... A>
inline void ops_launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, int cluster, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  ops_note_launch(cudaLaunchKernelEx(&cfg, kernel, P(args)...));
}

// A matrix operand: `rows` rows of `cols` contiguous elements, `ld` elements apart.
struct Mat {
  const void* p;
  int64_t rows, cols, ld;
  int es;  // bytes of an element
};
inline bool mat_aligned(const Mat& m) { return ((uintptr_t)m.p & 15) == 0 && (m.ld * m.es) % 16 == 0; }

// ---- asd_ops_rows.cu: one row at a time -------------------------------------------------------------
asd_status ops_rows_prepare();
void launch_rmsnorm(const asd_ops* o, const asd_rmsnorm_args* a, cudaStream_t st);
int64_t rmsnorm_backward_bytes(const asd_ops* o, const asd_rmsnorm_backward_args* a);
void launch_rmsnorm_backward(const asd_ops* o, const asd_rmsnorm_backward_args* a, cudaStream_t st);
void launch_quantize(const asd_ops* o, const asd_quantize_args* a, cudaStream_t st);
// Operands that are copied to rows of a multiple of 16 bytes before a product reads them, in one launch.
struct Packs {
  int n = 0;
  Mat src[4];
  void* dst[4];
  int64_t ld[4];  // elements
};
void launch_packs(const asd_ops* o, const Packs& packs, cudaStream_t st);

// ---- asd_ops_gemm.cu: matrix products -----------------------------------------------------------------
// C[m, n] = sum_k A(m, k) B(n, k).  An operand is read either as a row-major matrix [its m or n, k] or, `mn` true, as
// the transpose of a row-major matrix [k, its m or n].
struct Operand {
  Mat mat;
  bool mn;
};
enum OpsEpi { OPS_STORE = 0, OPS_GATE = 1, OPS_GATE_GRAD = 2, OPS_I8 = 3 };
struct OpsGemm {
  int epi;
  int type;    // asd_type of the 16-bit operands and outputs (OPS_I8: of the output)
  int act;     // OPS_GATE
  int64_t m, n, k[2];
  int parts;   // OPS_STORE: 1, or 2 sums over k one after the other (k[0] of a[0], b[0], then k[1] of a[1], b[1])
  Operand a[2], b[2];  // OPS_GATE: b[0] the gate's weights, b[1] the value's
  void* c[2];          // outputs; OPS_GATE: c[0] = h; OPS_GATE_GRAD: c[0] = dg, c[1] = du
  int64_t ldc;
  int slices;          // ops_gemm_list: > 1: the sum in that many slices, through `part` (part_bytes)
  float* part;
  uint8_t* kept;       // OPS_GATE: where the gate's two factors are kept, or NULL; OPS_GATE_GRAD: where they were
  const float* scale_a;  // OPS_I8
  const float* scale_b;
  const float* bias;
};
int64_t gated_kept_bytes(int64_t rows, int64_t hidden);
// `early`: the kernel before this one in the stream belongs to the same call, which does not write b.
asd_status ops_gemm(const asd_ops* o, const OpsGemm& g, bool early, cudaStream_t st);
// Up to four independent OPS_STORE products of one type.
constexpr int kMostProducts = 4;
asd_status ops_gemm_list(const asd_ops* o, const OpsGemm* g, int n, cudaStream_t st);
// Slices of the sum that are worth their partial sums (1: none), and the bytes of these.
int sum_slices(const asd_ops* o, int64_t m, int64_t n, int64_t k);
int64_t part_bytes(int64_t m, int64_t n, int slices);
asd_status ops_gemm_prepare();  // per device: opt-in to large shared memory

// ---- asd_ops_stream.cu: matrix products of few rows ---------------------------------------------------
constexpr int kStreamMaxRows = 8;
asd_status ops_stream_prepare();
bool use_stream(const OpsGemm& g);
asd_status ops_gemm_stream(const asd_ops* o, const OpsGemm& g, bool early, cudaStream_t st);

// ---- asd_ops_split.cu: matrix products with too few tiles ----------------------------------------------
struct SplitPlan {
  int nb, split, stages;  // rows of a CTA, CTAs that share a sum, stages of its operands
  double clocks;          // estimate
};
constexpr int64_t kSplitMostRows = 16384;  // beyond, tiles of whole waves are enough
SplitPlan plan_split(const asd_ops* o, const OpsGemm& g, bool early);
asd_status ops_split_prepare();
asd_status ops_gemm_split(const asd_ops* o, const OpsGemm& g, const SplitPlan& p, bool early, cudaStream_t st);

// A tensor map of an operand: boxes of 128 bytes by `tile_rows` rows, or of 64 by 64 elements where it is read across k.
bool encode_operand(CUtensorMap* out, const Operand& x, int type, bool i8, int tile_rows);

}  // namespace asd
