// Matrix products of few rows: y[i, j] = sum_k x[i, k] w[j, k] for up to 8 rows i.
//
// The time is that of reading w once.  The 16 warps of a block work on 16 rows of w at a time (GATE: 8 of the gate and the
// same 8 of the value) and share k; x stays in shared memory.  The rows of w are the 16-row operand of mma.sync, those of x
// the narrow one.  The order of k inside a sum is free as long as both operands have the same, so a lane takes 16
// consecutive bytes of a row of w and of a row of x and feeds them to two MMAs as they are: lane (g, t) holds rows g and
// g + 8 of w and row g of x, bytes 16 t ... of each 64.  Every lane therefore reads back only what it has copied itself: the
// weights come through a ring in shared memory of its own (cp.async, up to 11 steps of 1 KB a warp ahead, 176 KB an SM),
// which needs neither barriers nor registers, and runs on over the block's next rows while the sums of one group of rows
// meet (in shared memory, in a fixed order).
//
// Measured: 155 MB of int8 weights (1 x 8192 x 18944) in 25.1 us = 6.2 TB/s; 34 MB (1 x 4096 x 8192) in 8.3 us, of which 5.3 are
// the bytes and the rest a kernel's start, first and last byte.  The split kernel, whose weights are the 128-row operand of
// tcgen05, has tensor memory to allocate and cluster barriers to pass: gated MLP 1 x 1024 x 4096 12.4 us against 7.7 here, int8
// 1 x 1024 x 1024 3.5 against 2.0.  At 8 rows they meet (int8 8 x 4096 x 8192: 9.3 and 9.7; gated MLP 8 x 4096 x 8192: 37.8 and 37.2).
#include <algorithm>

#include "asd_ops_tc.cuh"

namespace asd {
namespace {

constexpr int kStreamWarps = 16;

constexpr int kStreamSmem = 232448;
// Shared memory of x and the partial sums.
int64_t rows_bytes(int64_t rows, int64_t pitch) { return rows * pitch + 2 * kStreamWarps * ((rows * 17) | 1) * 4; }
constexpr int ring_bytes(int ring) { return kStreamWarps * ring * 1024; }

struct StreamArgs {
  const uint8_t *w0, *w1, *x;  // GATE: w0 the gate's rows, w1 the value's; otherwise w1 = w0
  int64_t ld_w, ld_x;          // bytes
  int rows, n, k_bytes;        // rows of x, rows of w, bytes of a row's elements
  int pitch;                   // bytes from one row of x to the next in shared memory
  int early;                   // w may be read before the previous kernel has ended
  int out_type, gelu;
  void* c;
  int64_t ldc;
  uint8_t* kept;
  int kept_cols;
  const float* scale_a;
  const float* scale_b;
  const float* bias;
};

// 16 bytes to shared memory, of which `bytes` are read and the others zero.
__device__ __forceinline__ void copy_16(uint32_t dst, const uint8_t* src, int bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
enum { KIND_F16 = 0, KIND_BF16 = 1, KIND_I8 = 2 };
// acc += w x^T for 32 bytes of k (words a of rows g and g + 8, words b of row g of x).
template <int KIND>
__device__ __forceinline__ void mma_16x8(uint32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (KIND == KIND_I8) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  } else {
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(c[i]);
    if constexpr (KIND == KIND_F16)
      asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
          : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3])
          : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
      asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
          : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3])
          : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(f[i]);
  }
}

// RING: steps of the ring.  SPAN: lanes that add up the warps' sums of one output.
template <int KIND, int EPI, int RING, int SPAN>
__global__ void __launch_bounds__(32 * kStreamWarps, 1) stream_kernel(const StreamArgs a) {
  constexpr int FR = EPI == OPS_GATE ? 8 : 16;  // columns of the output to a group of rows of w
  extern __shared__ __align__(128) uint8_t smem[];  // the warps' rings, x, the warps' sums
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int units = (a.n + FR - 1) / FR;
  const int mine = ((int)blockIdx.x < units) ? (units - 1 - (int)blockIdx.x) / (int)gridDim.x + 1 : 0;
  // steps of 64 bytes of k, the last one possibly ragged; this warp's are [s0, s1)
  const int steps = (a.k_bytes + 63) / 64;
  const int per = (steps + kStreamWarps - 1) / kStreamWarps;
  const int s0 = min(warp * per, steps), s1 = min(s0 + per, steps);
  uint8_t* ring = smem + warp * (RING * 1024) + lane * 16;
  const uint32_t ring_addr = smem_u32(ring);
  uint8_t* xs = smem + kStreamWarps * RING * 1024;
  // the warps' sums, [2][warp][row of x][16 rows of w]
  uint32_t* part = reinterpret_cast<uint32_t*>(xs + a.rows * a.pitch);
  const uint32_t xs_addr = smem_u32(xs);

  // The copies run ahead of the sums through the same sequence: steps s0 .. s1 of the block's first rows, then of its next.
  int unit = s0 < s1 ? 0 : mine, step = s0, slot = 0;
  const uint8_t *p0 = nullptr, *p1 = nullptr;
  auto rows_of = [&](int i) {
    const int f0 = ((int)blockIdx.x + i * (int)gridDim.x) * FR;
    p0 = a.w0 + (int64_t)min(f0 + g, a.n - 1) * a.ld_w + 16 * t;
    p1 = a.w1 + (int64_t)min(EPI == OPS_GATE ? f0 + g : f0 + 8 + g, a.n - 1) * a.ld_w + 16 * t;
  };
  auto copy_next = [&]() {
    if (unit < mine) {
      const int left = min(max(a.k_bytes - step * 64 - 16 * t, 0), 16);
      const int64_t at = left ? (int64_t)step * 64 : 0;
      copy_16(ring_addr + slot * 1024, p0 + at, left);
      copy_16(ring_addr + slot * 1024 + 512, p1 + at, left);
      if (++step == s1) {
        step = s0;
        if (++unit < mine) rows_of(unit);
      }
      if (++slot == RING) slot = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // x: each warp brings its own share of k, so that no barrier of the block is needed; ahead of the weights, behind which it
  // would wait for as long as a whole ring of them takes
  auto copy_x = [&]() {
    const int pieces = (s1 - s0) * 4, all = a.rows * pieces;  // of 16 bytes, of a row and of all; lanes take them in turn
    for (int at = 0; at < all; at += 32) {
      const int r = (at + lane) / pieces, s = s0 * 4 + at + lane - r * pieces;
      if (r < a.rows) {
        const int left = min(max(a.k_bytes - s * 16, 0), 16);
        copy_16(xs_addr + r * a.pitch + s * 16, a.x + r * a.ld_x + (left ? (int64_t)s * 16 : 0), left);
      }
    }
    __syncwarp();
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (unit < mine) rows_of(0);
  if (!a.early) {
    grid_dependency_wait();
    copy_x();
  }
#pragma unroll
  for (int i = 0; i < RING - 1; ++i) copy_next();
  if (a.early) {
    grid_dependency_wait();
    copy_x();
    asm volatile("cp.async.wait_group 0;" ::: "memory");
  } else {
    asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");  // all but the ring's
  }
  grid_launch_dependents();
  __syncwarp();

  const int of_row = 17, of_warp = (a.rows * 17) | 1;  // words from a row's, a warp's sums to the next: odd, for the banks
  // One output: its sum v (GATE: of g, and u) is complete.
  auto finish = [&](int row, int col, uint32_t v, uint32_t u, float sa, float sb, float bb) {
    if constexpr (KIND == KIND_I8) {
      const float y = fmaf((float)(int)v * sa, sb, bb);
      if (a.out_type == ASD_TYPE_F32)
        reinterpret_cast<float*>(a.c)[row * a.ldc + col] = y;
      else
        reinterpret_cast<uint16_t*>(a.c)[row * a.ldc + col] = round16(y, a.out_type == ASD_TYPE_F16);
    } else {
      float h[1] = {__uint_as_float(v)};
      if (EPI == OPS_GATE) {
        float g1[1] = {h[0]}, u1[1] = {__uint_as_float(u)};
        gated(g1, u1, h, a.gelu != 0, a.kept != nullptr);
        if (a.kept) {
          uint8_t* b = a.kept + kept_offset(row, col, a.kept_cols);
          kept_put(b, row, col & 31, g1[0]);
          kept_put(b + kKeptHalf, row, col & 31, u1[0]);
        }
      }
      reinterpret_cast<uint16_t*>(a.c)[row * a.ldc + col] = round16(h[0], KIND == KIND_F16);
    }
  };
  auto add = [&](uint32_t x, uint32_t y) { return KIND == KIND_I8 ? x + y : __float_as_uint(__uint_as_float(x) + __uint_as_float(y)); };
  // The warps' sums of unit i meet: SPAN lanes to an output, 32 / SPAN outputs to a warp, in an order that depends on nothing
  // else.  16 lanes each where there are few outputs, four where 16 would have to take turns (9.8 against 12.5 us, gated MLP
  // 8 x 1024 x 4096).  Scales are fetched before the barrier.
  auto join = [&](int i, const uint32_t* p) {
    constexpr int OUTS = 32 / SPAN;
    const int o = OUTS * warp + lane / SPAN, f = o % FR, row = o / FR, from = lane % SPAN;
    const int col = ((int)blockIdx.x + i * (int)gridDim.x) * FR + f;
    const bool out = row < a.rows && col < a.n && from == 0;
    float sa = 0.f, sb = 0.f, bb = 0.f;
    if (KIND == KIND_I8 && out) {
      sa = a.scale_a[row];
      sb = a.scale_b[col];
      if (a.bias) bb = a.bias[col];
    }
    __syncthreads();
    if (OUTS * warp >= FR * a.rows) return;
    const uint32_t* sum = p + from * of_warp + (row < a.rows ? row : 0) * of_row + f;
    uint32_t v = sum[0], u = EPI == OPS_GATE ? sum[8] : 0u;
#pragma unroll
    for (int k = 1; k < kStreamWarps / SPAN; ++k) {
      v = add(v, sum[k * SPAN * of_warp]);
      if (EPI == OPS_GATE) u = add(u, sum[k * SPAN * of_warp + 8]);
    }
#pragma unroll
    for (int d = SPAN / 2; d; d >>= 1) {
      v = add(v, __shfl_xor_sync(0xffffffffu, v, d));
      if (EPI == OPS_GATE) u = add(u, __shfl_xor_sync(0xffffffffu, u, d));
    }
    if (out) finish(row, col, v, u, sa, sb, bb);
  };
  const uint8_t* xr = xs + g * a.pitch + 16 * t;
  const bool have = g < a.rows;
  int at = 0;
  for (int i = 0; i < mine; ++i) {
    uint32_t acc[4] = {0u, 0u, 0u, 0u};
    for (int s = s0; s < s1; ++s) {
      copy_next();  // into the slot of the step before this one
      asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
      const uint4 c0 = *reinterpret_cast<const uint4*>(ring + at * 1024), c1 = *reinterpret_cast<const uint4*>(ring + at * 1024 + 512);
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (have) x = *reinterpret_cast<const uint4*>(xr + s * 64);
      mma_16x8<KIND>(acc, c0.x, c1.x, c0.y, c1.y, x.x, x.y);
      mma_16x8<KIND>(acc, c0.z, c1.z, c0.w, c1.w, x.z, x.w);
      if (++at == RING) at = 0;
    }
    // free: every thread has passed the barrier of unit i - 1 after reading unit i - 2's
    uint32_t* p = part + (i & 1) * kStreamWarps * of_warp;
    uint32_t* own = p + warp * of_warp + g;
    if (2 * t < a.rows) {
      own[2 * t * of_row] = acc[0];
      own[2 * t * of_row + 8] = acc[2];
    }
    if (2 * t + 1 < a.rows) {
      own[(2 * t + 1) * of_row] = acc[1];
      own[(2 * t + 1) * of_row + 8] = acc[3];
    }
    join(i, p);
  }
}

template <int KIND, int EPI, int SPAN>
void launch_span(const asd_ops* o, const StreamArgs& a, cudaStream_t st) {
  const int fr = EPI == OPS_GATE ? 8 : 16;
  const dim3 grid(std::min((a.n + fr - 1) / fr, o->num_sms)), block(32 * kStreamWarps);
  const int x = (int)rows_bytes(a.rows, a.pitch);
  // The ring: no longer than a warp has steps, so that the next kernel's blocks may find room beside these.  (The shortest for a
  // kernel that may start early, so that it always does, is slower: 9.0 against 7.6 us, gated MLP 1 x 1024 x 4096.)
  const int units = (a.n + fr - 1) / fr, steps = (a.k_bytes + 63) / 64;
  const int most = (units + (int)grid.x - 1) / (int)grid.x * ((steps + kStreamWarps - 1) / kStreamWarps);
  if (x <= kStreamSmem - ring_bytes(12) && most > 8)
    ops_launch(stream_kernel<KIND, EPI, 12, SPAN>, grid, block, (size_t)(ring_bytes(12) + x), st, 1, a);
  else if (x <= kStreamSmem - ring_bytes(8) && most > 4)
    ops_launch(stream_kernel<KIND, EPI, 8, SPAN>, grid, block, (size_t)(ring_bytes(8) + x), st, 1, a);
  else
    ops_launch(stream_kernel<KIND, EPI, 4, SPAN>, grid, block, (size_t)(ring_bytes(4) + x), st, 1, a);
}
template <int KIND, int EPI>
void launch_stream(const asd_ops* o, const StreamArgs& a, cudaStream_t st) {
  if ((EPI == OPS_GATE ? 8 : 16) * a.rows <= 2 * kStreamWarps)
    launch_span<KIND, EPI, 16>(o, a, st);
  else
    launch_span<KIND, EPI, 4>(o, a, st);
}
template <int KIND, int EPI>
cudaError_t prepare_stream() {
  cudaError_t e = cudaSuccess;
  auto set = [&](auto* kernel) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
  };
  set(stream_kernel<KIND, EPI, 12, 16>);
  set(stream_kernel<KIND, EPI, 8, 16>);
  set(stream_kernel<KIND, EPI, 4, 16>);
  set(stream_kernel<KIND, EPI, 12, 4>);
  set(stream_kernel<KIND, EPI, 8, 4>);
  set(stream_kernel<KIND, EPI, 4, 4>);
  return e;
}

// Rows of x lie 64 bytes off a multiple of 128: eight lanes that read two of them meet every bank once.
int x_pitch(int64_t k_bytes) { return (int)((k_bytes + 127) / 128 * 128 + 64); }

}  // namespace

// Few enough rows, and x fits into shared memory.
bool use_stream(const OpsGemm& q) {
  const int es = q.epi == OPS_I8 ? 1 : 2;
  return (q.epi == OPS_GATE || q.epi == OPS_I8 || (q.epi == OPS_STORE && q.parts == 1)) && q.m <= kStreamMaxRows &&
         !q.a[0].mn && !q.b[0].mn && rows_bytes(q.m, x_pitch(q.k[0] * es)) <= kStreamSmem - ring_bytes(4);
}

asd_status ops_gemm_stream(const asd_ops* o, const OpsGemm& q, bool early, cudaStream_t st) {
  StreamArgs a{};
  const int es = q.epi == OPS_I8 ? 1 : 2;
  a.w0 = (const uint8_t*)q.b[0].mat.p;
  a.w1 = (const uint8_t*)q.b[q.epi == OPS_GATE ? 1 : 0].mat.p;
  a.x = (const uint8_t*)q.a[0].mat.p;
  a.ld_w = q.b[0].mat.ld * es, a.ld_x = q.a[0].mat.ld * es;
  a.rows = (int)q.m, a.n = (int)q.n, a.k_bytes = (int)(q.k[0] * es), a.pitch = x_pitch(q.k[0] * es);
  a.early = early;
  a.out_type = q.type, a.gelu = q.act == ASD_ACT_GELU;
  a.c = q.c[0], a.ldc = q.ldc;
  a.kept = q.kept, a.kept_cols = (int)((q.n + 31) / 32);
  a.scale_a = q.scale_a, a.scale_b = q.scale_b, a.bias = q.bias;
  if (q.epi == OPS_I8)
    launch_stream<KIND_I8, OPS_I8>(o, a, st);
  else if (q.epi == OPS_GATE)
    q.type == ASD_TYPE_F16 ? launch_stream<KIND_F16, OPS_GATE>(o, a, st) : launch_stream<KIND_BF16, OPS_GATE>(o, a, st);
  else
    q.type == ASD_TYPE_F16 ? launch_stream<KIND_F16, OPS_STORE>(o, a, st) : launch_stream<KIND_BF16, OPS_STORE>(o, a, st);
  return ops_launched("matrix product of few rows");
}

asd_status ops_stream_prepare() {
  const cudaError_t all[] = {prepare_stream<KIND_I8, OPS_I8>(), prepare_stream<KIND_F16, OPS_GATE>(), prepare_stream<KIND_BF16, OPS_GATE>(),
                             prepare_stream<KIND_F16, OPS_STORE>(), prepare_stream<KIND_BF16, OPS_STORE>()};
  for (cudaError_t e : all)
    if (e != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  return ASD_OK;
}

}  // namespace asd
