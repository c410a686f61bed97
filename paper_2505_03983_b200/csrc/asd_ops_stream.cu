// Matrix products of few rows: y[i, j] = sum_k x[i, k] w[j, k] for up to 32 rows i.
//
// The time is that of reading w once, so the weights go from memory straight into the registers of the warps that multiply
// them, without shared memory, barriers or tensor memory in between.  A warp owns 16 rows of w (GATE: 8 of the gate and the
// same 8 of the value) and a share of k; they are the 16-row operand of mma.sync, the rows of x the narrow one.  The order
// of k inside a sum is free as long as both operands have the same, so a lane takes 16 consecutive bytes of a row of w and
// of a row of x and feeds them to two MMAs as they are: lane (g, t) holds rows g and g + 8 of w and row g of x, bytes
// 16 t ... of each 64.  Each warp keeps 8 to 16 such loads in flight.  The eight warps of a block share 16 to 128 rows of w
// and split k between them; their partial sums meet in shared memory in a fixed order.
#include <algorithm>

#include "asd_ops_tc.cuh"

namespace asd {
namespace {

constexpr int kStreamWarps = 8;
constexpr int kStreamUnroll = 4;  // loads of a row of w that are issued together

struct StreamArgs {
  const uint8_t *w0, *w1, *x;  // GATE: w0 the gate's rows, w1 the value's; otherwise w1 = w0
  int64_t ld_w, ld_x;          // bytes
  int rows, n, k_bytes;        // rows of x, rows of w, bytes of a row's elements
  int split;                   // warps that share a k: 1, 2, 4, 8
  int early;                   // w may be read before the previous kernel has ended
  int out_type, gelu;
  void* c;
  int64_t ldc;
  uint8_t* gu;
  int gu_cols;
  const float* scale_a;
  const float* scale_b;
  const float* bias;
};

// Weights are read once: past L1, which is left to x.
__device__ __forceinline__ uint4 load_once(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::128B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// The last bytes of a row: what lies beyond it counts as zero.
__device__ __forceinline__ uint4 load_part(const uint8_t* p, int bytes) {
  uint32_t w[4] = {0, 0, 0, 0};
  for (int i = 0; i < min(bytes, 16); ++i) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
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

// NT: groups of 8 rows of x.
template <int KIND, int NT, int EPI>
__global__ void __launch_bounds__(32 * kStreamWarps, 2) stream_kernel(const StreamArgs a) {
  constexpr int FR = EPI == OPS_GATE ? 8 : 16;  // rows of w, or columns of h, of a warp
  constexpr int U = kStreamUnroll;
  __shared__ uint32_t part[kStreamWarps][NT * 8][17];  // a warp's sums: [row of x][row of w]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int groups = kStreamWarps / a.split;  // of FR rows, in this block
  const int f0 = (blockIdx.x * groups + warp / a.split) * FR;
  const int share = warp % a.split;
  const uint8_t* p0 = a.w0 + (int64_t)min(f0 + g, a.n - 1) * a.ld_w + 16 * t;
  const uint8_t* p1 = a.w1 + (int64_t)min(EPI == OPS_GATE ? f0 + g : f0 + 8 + g, a.n - 1) * a.ld_w + 16 * t;
  const int whole = a.k_bytes / 64;  // steps of 64 bytes; a ragged rest is the last share's
  const int per = (whole + a.split - 1) / a.split;
  const int s0 = min(share * per, whole), s1 = min(s0 + per, whole);

  uint32_t acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0u;
  uint4 c0[U], c1[U];
  auto fetch = [&](int s, uint4(&v0)[U], uint4(&v1)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < s1) {
        v0[u] = load_once(p0 + (int64_t)(s + u) * 64);
        v1[u] = load_once(p1 + (int64_t)(s + u) * 64);
      }
  };
  auto multiply = [&](const uint4& v0, const uint4& v1, const uint4& b, uint32_t(&c)[4]) {
    mma_16x8<KIND>(c, v0.x, v1.x, v0.y, v1.y, b.x, b.y);
    mma_16x8<KIND>(c, v0.z, v1.z, v0.w, v1.w, b.z, b.w);
  };

  if (!a.early) grid_dependency_wait();
  fetch(s0, c0, c1);
  if (a.early) grid_dependency_wait();
  grid_launch_dependents();

  const uint8_t* px[NT];
  bool have[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    have[i] = g + 8 * i < a.rows;
    px[i] = a.x + (int64_t)(have[i] ? g + 8 * i : 0) * a.ld_x + 16 * t;
  }
  for (int s = s0; s < s1; s += U) {
    uint4 n0[U], n1[U];
    fetch(s + U, n0, n1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u < s1) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          uint4 b = make_uint4(0u, 0u, 0u, 0u);
          if (have[i]) b = *reinterpret_cast<const uint4*>(px[i] + (int64_t)(s + u) * 64);
          multiply(c0[u], c1[u], b, acc[i]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      c0[u] = n0[u];
      c1[u] = n1[u];
    }
  }
  if (share == a.split - 1 && a.k_bytes % 64) {
    const int left = a.k_bytes - whole * 64 - 16 * t;
    const uint4 v0 = load_part(p0 + (int64_t)whole * 64, left), v1 = load_part(p1 + (int64_t)whole * 64, left);
#pragma unroll
    for (int i = 0; i < NT; ++i) multiply(v0, v1, load_part(px[i] + (int64_t)whole * 64, have[i] ? left : 0), acc[i]);
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    part[warp][8 * i + 2 * t][g] = acc[i][0];
    part[warp][8 * i + 2 * t + 1][g] = acc[i][1];
    part[warp][8 * i + 2 * t][g + 8] = acc[i][2];
    part[warp][8 * i + 2 * t + 1][g + 8] = acc[i][3];
  }
  __syncthreads();

  const int cols = groups * FR;
  for (int e = threadIdx.x; e < cols * a.rows; e += 32 * kStreamWarps) {
    const int f = e % cols, row = e / cols, col = blockIdx.x * cols + f;
    if (col >= a.n) continue;
    const int w0 = (f / FR) * a.split, r = f % FR;
    if constexpr (KIND == KIND_I8) {
      int v = 0;
      for (int s = 0; s < a.split; ++s) v += (int)part[w0 + s][row][r];
      const float y = fmaf((float)v * a.scale_a[row], a.scale_b[col], a.bias ? a.bias[col] : 0.f);
      if (a.out_type == ASD_TYPE_F32)
        reinterpret_cast<float*>(a.c)[row * a.ldc + col] = y;
      else
        reinterpret_cast<uint16_t*>(a.c)[row * a.ldc + col] = round16(y, a.out_type == ASD_TYPE_F16);
    } else {
      float v = 0.f, u = 0.f;
      for (int s = 0; s < a.split; ++s) {
        v += __uint_as_float(part[w0 + s][row][r]);
        if (EPI == OPS_GATE) u += __uint_as_float(part[w0 + s][row][r + 8]);
      }
      if (EPI == OPS_GATE) {
        if (a.gu) {
          uint8_t* b = a.gu + gu_block_offset(row, col, a.gu_cols);
          gu_put(b, row & 31, col & 31, v);
          gu_put(b + kGuHalf, row & 31, col & 31, u);
        }
        v = gate_value(v, a.gelu != 0) * u;
      }
      reinterpret_cast<uint16_t*>(a.c)[row * a.ldc + col] = round16(v, KIND == KIND_F16);
    }
  }
}

template <int KIND, int EPI>
void launch_nt(const StreamArgs& a, dim3 grid, cudaStream_t st) {
  const dim3 block(32 * kStreamWarps);
  if (a.rows <= 8)
    ops_launch(stream_kernel<KIND, 1, EPI>, grid, block, 0, st, 1, a);
  else if (a.rows <= 16)
    ops_launch(stream_kernel<KIND, 2, EPI>, grid, block, 0, st, 1, a);
  else
    ops_launch(stream_kernel<KIND, 4, EPI>, grid, block, 0, st, 1, a);
}

}  // namespace

bool use_stream(const OpsGemm& q) {
  return (q.epi == OPS_GATE || q.epi == OPS_I8 || (q.epi == OPS_STORE && q.parts == 1 && q.groups == 1)) && q.m <= kStreamMaxRows &&
         !q.a[0].mn && !q.b[0].mn;
}

asd_status ops_gemm_stream(const asd_ops* o, const OpsGemm& q, bool early, cudaStream_t st) {
  StreamArgs a{};
  const int es = q.epi == OPS_I8 ? 1 : 2;
  a.w0 = (const uint8_t*)q.b[0].mat.p;
  a.w1 = (const uint8_t*)q.b[q.epi == OPS_GATE ? 1 : 0].mat.p;
  a.x = (const uint8_t*)q.a[0].mat.p;
  a.ld_w = q.b[0].mat.ld * es, a.ld_x = q.a[0].mat.ld * es;
  a.rows = (int)q.m, a.n = (int)q.n, a.k_bytes = (int)(q.k[0] * es);
  a.early = early;
  a.out_type = q.type, a.gelu = q.act == ASD_ACT_GELU;
  a.c = q.c[0], a.ldc = q.ldc;
  a.gu = q.gu, a.gu_cols = (int)((q.n + 31) / 32);
  a.scale_a = q.scale_a, a.scale_b = q.scale_b, a.bias = q.bias;
  // as few warps to a k as give two blocks to every SM, and at least 256 bytes of k to a warp
  const int fr = q.epi == OPS_GATE ? 8 : 16;
  const int64_t units = (q.n + fr - 1) / fr;
  a.split = 1;
  while (a.split < kStreamWarps && units * a.split < 2 * (int64_t)kStreamWarps * o->num_sms && a.k_bytes / (2 * a.split) >= 256) a.split *= 2;
  const int groups = kStreamWarps / a.split;
  const dim3 grid((unsigned)((units + groups - 1) / groups));
  if (q.epi == OPS_I8)
    launch_nt<KIND_I8, OPS_I8>(a, grid, st);
  else if (q.epi == OPS_GATE)
    q.type == ASD_TYPE_F16 ? launch_nt<KIND_F16, OPS_GATE>(a, grid, st) : launch_nt<KIND_BF16, OPS_GATE>(a, grid, st);
  else
    q.type == ASD_TYPE_F16 ? launch_nt<KIND_F16, OPS_STORE>(a, grid, st) : launch_nt<KIND_BF16, OPS_STORE>(a, grid, st);
  return ops_launched("matrix product of few rows");
}

}  // namespace asd
