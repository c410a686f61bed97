// The norms between two blocks, fused with the gate and the scale of the residual branch:
//   n = x / sqrt(mean(x^2) + eps)  (or x),  s = r + alpha gate w_post n,  y = s / sqrt(mean(s^2) + eps) w
// and its gradients.  A row of the gate belongs to a run of `group` rows.  All kernels are bound by memory: a row of x and r is
// read once, s and y are written once (16 / 32 bits, or y in 8 with a scale).
//
// Backward, with z = s rho, rho = 1 / sqrt(mean(s^2) + eps) and rho_x that of x:
//   dS = ds + rho dy w - z rho mean(dy w z)                                    the residual's gradient
//   dx = rho_x (c dS - n mean(c dS n)),  c = alpha gate w_post                 (without the norm: c dS)
//   dw = sum dy z;  with U_g = sum over the rows of gate row g of dS n:  dgate_g = alpha w_post U_g,  dw_post = alpha sum_g gate_g U_g
// All means of a row are linear in six sums over it (s^2, x^2, dy w s, and c x times ds, dy w and s), which are therefore taken in
// one pass and one barrier (narrow rows, whose sums need none, take that of c n dS itself), and both gradients of the gate's product come from the one sum U.
#include <algorithm>

#include "asd_ops_rows.cuh"

namespace asd {
namespace {

// ---- forward ---------------------------------------------------------------------------------------------

struct BlockArgs {
  int rows, width, group, post;
  int ring_gate;  // a row of the gate to every row, brought with it
  int* err;
  int w_f32, p_f32, g_f32;
  float eps, alpha;
  const void *x, *r, *w, *wp, *gate;
  void *s, *y;
  float* scale;
  int64_t ld_x, ld_r, ld_g, ld_s, ld_y;
};

template <typename T>
__device__ __forceinline__ const void* gate_row(const void* gate, int g_f32, int64_t row, int64_t ld) {
  if (!gate) return nullptr;
  return reinterpret_cast<const uint8_t*>(gate) + row * ld * (g_f32 ? 4 : (int)sizeof(T));
}
__device__ __forceinline__ float rho_of(float sq, int width, float eps) { return 1.f / sqrtf(sq / (float)width + eps); }

// How the kernels for rows of 257 to 16384 (backward: 8192) elements hold a row: TPR threads, 16 elements each and always the same
// columns, so that weights and sums over rows stay in registers.  A block walks down a run of neighbouring rows, which come through
// shared memory, `stages` of them at a time.  Rows in 16-byte pieces (VEC = 8) are brought by bulk copies that one thread issues,
// others are staged by all of the block's.  8192 x 4096 in bf16, forward and backward: one row to a block without a ring 106 us;
// eight elements to a thread, where the fixed work of a row doubles, 130 us backward; 16 elements and copies by every thread for
// itself, with some 300 instructions a row and warp for addresses, sums and copies, 54 and 90; now 47 and 70 (4.6 and 5.1 TB/s of
// DRAM, a part of the outputs being still in L2; half of the issue slots), and 11 more for the join of the sums over rows.
constexpr int kWalkPer = 16, kWalkVecs = kWalkPer / 8, kMostStages = 4;
constexpr int kMostWalkWidth = 1024 * kWalkPer;
constexpr long long kWaitClocks = 400000000ll;  // some 0.2 s

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool bar_passed(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok;
}
// The parts of a row that lie in the ring: PARTS of the operands' type, then possibly the row's gate, in a type of its own.
template <typename T, int VEC, int TPR, int PARTS>
struct Ring {
  uint8_t* mem;
  uint64_t* bars;  // one a stage
  int width, pitch, stages, t;
  int stage_bytes;
  const T* base[PARTS];  // NULL: not there
  int64_t ld[PARTS];
  const uint8_t* gate;   // NULL: not in the ring; otherwise a row of `gate_bytes` to every row of the operands
  int64_t ld_gate;       // bytes
  int gate_bytes;
  int* err;
  volatile int* dead;

  __device__ __forceinline__ int column(int v, int i) const { return VEC == 8 ? (v * TPR + t) * 8 + i : (v * 8 + i) * TPR + t; }
  __device__ __forceinline__ bool any(int v) const { return column(v, 0) < width; }
  __device__ __forceinline__ uint8_t* row(int stage, int part) const { return mem + stage * stage_bytes + part * pitch; }
  // The threads' elements beyond a row's end, and a part that is not there, are read as zeros that are written here once: a
  // condition at each read of a row costs more than the read.
  __device__ __forceinline__ void init() const {
    if (VEC == 8) {
      if (t == 0) {
        for (int i = 0; i < stages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_at(bars + i)) : "memory");
        *dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      }
      for (int i = 0; i < stages; ++i) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
          for (int at = (base[part] ? width * (int)sizeof(T) : 0) + 16 * t; at < pitch; at += 16 * TPR)
            *reinterpret_cast<uint4*>(row(i, part) + at) = make_uint4(0u, 0u, 0u, 0u);
      }
    } else {
      for (int at = 16 * t; at < stages * PARTS * pitch; at += 16 * TPR) *reinterpret_cast<uint4*>(mem + at) = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
  }
  __device__ __forceinline__ void copy(const void* src, uint8_t* dst, int bytes, uint32_t bar) const {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_at(dst)), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
  }
  // Starts the copies of row r.  Every thread has to have read what the stage held.
  __device__ __forceinline__ void fetch(int64_t r, int end, int stage) const {
    if constexpr (VEC == 8) {
      if (t != 0 || r >= end) return;
      const uint32_t bar = smem_at(bars + stage);
      const int bytes = width * (int)sizeof(T);
      int all = gate ? gate_bytes : 0;
#pragma unroll
      for (int part = 0; part < PARTS; ++part) all += base[part] ? bytes : 0;
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(all) : "memory");
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        if (base[part]) copy(base[part] + r * ld[part], row(stage, part), bytes, bar);
      if (gate) copy(gate + r * ld_gate, row(stage, PARTS), gate_bytes, bar);
    } else {
      if (r < end) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
          if (base[part]) {
            const T* p = base[part] + r * ld[part];
            stage_row(row(stage, part), p, width * (int)sizeof(T), t, TPR, r == 0);
            // the piece behind it, which a row that starts further off 16 bytes has reached
            if (t == part) *reinterpret_cast<uint4*>(row(stage, part) + (((int)((uintptr_t)p & 15) + width * (int)sizeof(T) + 15) & ~15)) = make_uint4(0u, 0u, 0u, 0u);
          }
      }
      commit_copies();
    }
  }
  // Row r may be read from its stage, which it is the (2 k + parity)-th to use.
  __device__ __forceinline__ void arrive(int64_t r, int end, int stage, uint32_t parity) const {
    if constexpr (VEC == 8) {
      const uint32_t bar = smem_at(bars + stage);
      if (bar_passed(bar, parity)) return;
      const long long t0 = clock64(), limit = *dead ? 2000ll : kWaitClocks;
      while (!bar_passed(bar, parity)) {
        if (clock64() - t0 > limit) {
          *dead = 1;
          atomicExch(err, (int)ASD_ERR_TIMEOUT);
          return;
        }
      }
    } else {
      if (stages == 1) {
        __syncthreads();  // the row before is no longer read
        fetch(r, end, 0);
      }
      wait_copies<0>();
      __syncthreads();
      if (stages > 1) fetch(r + 1, end, stage ^ 1);  // two stages: the other one's row is done with
    }
  }
  // After a barrier that all threads have come to since they read row r - 1.
  __device__ __forceinline__ void refill(int64_t r, int first, int end, int stage) const {
    if (VEC == 8 && stages > 1 && r > first) fetch(r - 1 + stages, end, stage == 0 ? stages - 1 : stage - 1);
  }
  // After row r, where the ring has room for one row only.
  __device__ __forceinline__ void turn(int64_t r, int end) const {
    if (VEC == 8 && stages == 1) {
      __syncthreads();
      fetch(r + 1, end, 0);
    }
  }
  __device__ __forceinline__ void end() const {
    if (VEC == 8 && *dead) {  // a wait ran out: time for the copies in flight to land
      const long long t0 = clock64();
      while (clock64() - t0 < 2000000ll) {
      }
    }
  }
  // Vector v of a part; elements beyond the row's end are 0.
  __device__ __forceinline__ void read(int64_t r, int stage, int part, int v, float2 (&f)[4]) const {
    if constexpr (VEC == 8) {
      constexpr int PV = (int)sizeof(T) / 2;  // 16-byte pieces of eight elements
      uint32_t e[4 * PV];
      const uint4* p = reinterpret_cast<const uint4*>(row(stage, part)) + (v * TPR + t) * PV;
#pragma unroll
      for (int k = 0; k < PV; ++k) reinterpret_cast<uint4*>(e)[k] = p[k];
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = unpack<T>(e, i);
    } else {
      const T* p = staged<T>(row(stage, part), base[part] + r * ld[part]);  // the zeros behind the row's end are part of the buffer
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = make_float2(to_f<T>(p[column(v, 2 * i)]), to_f<T>(p[column(v, 2 * i + 1)]));
    }
  }
  // The columns of vector v of a weight (NULL: 1); 0 beyond the row's end.
  __device__ __forceinline__ void weight(const void* p, int f32, int v, float2 (&f)[4]) const {
    float e[8];
    if (VEC == 8 && any(v)) {
      load_weight<8, T>(p, f32, column(v, 0), e);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float one[1] = {0.f};
        if (column(v, i) < width) load_weight<1, T>(p, f32, column(v, i), one);
        e[i] = one[0];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(e[2 * i], e[2 * i + 1]);
  }
  __device__ __forceinline__ void store(T* to, int v, const float2 (&f)[4]) const {
    if constexpr (VEC == 8) {
      const float e[8] = {f[0].x, f[0].y, f[1].x, f[1].y, f[2].x, f[2].y, f[3].x, f[3].y};
      if (any(v)) store_vec<8, T>(to + column(v, 0), e);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (column(v, 2 * i) < width) to[column(v, 2 * i)] = from_f<T>(f[i].x);
        if (column(v, 2 * i + 1) < width) to[column(v, 2 * i + 1)] = from_f<T>(f[i].y);
      }
    }
  }
};
// Where a block is in the ring.
struct Place {
  int stage;
  uint32_t parity;
  __device__ __forceinline__ void next(int stages) {
    if (++stage == stages) stage = 0, parity ^= 1u;
  }
};
// The sum over a block, each thread getting it; buf: a word a warp.
template <int TPR>
__device__ __forceinline__ float block_sum(float v, float* buf) {
  constexpr int NW = TPR / 32;
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  v = buf[threadIdx.x & (NW - 1)];
#pragma unroll
  for (int o = NW / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__host__ __device__ __forceinline__ int range_start(int64_t i, int64_t rows, int64_t ranges) { return (int)(i * rows / ranges); }
__host__ __device__ __forceinline__ int range_of(int64_t row, int64_t rows, int64_t ranges) { return (int)(((row + 1) * ranges - 1) / rows); }
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// 1 / sqrt(mean + eps), within 2 ulp.
__device__ __forceinline__ float rho_fast(float sq, float inv_width, float eps) { return rsqrtf(fmaf(sq, inv_width, eps)); }

// A block to a row.  kRowBlock threads, kPer elements each, in 16-byte pieces (LONG: any number, read again for each pass).
constexpr int kRowBlock = 512;
template <typename T, int VEC, bool Q8, bool LONG>
__global__ void __launch_bounds__(kRowBlock) block_norm_kernel(const BlockArgs a) {
  constexpr int TPR = kRowBlock, NV = kPer / VEC;
  __shared__ float buf_x[TPR / 32], buf_s[TPR / 32];
  __shared__ uint32_t buf_m[TPR / 32];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x, row = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
  const T* r = reinterpret_cast<const T*>(a.r) + row * a.ld_r;
  T* so = reinterpret_cast<T*>(a.s) + row * a.ld_s;
  const void* gate = gate_row<T>(a.gate, a.g_f32, row / a.group, a.ld_g);
  float rho_x = a.alpha;  // times alpha
  // x to the rounded s
  auto join = [&](int col, float(&f)[VEC], const float(&res)[VEC]) {
    float p[VEC], g[VEC];
    load_weight<VEC, T>(a.wp, a.p_f32, col, p);
    load_weight<VEC, T>(gate, a.g_f32, col, g);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = to_f<T>(from_f<T>(fmaf(f[i] * rho_x, p[i] * g[i], res[i])));
  };
  if constexpr (!LONG) {
    float f[NV][VEC], res[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[v][i] = res[v][i] = 0.f;
      if (col < a.width) {
        load_vec<VEC, T>(x + col, f[v]);
        load_vec<VEC, T>(r + col, res[v]);
      }
    }
    float sq = 0.f;
    if (a.post) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sq = fmaf(f[v][i], f[v][i], sq);
      rho_x *= rho_of(row_sum<TPR>(sq, buf_x), a.width, a.eps);
    }
    sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width) {
        join(col, f[v], res[v]);
        store_vec<VEC, T>(so + col, f[v]);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sq = fmaf(f[v][i], f[v][i], sq);
      }
    }
    const float rho = rho_of(row_sum<TPR>(sq, buf_s), a.width, a.eps);
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width) {
        float w[VEC];
        load_weight<VEC, T>(a.w, a.w_f32, col, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          f[v][i] = f[v][i] * rho * w[i];
          if (Q8) most = max(most, mag(f[v][i]));
        }
        if (!Q8) store_vec<VEC, T>(reinterpret_cast<T*>(a.y) + row * a.ld_y + col, f[v]);
      }
    }
    if (Q8) {
      const RowScale rs = row_scale(row_max<TPR>(most, buf_m));
      int8_t* y = reinterpret_cast<int8_t*>(a.y) + row * a.ld_y;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * TPR + t) * VEC;
        if (col < a.width) put_q<VEC>(y + col, f[v], rs);
      }
      if (t == 0) a.scale[row] = rs.scale;
    }
  } else {
    float sq = 0.f;
    if (a.post) {
      for (int col = t * VEC; col < a.width; col += TPR * VEC) {
        float f[VEC];
        load_vec<VEC, T>(x + col, f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sq = fmaf(f[i], f[i], sq);
      }
      rho_x *= rho_of(row_sum<TPR>(sq, buf_x), a.width, a.eps);
    }
    sq = 0.f;
    for (int col = t * VEC; col < a.width; col += TPR * VEC) {
      float f[VEC], res[VEC];
      load_vec<VEC, T>(x + col, f);
      load_vec<VEC, T>(r + col, res);
      join(col, f, res);
      store_vec<VEC, T>(so + col, f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sq = fmaf(f[i], f[i], sq);
    }
    const float rho = rho_of(row_sum<TPR>(sq, buf_s), a.width, a.eps);
    auto again = [&](int col, float(&f)[VEC]) {  // from the s that this thread has stored
      load_vec<VEC, T>(so + col, f);
      float w[VEC];
      load_weight<VEC, T>(a.w, a.w_f32, col, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = f[i] * rho * w[i];
    };
    uint32_t most = 0;
    for (int col = t * VEC; col < a.width; col += TPR * VEC) {
      float f[VEC];
      again(col, f);
      if (Q8) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) most = max(most, mag(f[i]));
      } else {
        store_vec<VEC, T>(reinterpret_cast<T*>(a.y) + row * a.ld_y + col, f);
      }
    }
    if (Q8) {
      const RowScale rs = row_scale(row_max<TPR>(most, buf_m));
      for (int col = t * VEC; col < a.width; col += TPR * VEC) {
        float f[VEC];
        again(col, f);
        put_q<VEC>(reinterpret_cast<int8_t*>(a.y) + row * a.ld_y + col, f, rs);
      }
      if (t == 0) a.scale[row] = rs.scale;
    }
  }
}

// Many rows of up to 16384 elements: x and r through the ring.  (4096 x 9000 in bf16 70 us by 1024 threads a row, 160 with a row in
// the registers of a block of 512, which an SM has room for one of.)
constexpr int walk_side(int tpr) { return 1024 / tpr; }  // blocks of an SM
template <typename T, int VEC, int TPR, bool Q8>
__global__ void __launch_bounds__(TPR, walk_side(TPR)) block_walk_kernel(const BlockArgs a, int stages, int pitch, int stage_bytes) {
  extern __shared__ __align__(16) uint4 ring_mem[];
  __shared__ float buf_x[TPR / 32], buf_s[2][TPR / 32];  // without x's norm one barrier a row: two buffers in turn
  __shared__ uint32_t buf_m[TPR / 32];
  dep_wait();
  dep_launch();
  const int r1 = range_start(blockIdx.x + 1, a.rows, gridDim.x);
  int row = range_start(blockIdx.x, a.rows, gridDim.x);
  __shared__ uint64_t bars[kMostStages];
  __shared__ int dead;
  const int es_gate = a.g_f32 ? 4 : (int)sizeof(T);
  const Ring<T, VEC, TPR, 2> ring{reinterpret_cast<uint8_t*>(ring_mem), bars, a.width, pitch, stages, (int)threadIdx.x, stage_bytes,
                                  {reinterpret_cast<const T*>(a.x), reinterpret_cast<const T*>(a.r)}, {a.ld_x, a.ld_r},
                                  a.ring_gate ? reinterpret_cast<const uint8_t*>(a.gate) : nullptr, a.ld_g * es_gate, a.width * es_gate, a.err, &dead};
  ring.init();
  const int first = row;
  T* so = reinterpret_cast<T*>(a.s) + row * a.ld_s;
  T* yo = reinterpret_cast<T*>(a.y) + (Q8 ? 0 : row * a.ld_y);
  const float inv_width = 1.f / (float)a.width;
  float2 w[kWalkVecs][4], c[kWalkVecs][4];
#pragma unroll
  for (int v = 0; v < kWalkVecs; ++v) ring.weight(a.w, a.w_f32, v, w[v]);
  for (int i = 0; i < (VEC == 8 ? stages : stages - 1); ++i) ring.fetch((int64_t)row + i, r1, i);
  Place at{0, 0u};
  int side = 0;
  while (row < r1) {
    const int g = row / a.group, end = (int)min((int64_t)r1, ((int64_t)g + 1) * a.group);
    const void* gate = gate_row<T>(a.gate, a.g_f32, g, a.ld_g);
    if (a.ring_gate) {
      ring.arrive(row, r1, at.stage, at.parity);
      gate = ring.row(at.stage, 2);
    }
#pragma unroll
    for (int v = 0; v < kWalkVecs; ++v) {  // c = alpha gate w_post
      float2 p[4];
      ring.weight(gate, a.g_f32, v, c[v]);
      ring.weight(a.wp, a.p_f32, v, p);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[v][i] = mul2(mul2(c[v][i], p[i]), both(a.alpha));
    }
    for (; row < end; ++row, side ^= 1, so += a.ld_s) {
      const int stage = at.stage;
      ring.arrive(row, r1, stage, at.parity);
      float rho_x = 1.f;
      if (a.post) {
        float2 sq = both(0.f);
#pragma unroll
        for (int v = 0; v < kWalkVecs; ++v) {
          float2 x[4];
          ring.read(row, stage, 0, v, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) sq = fma2(x[i], x[i], sq);
        }
        rho_x = rho_fast(block_sum<TPR>(sq.x + sq.y, buf_x), inv_width, a.eps);
        ring.refill(row, first, r1, stage);
      }
      float2 s[kWalkVecs][4], sq = both(0.f);
#pragma unroll
      for (int v = 0; v < kWalkVecs; ++v) {
        float2 x[4];
        ring.read(row, stage, 0, v, x);
        ring.read(row, stage, 1, v, s[v]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = fma2(mul2(x[i], both(rho_x)), c[v][i], s[v][i]);
          s[v][i] = make_float2(to_f<T>(from_f<T>(f.x)), to_f<T>(from_f<T>(f.y)));
          sq = fma2(s[v][i], s[v][i], sq);
        }
        ring.store(so, v, s[v]);
      }
      const float rho = rho_fast(block_sum<TPR>(sq.x + sq.y, buf_s[side]), inv_width, a.eps);
      if (!a.post) ring.refill(row, first, r1, stage);
      uint32_t most = 0;
#pragma unroll
      for (int v = 0; v < kWalkVecs; ++v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[v][i] = mul2(mul2(s[v][i], both(rho)), w[v][i]);
          if (Q8) {  // elements beyond the row's end are not there to make 0 inf of
            if (VEC == 8 ? ring.any(v) : ring.column(v, 2 * i) < a.width) most = max(most, mag(s[v][i].x));
            if (VEC == 8 ? ring.any(v) : ring.column(v, 2 * i + 1) < a.width) most = max(most, mag(s[v][i].y));
          }
        }
        if (!Q8) ring.store(yo, v, s[v]);
      }
      if (!Q8) yo += a.ld_y;
      if (Q8) {
        const RowScale rs = row_scale(row_max<TPR>(most, buf_m));
        int8_t* y = reinterpret_cast<int8_t*>(a.y) + row * a.ld_y;
#pragma unroll
        for (int v = 0; v < kWalkVecs; ++v) {
          const float e[8] = {s[v][0].x, s[v][0].y, s[v][1].x, s[v][1].y, s[v][2].x, s[v][2].y, s[v][3].x, s[v][3].y};
          if constexpr (VEC == 8) {
            if (ring.any(v)) put_q<8>(y + ring.column(v, 0), e, rs);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (ring.column(v, i) < a.width) y[ring.column(v, i)] = rs.ok ? (int8_t)rounded_bits(e[i], rs.inv) : (int8_t)0;
          }
        }
        if (threadIdx.x == 0) a.scale[row] = rs.scale;
      }
      ring.turn(row, r1);
      at.next(stages);
    }
  }
  ring.end();
}

// Narrow rows, up to 256 elements, several to a warp: L lanes a row, eight elements to a lane, and every such slot of a block walks
// down a run of rows of its own, with its weights in registers and the next row on its way.  The slots of a warp take part in
// its shuffles until the last of them is done.  131072 x 128 in bf16 with one row to a slot and nothing ahead: 45 us forward, 108
// backward.
template <int VEC, int L, typename T>
struct NarrowRow {
  T e[kNarrow];
  __device__ __forceinline__ void load(const T* p, int width, int t, bool live) {
    if constexpr (VEC == 8) {
      uint4* to = reinterpret_cast<uint4*>(e);
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) to[i] = make_uint4(0u, 0u, 0u, 0u);
      if (live && kNarrow * t < width) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) to[i] = reinterpret_cast<const uint4*>(p + kNarrow * t)[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) e[i] = live && t + L * i < width ? p[t + L * i] : from_f<T>(0.f);
    }
  }
  __device__ __forceinline__ void get(float (&f)[kNarrow]) const {
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) f[i] = to_f<T>(e[i]);
  }
};
__device__ __forceinline__ int most_steps(int steps, int lanes) {
  for (int o = lanes; o < 32; o <<= 1) steps = max(steps, __shfl_xor_sync(0xffffffffu, steps, o));
  return steps;
}
template <typename T, int VEC, int L, bool Q8>
__global__ void __launch_bounds__(kNarrowBlock) narrow_block_kernel(const BlockArgs a, int ranges) {
  dep_wait();
  dep_launch();
  const int t = threadIdx.x % L, range = blockIdx.x * (kNarrowBlock / L) + threadIdx.x / L;
  const bool there = range < ranges;
  const int r0 = there ? range_start(range, a.rows, ranges) : 0, r1 = there ? range_start(range + 1, a.rows, ranges) : 0;
  const int steps = most_steps(r1 - r0, L);
  const float inv_width = 1.f / (float)a.width;
  const T* x = reinterpret_cast<const T*>(a.x) + r0 * a.ld_x;
  const T* r = reinterpret_cast<const T*>(a.r) + r0 * a.ld_r;
  NarrowRow<VEC, L, T> next_x, next_r;
  next_x.load(x, a.width, t, r0 < r1);
  next_r.load(r, a.width, t, r0 < r1);
  float w[kNarrow], p[kNarrow], c[kNarrow];
  narrow_weight<VEC, L, T>(a.w, a.w_f32, a.width, t, w);
  narrow_weight<VEC, L, T>(a.wp, a.p_f32, a.width, t, p);
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) c[i] = 0.f;
  int s1 = r0;
  for (int row = r0; row < r0 + steps; ++row) {
    const bool live = row < r1;  // the lanes of rows beyond the last take part in the shuffles
    if (live && row == s1) {
      const int g = row / a.group;
      s1 = (int)min((int64_t)r1, ((int64_t)g + 1) * a.group);
      narrow_weight<VEC, L, T>(gate_row<T>(a.gate, a.g_f32, g, a.ld_g), a.g_f32, a.width, t, c);
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) c[i] *= a.alpha * p[i];
    }
    float f[kNarrow], res[kNarrow];
    next_x.get(f);
    next_r.get(res);
    x += a.ld_x, r += a.ld_r;
    next_x.load(x, a.width, t, row + 1 < r1);
    next_r.load(r, a.width, t, row + 1 < r1);
    float rho_x = 1.f;
    if (a.post) {
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) sq = fmaf(f[i], f[i], sq);
      rho_x = rho_fast(group_sum<L>(sq), inv_width, a.eps);
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) {
      // elements beyond the row's end are not there to make 0 inf of
      f[i] = narrow_column<VEC, L>(t, i) < a.width ? to_f<T>(from_f<T>(fmaf(f[i] * rho_x, c[i], res[i]))) : 0.f;
      sq = fmaf(f[i], f[i], sq);
    }
    if (live) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.s) + row * a.ld_s, a.width, t, f);
    const float rho = rho_fast(group_sum<L>(sq), inv_width, a.eps);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) {
      f[i] = narrow_column<VEC, L>(t, i) < a.width ? f[i] * rho * w[i] : 0.f;
      if (Q8) most = max(most, mag(f[i]));
    }
    if (!Q8) {
      if (live) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.y) + row * a.ld_y, a.width, t, f);
    } else {
      const RowScale rs = row_scale(group_max<L>(most));
      if (live) {
        narrow_put_q<VEC, L>(reinterpret_cast<int8_t*>(a.y) + row * a.ld_y, a.width, t, f, rs);
        if (t == 0) a.scale[row] = rs.scale;
      }
    }
  }
}

constexpr int kWalkSmem = 225 * 1024;
// Shared memory that one of `side` blocks of an SM may ask for, next to what it declares and the 1 KB that a block costs; it is given out
// in pieces of 128 bytes.
int walk_room(int side, int declared) { return std::min(kWalkSmem, 228 * 1024 / side / 128 * 128 - 1024 - declared); }
// What the kernels declare beside it: words a warp (forward: sums of x, two of s, a maximum; backward: two of eight sums), barriers, a flag.
int walk_declared(int threads) { return threads / 32 * 16 + 128; }
int grad_declared(int threads) { return threads / 32 * 64 + 128; }
int walk_threads(int width) { return width <= 1024 ? 64 : width <= 2048 ? 128 : width <= 4096 ? 256 : width <= 8192 ? 512 : 1024; }
// Bytes of a part of a row in the ring: all that the threads read, 32 more for one that does not start on 16 bytes.
int walk_pitch(int width, int es, bool vec) { return walk_threads(width) * kWalkPer * es + (vec ? 0 : 32); }
template <typename T, int VEC, bool Q8>
void walk_rows_of(const asd_ops* o, BlockArgs n, cudaStream_t st) {
  const int threads = walk_threads(n.width), pitch = walk_pitch(n.width, sizeof(T), VEC == 8);
  n.ring_gate = VEC == 8 && n.gate && n.group == 1;
  n.err = o->err;
  const int stage_bytes = 2 * pitch + (n.ring_gate ? n.width * (n.g_f32 ? 4 : (int)sizeof(T)) : 0);  // one of them always finds room
  // as many blocks of an SM as its registers hold, unless shared memory then has no room for a row ahead
  int side = walk_side(threads);
  auto room = [&]() { return walk_room(side, walk_declared(threads)) / stage_bytes; };
  while (side > 1 && room() < 2) --side;
  const int stages = std::max(1, std::min(VEC == 8 ? kMostStages : 2, room()));
  const dim3 grid(std::min(n.rows, side * o->num_sms)), block(threads);
  void (*kernel)(BlockArgs, int, int, int) = threads == 64    ? block_walk_kernel<T, VEC, 64, Q8>
                                             : threads == 128 ? block_walk_kernel<T, VEC, 128, Q8>
                                             : threads == 256 ? block_walk_kernel<T, VEC, 256, Q8>
                                             : threads == 512 ? block_walk_kernel<T, VEC, 512, Q8>
                                                              : block_walk_kernel<T, VEC, 1024, Q8>;
  ops_launch(kernel, grid, block, (size_t)stages * stage_bytes, st, 1, n, stages, pitch, stage_bytes);
}
template <typename T, bool Q8>
void block_t(const asd_ops* o, const BlockArgs& n, bool vec, cudaStream_t st) {
  if (n.width <= kNarrowWidth) {
    with_lanes(n.width, [&](auto lanes) {
      constexpr int L = decltype(lanes)::value;
      const int ranges = std::min(n.rows, 8 * o->num_sms * (kNarrowBlock / L));
      ops_launch(vec ? narrow_block_kernel<T, 8, L, Q8> : narrow_block_kernel<T, 1, L, Q8>, dim3(narrow_grid(ranges, L, kNarrowBlock)),
                 dim3(kNarrowBlock), 0, st, 1, n, ranges);
    });
    return;
  }
  if (n.width > kMostWalkWidth) {
    ops_launch(vec ? block_norm_kernel<T, 8, Q8, true> : block_norm_kernel<T, 1, Q8, true>, dim3(n.rows), dim3(kRowBlock), 0, st, 1, n);
    return;
  }
  // few rows: a block to each, with the row in registers
  if (vec && n.rows <= o->num_sms)
    ops_launch(block_norm_kernel<T, 8, Q8, false>, dim3(n.rows), dim3(kRowBlock), 0, st, 1, n);
  else
    vec ? walk_rows_of<T, 8, Q8>(o, n, st) : walk_rows_of<T, 1, Q8>(o, n, st);
}

// ---- backward --------------------------------------------------------------------------------------------

constexpr int kMostGradWidth = 512 * kWalkPer;  // beyond, columns are summed by a kernel of their own

// Rows are cut into `ranges` runs of neighbouring rows, [i rows / ranges, (i + 1) rows / ranges), each walked over by one block (or
// one row slot of it).  A range's sums of dw and dw_post go to part_w and part_post; the gradient of a row of the gate whose rows
// are all in the range is complete at their last, otherwise its part goes to part_gate: 0 if the part begins where the range
// begins, 1 if not (at most two of a range's gate rows reach beyond it).
struct BlockGradArgs {
  int rows, width, group, post, ranges;
  int w_f32, p_f32, g_f32;
  int stages, pitch, stage_bytes;  // rows in shared memory, bytes of a part of one, of all its parts
  int ring_gate;                   // a row of the gate to every row, brought with it
  int* err;
  int ldp;            // elements from one row of partial sums to the next: a multiple of 4
  int wide_dg;        // rows of dgate are on 16 bytes
  float eps, alpha;
  const void *dy, *ds, *x, *s, *w, *wp, *gate;
  void *dx, *dr, *dgate;
  int64_t ld_dy, ld_ds, ld_x, ld_s, ld_g, ld_dx, ld_dr, ld_dg;
  float *part_w, *part_post, *part_gate;  // [blocks, ldp], [blocks, ldp], [ranges, 2, ldp]; NULL: not wanted
  float* stats;                           // wide rows: [rows, 4]
};

template <typename T>
__device__ __forceinline__ void put_value(void* p, int64_t at, float v, bool f32) {
  if (f32)
    reinterpret_cast<float*>(p)[at] = v;
  else
    reinterpret_cast<T*>(p)[at] = from_f<T>(v);
}
// The sum u of dS n over the rows [s0, s1) of gate row g, which range `i` from row r0 on has walked over: one column of it.
template <typename T>
__device__ __forceinline__ void flush_gate(const BlockGradArgs& a, int i, int r0, int g, int s0, int s1, int col, float u, float wp) {
  const float v = a.alpha * wp * u;
  if (s0 == (int64_t)g * a.group && s1 == ((int64_t)g + 1) * a.group)
    put_value<T>(a.dgate, (int64_t)g * a.ld_dg + col, v, a.g_f32);
  else
    a.part_gate[((int64_t)2 * i + (s0 == r0 ? 0 : 1)) * a.ldp + col] = v;
}

// The sums of eight values over a block, each thread getting all of them.  `buf`: 8 words a warp, free again after another barrier.
// In a warp each step halves the values that a lane holds.
template <int TPR>
__device__ __forceinline__ void block_sums(float (&v)[8], float* buf) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int w = 16, n = 4; n; w >>= 1, n >>= 1) {
    const bool up = lane & w;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
    }
  }
  v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
  v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
  if ((lane & 3) == 0) buf[(threadIdx.x >> 5) * 8 + (lane >> 2)] = v[0];  // bits 4, 3, 2 of the lane are bits 2, 1, 0 of the value's number
  __syncthreads();
  float s = 0.f;
  if constexpr (TPR >= 128) {
#pragma unroll
    for (int i = 0; i < TPR / 128; ++i) s += buf[i * 32 + lane];
  } else {
    if (lane < TPR / 4) s = buf[lane];
  }
  s += __shfl_xor_sync(0xffffffffu, s, 8);
  s += __shfl_xor_sync(0xffffffffu, s, 16);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __shfl_sync(0xffffffffu, s, i);
}

// A vector of a row of partial sums, whose address is a multiple of four elements.
template <int VEC, typename R>
__device__ __forceinline__ void put_sums(const R& ring, float* to, int v, const float2 (&f)[4]) {
  if constexpr (VEC == 8) {
    if (!ring.any(v)) return;
    float4* p = reinterpret_cast<float4*>(to + ring.column(v, 0));
    p[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    p[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (ring.column(v, i) < ring.width) to[ring.column(v, i)] = i & 1 ? f[i >> 1].y : f[i >> 1].x;
  }
}

// A row's factors from its six sums: dS = ds + rho (dy w) + k z,  dx = rho_x (c dS) + kx n.  (rho^3, for k s, may leave the range of
// 32 bits where the gradient does not.)
struct RowFactors {
  float rho, k, rho_x, kx;
};
__device__ __forceinline__ RowFactors row_factors(float ss, float xx, float gs, float inv_width, const BlockGradArgs& a) {
  RowFactors f;
  f.rho = rho_fast(ss, inv_width, a.eps);
  f.k = -(f.rho * gs * inv_width) * f.rho;
  f.rho_x = a.post ? rho_fast(xx, inv_width, a.eps) : 1.f;
  f.kx = 0.f;
  return f;
}
// kx from the sum of c x times dS, which is linear in those of c x times ds, dy w and s.
__device__ __forceinline__ void factor_of_n(RowFactors& f, float cx_ds, float cx_g, float cx_s, float inv_width) {
  const float dot = fmaf(f.k, f.rho * cx_s, fmaf(f.rho, cx_g, cx_ds));
  f.kx = -(f.rho_x * dot * inv_width) * f.rho_x;
}
// Rows of x and s so small that their products leave the normal range where those of n and z do not (which matters with an eps
// of the same size): the sum of c n dS is taken itself, once the other factors are known.
__device__ __forceinline__ bool products_too_small(float ss, float xx, float inv_width, const BlockGradArgs& a) {
  return a.post && xx > 0.f && (ss * inv_width) * (xx * inv_width) < 7.52316385e-37f;  // 2^-120
}

// The sum dw_post is added to once for each run of a gate row, and lives in shared memory behind the ring.
constexpr int grad_side(int tpr) { return 512 / tpr; }  // blocks of an SM
template <typename T, int VEC, int TPR>
__global__ void __launch_bounds__(TPR, grad_side(TPR)) block_grad_kernel(const BlockGradArgs a) {
  constexpr int NV = kWalkVecs;
  extern __shared__ __align__(16) uint4 ring_mem[];
  __shared__ float buf[2][TPR / 32 * 8];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x;
  const int r0 = range_start(blockIdx.x, a.rows, a.ranges), r1 = range_start(blockIdx.x + 1, a.rows, a.ranges);
  __shared__ uint64_t bars[kMostStages];
  __shared__ int dead;
  const int es_gate = a.g_f32 ? 4 : (int)sizeof(T);
  const Ring<T, VEC, TPR, 4> ring{reinterpret_cast<uint8_t*>(ring_mem), bars, a.width, a.pitch, a.stages, t, a.stage_bytes,
                                  {reinterpret_cast<const T*>(a.s), reinterpret_cast<const T*>(a.dy), reinterpret_cast<const T*>(a.x), reinterpret_cast<const T*>(a.ds)},
                                  {a.ld_s, a.ld_dy, a.ld_x, a.ld_ds},
                                  a.ring_gate ? reinterpret_cast<const uint8_t*>(a.gate) : nullptr, a.ld_g * es_gate, a.width * es_gate, a.err, &dead};
  ring.init();
  float4* acc_p = reinterpret_cast<float4*>(reinterpret_cast<uint8_t*>(ring_mem) + (size_t)a.stages * a.stage_bytes) + t;  // [2 NV][TPR]
  T* dr = reinterpret_cast<T*>(a.dr) + (a.dr ? r0 * a.ld_dr : 0);
  T* dx = reinterpret_cast<T*>(a.dx) + (a.dx ? r0 * a.ld_dx : 0);
  const float inv_width = 1.f / (float)a.width;
  const float2 zero = make_float2(0.f, 0.f);
  float2 w[NV][4], c[NV][4], u[NV][4], acc_w[NV][4];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    ring.weight(a.w, a.w_f32, v, w[v]);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[v][i] = acc_w[v][i] = zero;
    if (a.part_post) acc_p[2 * v * TPR] = acc_p[(2 * v + 1) * TPR] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int i = 0; i < (VEC == 8 ? a.stages : a.stages - 1); ++i) ring.fetch((int64_t)r0 + i, r1, i);
  Place at{0, 0u};
  int side = 0;
  for (int row = r0; row < r1;) {
    const int g = row / a.group, s0 = row;
    const int s1 = (int)min((int64_t)r1, ((int64_t)g + 1) * a.group);
    const void* gate = gate_row<T>(a.gate, a.g_f32, g, a.ld_g);
    if (a.ring_gate) {
      ring.arrive(row, r1, at.stage, at.parity);
      gate = ring.row(at.stage, 4);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float2 p[4];
      ring.weight(gate, a.g_f32, v, c[v]);
      ring.weight(a.wp, a.p_f32, v, p);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[v][i] = mul2(mul2(c[v][i], p[i]), both(a.alpha));
    }
    for (; row < s1; ++row, side ^= 1) {
      const int stage = at.stage;
      ring.arrive(row, r1, stage, at.parity);
      float2 m[6] = {zero, zero, zero, zero, zero, zero};
      auto add_up = [&](auto with_norm) {
        constexpr bool post = decltype(with_norm)::value;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          float2 s[4], dy[4], x[4], ds[4];
          ring.read(row, stage, 0, v, s);
          ring.read(row, stage, 1, v, dy);
          if (post) {
            ring.read(row, stage, 2, v, x);
            ring.read(row, stage, 3, v, ds);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 gi = mul2(dy[i], w[v][i]);
            m[0] = fma2(s[i], s[i], m[0]);
            m[2] = fma2(gi, s[i], m[2]);
            if (post) {
              const float2 cx = mul2(c[v][i], x[i]);
              m[1] = fma2(x[i], x[i], m[1]);
              m[3] = fma2(cx, ds[i], m[3]);
              m[4] = fma2(cx, gi, m[4]);
              m[5] = fma2(cx, s[i], m[5]);
            }
          }
        }
      };
      if (a.post)
        add_up(std::true_type());
      else
        add_up(std::false_type());
      float sum[8] = {m[0].x + m[0].y, m[1].x + m[1].y, m[2].x + m[2].y, m[3].x + m[3].y, m[4].x + m[4].y, m[5].x + m[5].y, 0.f, 0.f};
      block_sums<TPR>(sum, buf[side]);
      ring.refill(row, r0, r1, stage);
      RowFactors f = row_factors(sum[0], sum[1], sum[2], inv_width, a);
      if (a.post) factor_of_n(f, sum[3], sum[4], sum[5], inv_width);
      if (products_too_small(sum[0], sum[1], inv_width, a)) {
        float dot[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int v = 0; v < NV; ++v) {
          float2 s[4], dy[4], x[4], ds[4];
          ring.read(row, stage, 0, v, s);
          ring.read(row, stage, 1, v, dy);
          ring.read(row, stage, 2, v, x);
          ring.read(row, stage, 3, v, ds);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 wv = v ? w[NV - 1][i] : w[0][i], cv = v ? c[NV - 1][i] : c[0][i];
            const float2 dS = fma2(mul2(s[i], both(f.rho)), both(f.k), fma2(mul2(dy[i], wv), both(f.rho), ds[i]));
            const float2 part = mul2(mul2(cv, dS), mul2(x[i], both(f.rho_x)));
            dot[0] += part.x + part.y;
          }
        }
        block_sums<TPR>(dot, buf[side ^ 1]);
        __syncthreads();  // the next row uses that buffer
        f.kx = -(dot[0] * inv_width) * f.rho_x;
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float2 s[4], dy[4], x[4], dS[4];
        ring.read(row, stage, 0, v, s);
        ring.read(row, stage, 1, v, dy);
        ring.read(row, stage, 2, v, x);
        ring.read(row, stage, 3, v, dS);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 z = mul2(s[i], both(f.rho)), n = mul2(x[i], both(f.rho_x));
          dS[i] = fma2(z, both(f.k), fma2(mul2(dy[i], w[v][i]), both(f.rho), dS[i]));
          acc_w[v][i] = fma2(dy[i], z, acc_w[v][i]);
          u[v][i] = fma2(dS[i], n, u[v][i]);
          x[i] = fma2(n, both(f.kx), mul2(mul2(c[v][i], dS[i]), both(f.rho_x)));
        }
        if (a.dr) ring.store(dr, v, dS);
        if (a.dx) ring.store(dx, v, x);
      }
      dr += a.ld_dr, dx += a.ld_dx;
      ring.turn(row, r1);
      at.next(a.stages);
    }
    if (a.part_post || a.part_gate) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float2 gw[4], p[4];
        ring.weight(gate, a.g_f32, v, gw);
        ring.weight(a.wp, a.p_f32, v, p);
        if (a.part_post) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float4& to = acc_p[(2 * v + h) * TPR];
            const float2 x = fma2(mul2(gw[2 * h], both(a.alpha)), u[v][2 * h], make_float2(to.x, to.y));
            const float2 y = fma2(mul2(gw[2 * h + 1], both(a.alpha)), u[v][2 * h + 1], make_float2(to.z, to.w));
            to = make_float4(x.x, x.y, y.x, y.y);
          }
        }
        if (a.part_gate) {
          const bool whole = s0 == (int64_t)g * a.group && s1 == ((int64_t)g + 1) * a.group;
#pragma unroll
          for (int i = 0; i < 4; ++i) u[v][i] = mul2(mul2(u[v][i], p[i]), both(a.alpha));
          const int64_t part = ((int64_t)2 * blockIdx.x + (s0 == r0 ? 0 : 1)) * a.ldp;
          if (!whole) {
            put_sums<VEC>(ring, a.part_gate + part, v, u[v]);
          } else if (VEC == 8 && !a.g_f32 && a.wide_dg) {
            ring.store(reinterpret_cast<T*>(a.dgate) + (int64_t)g * a.ld_dg, v, u[v]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (ring.column(v, i) < a.width) put_value<T>(a.dgate, (int64_t)g * a.ld_dg + ring.column(v, i), i & 1 ? u[v][i >> 1].y : u[v][i >> 1].x, a.g_f32);
          }
        }
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) u[v][i] = zero;
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if (a.part_w) put_sums<VEC>(ring, a.part_w + (int64_t)blockIdx.x * a.ldp, v, acc_w[v]);
    if (a.part_post) {
      const float4 x = acc_p[2 * v * TPR], y = acc_p[(2 * v + 1) * TPR];
      const float2 f[4] = {make_float2(x.x, x.y), make_float2(x.z, x.w), make_float2(y.x, y.y), make_float2(y.z, y.w)};
      put_sums<VEC>(ring, a.part_post + (int64_t)blockIdx.x * a.ldp, v, f);
    }
  }
  ring.end();
}

// Narrow rows: a range to each slot.
template <typename T, int VEC, int L>
__global__ void __launch_bounds__(kNarrowBlock) narrow_block_grad_kernel(const BlockGradArgs a) {
  constexpr int SLOTS = kNarrowBlock / L;
  __shared__ float sums[2][kNarrowBlock / 32][kNarrowWidth];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x % L, range = blockIdx.x * SLOTS + threadIdx.x / L;
  const bool there = range < a.ranges;
  const int r0 = there ? range_start(range, a.rows, a.ranges) : 0, r1 = there ? range_start(range + 1, a.rows, a.ranges) : 0;
  const float inv_width = 1.f / (float)a.width;
  const int steps = most_steps(r1 - r0, L);
  const T* at[4] = {reinterpret_cast<const T*>(a.s) + r0 * a.ld_s, reinterpret_cast<const T*>(a.dy) + r0 * a.ld_dy,
                    reinterpret_cast<const T*>(a.x) + r0 * a.ld_x, reinterpret_cast<const T*>(a.ds) + (a.ds ? r0 * a.ld_ds : 0)};
  NarrowRow<VEC, L, T> next[4];
  auto fetch = [&](bool live) {
#pragma unroll
    for (int k = 0; k < 4; ++k) next[k].load(at[k], a.width, t, live && (k < 3 || a.ds));
    at[0] += a.ld_s, at[1] += a.ld_dy, at[2] += a.ld_x, at[3] += a.ld_ds;
  };
  fetch(r0 < r1);
  float w[kNarrow], p[kNarrow], gate[kNarrow], u[kNarrow], acc_w[kNarrow], acc_p[kNarrow];
  narrow_weight<VEC, L, T>(a.w, a.w_f32, a.width, t, w);
  narrow_weight<VEC, L, T>(a.wp, a.p_f32, a.width, t, p);
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) {
    if (narrow_column<VEC, L>(t, i) >= a.width) w[i] = p[i] = 0.f;
    u[i] = acc_w[i] = acc_p[i] = gate[i] = 0.f;
  }
  int g = -1, s0 = 0, s1 = 0;
  for (int k = 0; k < steps; ++k) {
    const int row = r0 + k;
    const bool live = row < r1;
    if (live && row == (g < 0 ? r0 : s1)) {
      g = row / a.group, s0 = row, s1 = (int)min((int64_t)r1, ((int64_t)g + 1) * a.group);
      narrow_weight<VEC, L, T>(gate_row<T>(a.gate, a.g_f32, g, a.ld_g), a.g_f32, a.width, t, gate);
    }
    float s[kNarrow], dy[kNarrow], x[kNarrow], ds[kNarrow];
    next[0].get(s);
    next[1].get(dy);
    next[2].get(x);
    next[3].get(ds);
    fetch(row + 1 < r1);
    float ss = 0.f, xx = 0.f, gs = 0.f;
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) {
      ss = fmaf(s[i], s[i], ss);
      gs = fmaf(dy[i] * w[i], s[i], gs);
      xx = fmaf(x[i], x[i], xx);
    }
    ss = group_sum<L>(ss), gs = group_sum<L>(gs);
    if (a.post) xx = group_sum<L>(xx);
    RowFactors f = row_factors(ss, xx, gs, inv_width, a);
    float dx[kNarrow], dot = 0.f;  // dx: c dS at first
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) {
      const float z = s[i] * f.rho;
      x[i] *= f.rho_x;  // n
      ds[i] = fmaf(z, f.k, fmaf(dy[i] * w[i], f.rho, ds[i]));
      dx[i] = a.alpha * gate[i] * p[i] * ds[i];
      if (live) {
        acc_w[i] = fmaf(dy[i], z, acc_w[i]);
        u[i] = fmaf(ds[i], x[i], u[i]);
        dot = fmaf(dx[i], x[i], dot);
      }
    }
    if (a.post) f.kx = -(group_sum<L>(dot) * inv_width) * f.rho_x;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) dx[i] = fmaf(x[i], f.kx, dx[i] * f.rho_x);
    if (a.dr) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.dr) + row * a.ld_dr, a.width, t, ds);
    if (a.dx) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.dx) + row * a.ld_dx, a.width, t, dx);
    if (row + 1 == s1) {
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) {
        const int col = narrow_column<VEC, L>(t, i);
        if (a.part_gate && col < a.width) flush_gate<T>(a, range, r0, g, s0, s1, col, u[i], p[i]);
        acc_p[i] = fmaf(a.alpha * gate[i], u[i], acc_p[i]);
        u[i] = 0.f;
      }
    }
  }
  if (!a.part_w && !a.part_post) return;
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) {
    for (int o = L; o < 32; o <<= 1) {
      acc_w[i] += __shfl_xor_sync(0xffffffffu, acc_w[i], o);
      acc_p[i] += __shfl_xor_sync(0xffffffffu, acc_p[i], o);
    }
    if ((threadIdx.x & 31) < L) {
      sums[0][threadIdx.x >> 5][narrow_column<VEC, L>(t, i)] = acc_w[i];
      sums[1][threadIdx.x >> 5][narrow_column<VEC, L>(t, i)] = acc_p[i];
    }
  }
  __syncthreads();
  for (int col = threadIdx.x; col < a.width; col += kNarrowBlock) {
    float v[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kNarrowBlock / 32; ++k) v[0] += sums[0][k][col], v[1] += sums[1][k][col];
    if (a.part_w) a.part_w[(int64_t)blockIdx.x * a.ldp + col] = v[0];
    if (a.part_post) a.part_post[(int64_t)blockIdx.x * a.ldp + col] = v[1];
  }
}

// Rows of more than 8192: dr and dx row by row, each read twice, with the row's factors kept; then the sums by columns, VEC to a
// thread, over ranges that are few enough for their partial sums to be little beside the rows.  The accumulators of a walk would be 96
// registers for each of 1024 threads.  4096 x 9000 in bf16 156 us and 75 more with the sums; an element at a time and 296 ranges 337
// and 153.  Both wait for memory: more warps (80 registers, a few of them spilled) are faster than all of them kept.
constexpr int kLongBlock = 256;
template <int VEC, typename T>
__device__ __forceinline__ void load_or_zero(const T* p, int64_t at, float (&f)[VEC]) {
  if (p) {
    load_vec<VEC, T>(p + at, f);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = 0.f;
  }
}
template <typename T, int VEC>
__global__ void __launch_bounds__(kLongBlock, VEC == 8 ? 3 : 4) block_grad_long_kernel(const BlockGradArgs a) {
  __shared__ float buf[kLongBlock / 32 * 8];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* s = reinterpret_cast<const T*>(a.s) + row * a.ld_s;
  const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.ld_dy;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
  const T* ds = a.ds ? reinterpret_cast<const T*>(a.ds) + row * a.ld_ds : nullptr;
  const void* gate = gate_row<T>(a.gate, a.g_f32, row / a.group, a.ld_g);
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  struct Columns {
    float s[VEC], x[VEC], g[VEC], c[VEC], ds[VEC];  // g = dy w, c = alpha gate w_post
  };
  auto load = [&](int col, Columns& f) {
    float w[VEC], p[VEC], g[VEC];
    load_vec<VEC, T>(s + col, f.s);
    load_vec<VEC, T>(x + col, f.x);
    load_vec<VEC, T>(dy + col, f.g);
    load_or_zero<VEC, T>(ds, col, f.ds);
    load_weight<VEC, T>(a.w, a.w_f32, col, w);
    load_weight<VEC, T>(a.wp, a.p_f32, col, p);
    load_weight<VEC, T>(gate, a.g_f32, col, g);
#pragma unroll
    for (int i = 0; i < VEC; ++i) f.g[i] *= w[i], f.c[i] = a.alpha * p[i] * g[i];
  };
  for (int col = t * VEC; col < a.width; col += kLongBlock * VEC) {
    Columns f;
    load(col, f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float cx = f.c[i] * f.x[i];
      v[0] = fmaf(f.s[i], f.s[i], v[0]);
      v[1] = fmaf(f.x[i], f.x[i], v[1]);
      v[2] = fmaf(f.g[i], f.s[i], v[2]);
      v[3] = fmaf(cx, f.ds[i], v[3]);
      v[4] = fmaf(cx, f.g[i], v[4]);
      v[5] = fmaf(cx, f.s[i], v[5]);
    }
  }
  block_sums<kLongBlock>(v, buf);
  const float inv_width = 1.f / (float)a.width;
  RowFactors k = row_factors(v[0], v[1], v[2], inv_width, a);
  if (a.post) factor_of_n(k, v[3], v[4], v[5], inv_width);
  auto of_s = [&](const Columns& f, int i) { return fmaf(f.s[i] * k.rho, k.k, fmaf(f.g[i], k.rho, f.ds[i])); };  // dS
  if (products_too_small(v[0], v[1], inv_width, a)) {
    float dot[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int col = t * VEC; col < a.width; col += kLongBlock * VEC) {
      Columns f;
      load(col, f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) dot[0] = fmaf(f.c[i] * of_s(f, i), f.x[i] * k.rho_x, dot[0]);
    }
    __syncthreads();  // the sums of before have been read
    block_sums<kLongBlock>(dot, buf);
    k.kx = -(dot[0] * inv_width) * k.rho_x;
  }
  if (t == 0 && a.stats) reinterpret_cast<float4*>(a.stats)[row] = make_float4(k.rho, k.k, k.rho_x, 0.f);
  if (!a.dr && !a.dx) return;
  for (int col = t * VEC; col < a.width; col += kLongBlock * VEC) {
    Columns f;
    load(col, f);
    float dr[VEC], dx[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) dr[i] = of_s(f, i), dx[i] = fmaf(f.x[i] * k.rho_x, k.kx, f.c[i] * dr[i] * k.rho_x);
    if (a.dx) store_vec<VEC, T>(reinterpret_cast<T*>(a.dx) + row * a.ld_dx + col, dx);
    if (a.dr) store_vec<VEC, T>(reinterpret_cast<T*>(a.dr) + row * a.ld_dr + col, dr);
  }
}
template <typename T, int VEC>
__global__ void __launch_bounds__(128, VEC == 8 ? 6 : 8) block_columns_kernel(const BlockGradArgs a) {
  dep_wait();
  dep_launch();
  const int col = (blockIdx.x * 128 + threadIdx.x) * VEC, range = blockIdx.y;
  if (col >= a.width) return;
  const int r0 = range_start(range, a.rows, a.ranges), r1 = range_start(range + 1, a.rows, a.ranges);
  float w[VEC], p[VEC], acc_w[VEC], acc_p[VEC];
  load_weight<VEC, T>(a.w, a.w_f32, col, w);
  load_weight<VEC, T>(a.wp, a.p_f32, col, p);
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc_w[i] = acc_p[i] = 0.f;
  for (int64_t row = r0; row < r1;) {
    const int g = (int)(row / a.group), s0 = (int)row, s1 = (int)min((int64_t)r1, ((int64_t)g + 1) * a.group);
    float gate[VEC], u[VEC];
    load_weight<VEC, T>(gate_row<T>(a.gate, a.g_f32, g, a.ld_g), a.g_f32, col, gate);
#pragma unroll
    for (int i = 0; i < VEC; ++i) u[i] = 0.f;
#pragma unroll(VEC == 8 ? 2 : 4)
    for (; row < s1; ++row) {
      const float4 f = reinterpret_cast<const float4*>(a.stats)[row];
      float s[VEC], dy[VEC], x[VEC], ds[VEC];
      load_vec<VEC, T>(reinterpret_cast<const T*>(a.s) + row * a.ld_s + col, s);
      load_vec<VEC, T>(reinterpret_cast<const T*>(a.dy) + row * a.ld_dy + col, dy);
      load_vec<VEC, T>(reinterpret_cast<const T*>(a.x) + row * a.ld_x + col, x);
      load_or_zero<VEC, T>(reinterpret_cast<const T*>(a.ds), row * a.ld_ds + col, ds);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        acc_w[i] = fmaf(dy[i], s[i] * f.x, acc_w[i]);
        u[i] = fmaf(fmaf(s[i] * f.x, f.y, fmaf(dy[i] * w[i], f.x, ds[i])), x[i] * f.z, u[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      acc_p[i] = fmaf(a.alpha * gate[i], u[i], acc_p[i]);
      if (a.part_gate) flush_gate<T>(a, range, r0, g, s0, s1, col + i, u[i], p[i]);
    }
  }
  if (a.part_w) store_vec<VEC, float>(a.part_w + (int64_t)range * a.ldp + col, acc_w);
  if (a.part_post) store_vec<VEC, float>(a.part_post + (int64_t)range * a.ldp + col, acc_p);
}

// Joins partial sums in a fixed order, 128 columns to a block.  blockIdx.y: the sums of dw, those of dw_post, then rows of the gate
// that lie in several ranges: by their number, or where the gate has more rows than there are borders between ranges by the
// first border that they cross.  A sum is taken by the block's warps side by side, or, rows of a gate that has many and so few
// parts to each, by one.
constexpr int kJoinWarps = 32;
struct JoinArgs {
  int width, ldp, blocks;
  int rows, ranges, group, by_border, gate_jobs, split;  // split: a row of the gate is a block's
  const float *part_w, *part_post, *part_gate;
  void *dw, *dp, *dgate;
  int w_f32, p_f32, g_f32;
  int64_t ld_dg;
};
template <typename T>
__global__ void __launch_bounds__(32 * kJoinWarps) block_join_kernel(const JoinArgs a) {
  __shared__ float4 sum[kJoinWarps][32];
  dep_wait();
  dep_launch();
  const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 128 + 4 * lane;
  int job = blockIdx.y;
  const float* from = nullptr;
  const float* head = nullptr;  // the first part, where it is not the one before `from`
  void* to = nullptr;
  int64_t at = 0, step = a.ldp;
  int n = a.blocks, f32 = 0;
  bool split = true;
  if (a.part_w && job-- == 0) {
    from = a.part_w, to = a.dw, f32 = a.w_f32;
  } else if (a.part_post && job-- == 0) {
    from = a.part_post, to = a.dp, f32 = a.p_f32;
  } else {
    split = a.split;
    if (!split) job = kJoinWarps * job + y;
    if (job >= a.gate_jobs) return;
    int64_t g = job;
    if (a.by_border) {
      const int start = range_start(job + 1, a.rows, a.ranges);
      g = start / a.group;
      if (g * a.group == start || g * a.group < range_start(job, a.rows, a.ranges)) return;  // crosses none here, or one before
    }
    const int b0 = range_of(g * a.group, a.rows, a.ranges), b1 = range_of((g + 1) * a.group - 1, a.rows, a.ranges);
    if (b0 == b1) return;
    head = a.part_gate + ((int64_t)2 * b0 + (g * a.group > range_start(b0, a.rows, a.ranges) ? 1 : 0)) * a.ldp;
    from = a.part_gate + (int64_t)2 * (b0 + 1) * a.ldp, step = 2 * (int64_t)a.ldp, n = b1 - b0;
    to = a.dgate, f32 = a.g_f32, at = g * a.ld_dg;
  }
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < a.width) {
    const int mine = split ? y : 0, stride = split ? kJoinWarps : 1;
    if (head && mine == 0) s = *reinterpret_cast<const float4*>(head + col);
#pragma unroll 8
    for (int i = mine; i < n; i += stride) {
      const float4 v = *reinterpret_cast<const float4*>(from + i * step + col);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
  }
  if (split) {  // for all of the block
    sum[y][lane] = s;
    __syncthreads();
    if (y) return;
#pragma unroll
    for (int i = 1; i < kJoinWarps; ++i) {
      const float4 v = sum[i][lane];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
  }
  const float out[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < a.width) put_value<T>(to, at + col + e, out[e], f32);
}

// How the gradient's rows are cut: threads to a row, blocks, ranges, stages.
struct GradPlan {
  int threads, blocks, ranges, stages, pitch, stage_bytes, ring_gate;
  size_t smem;
};
// ring_gate: bytes of an element of a gate that is brought with every row, or 0.
GradPlan plan_grad(const asd_ops* o, int rows, int width, int es, bool vec, int ring_gate) {
  GradPlan p{};
  if (width <= kNarrowWidth) {
    const int lanes = width <= 64 ? 8 : width <= 128 ? 16 : 32, slots = kNarrowBlock / lanes;
    p.ranges = (int)std::min<int64_t>(rows, (int64_t)6 * o->num_sms * slots);
    p.blocks = (p.ranges + slots - 1) / slots;
    return p;
  }
  if (width > kMostGradWidth) {
    p.ranges = p.blocks = (int)std::min<int64_t>(rows, std::max(1, 6 * o->num_sms / ((width + 1023) / 1024)));
    return p;
  }
  p.threads = walk_threads(width);
  // the ranges have to be the same however the rows can be read, so that the workspace is: 32 bytes more for a staged part
  const int most = 4 * walk_pitch(width, es, false);
  const int sums = p.threads * kWalkPer * 4;
  auto room = [&](int side, int bytes) { return (walk_room(side, grad_declared(p.threads)) - sums) / bytes; };  // rows beside the sums
  int side = grad_side(p.threads);
  while (side > 1 && room(side, most) < 2) side /= 2;
  p.ranges = p.blocks = std::min(rows, side * o->num_sms);
  p.pitch = walk_pitch(width, es, vec);
  p.ring_gate = ring_gate && room(side, 4 * p.pitch + width * ring_gate) > 1;  // the gate is read after its row
  p.stage_bytes = 4 * p.pitch + (p.ring_gate ? width * ring_gate : 0);
  p.stages = std::max(1, std::min(vec ? kMostStages : 2, room(side, p.stage_bytes)));
  p.smem = (size_t)p.stages * p.stage_bytes + sums;
  return p;
}
bool grad_vec(const asd_block_rmsnorm_backward_args* a) {
  const int es = ops_type_size(a->type);
  return a->width % 8 == 0 && aligned(a->dy, a->ld_dy, es, 16) && (!a->ds || aligned(a->ds, a->ld_ds, es, 16)) && aligned(a->x, a->ld_x, es, 16) &&
         aligned(a->s, a->ld_s, es, 16) && aligned(a->weight, 0, 1, 16) && aligned(a->post_weight, 0, 1, 16) &&
         aligned(a->gate, a->gate ? a->ld_gate : 0, ops_type_size(a->gate_type), 16) && (!a->dx || aligned(a->dx, a->ld_dx, es, 16)) &&
         (!a->dresidual || aligned(a->dresidual, a->ld_dresidual, es, 16));
}
// The partial sums of a call, one after the other; with a NULL base their bytes.
struct GradSpace {
  float *w, *post, *gate, *stats;
  int64_t bytes;
};
GradSpace grad_space(const GradPlan& p, const asd_block_rmsnorm_backward_args* a) {
  GradSpace g{};
  float* at = (float*)a->workspace;
  const int64_t ldp = (a->width + 3) / 4 * 4;
  auto take = [&](int64_t n) {
    float* q = at ? at + g.bytes / 4 : nullptr;
    g.bytes += n * 4;
    return q;
  };
  if (a->dweight) g.w = take(p.blocks * ldp);
  if (a->dpost_weight) g.post = take(p.blocks * ldp);
  if (a->dgate) g.gate = take(2 * p.ranges * ldp);
  if (a->width > kMostGradWidth && (a->dweight || a->dpost_weight || a->dgate)) g.stats = take((int64_t)a->rows * 4);
  return g;
}

template <typename T, int VEC>
void grad_t(const BlockGradArgs& n, const GradPlan& p, cudaStream_t st) {
  if (n.width <= kNarrowWidth) {
    with_lanes(n.width, [&](auto lanes) {
      ops_launch(narrow_block_grad_kernel<T, VEC, decltype(lanes)::value>, dim3(p.blocks), dim3(kNarrowBlock), 0, st, 1, n);
    });
  } else if (n.width > kMostGradWidth) {
    ops_launch(block_grad_long_kernel<T, VEC>, dim3(n.rows), dim3(kLongBlock), 0, st, 1, n);
    if (n.stats) ops_launch(block_columns_kernel<T, VEC>, dim3((n.width + 128 * VEC - 1) / (128 * VEC), p.ranges), dim3(128), 0, st, 1, n);
  } else {
    void (*kernel)(BlockGradArgs) = p.threads == 64    ? block_grad_kernel<T, VEC, 64>
                                    : p.threads == 128 ? block_grad_kernel<T, VEC, 128>
                                    : p.threads == 256 ? block_grad_kernel<T, VEC, 256>
                                                       : block_grad_kernel<T, VEC, 512>;
    ops_launch(kernel, dim3(p.blocks), dim3(p.threads), p.smem, st, 1, n);
  }
}

template <typename K>
cudaError_t allow_smem(K* kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <typename T, int VEC>
cudaError_t prepare_block() {
  for (cudaError_t e :
       {allow_smem(block_walk_kernel<T, VEC, 64, false>, kWalkSmem), allow_smem(block_walk_kernel<T, VEC, 64, true>, kWalkSmem),
        allow_smem(block_walk_kernel<T, VEC, 128, false>, kWalkSmem), allow_smem(block_walk_kernel<T, VEC, 128, true>, kWalkSmem),
        allow_smem(block_walk_kernel<T, VEC, 256, false>, kWalkSmem), allow_smem(block_walk_kernel<T, VEC, 256, true>, kWalkSmem),
        allow_smem(block_walk_kernel<T, VEC, 512, false>, kWalkSmem), allow_smem(block_walk_kernel<T, VEC, 512, true>, kWalkSmem),
        allow_smem(block_walk_kernel<T, VEC, 1024, false>, kWalkSmem), allow_smem(block_walk_kernel<T, VEC, 1024, true>, kWalkSmem),
        allow_smem(block_grad_kernel<T, VEC, 64>, kWalkSmem), allow_smem(block_grad_kernel<T, VEC, 128>, kWalkSmem),
        allow_smem(block_grad_kernel<T, VEC, 256>, kWalkSmem), allow_smem(block_grad_kernel<T, VEC, 512>, kWalkSmem)})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}

}  // namespace

asd_status ops_block_prepare() {
  for (cudaError_t e : {prepare_block<float, 8>(), prepare_block<__half, 8>(), prepare_block<__nv_bfloat16, 8>(), prepare_block<float, 1>(),
                        prepare_block<__half, 1>(), prepare_block<__nv_bfloat16, 1>()})
    if (e != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  return ASD_OK;
}

void launch_block_rmsnorm(const asd_ops* o, const asd_block_rmsnorm_args* a, cudaStream_t st) {
  BlockArgs n{};
  n.rows = a->rows, n.width = a->width, n.group = a->gate ? a->group : a->rows, n.post = a->post_norm;
  n.w_f32 = a->w_type == ASD_TYPE_F32, n.p_f32 = a->post_type == ASD_TYPE_F32, n.g_f32 = a->gate_type == ASD_TYPE_F32;
  n.eps = a->eps, n.alpha = a->alpha;
  n.x = a->x, n.r = a->residual, n.w = a->weight, n.wp = a->post_weight, n.gate = a->gate, n.s = a->s, n.y = a->y, n.scale = a->scale;
  n.ld_x = a->ld_x, n.ld_r = a->ld_residual, n.ld_g = a->ld_gate, n.ld_s = a->ld_s, n.ld_y = a->ld_y;
  const int es = ops_type_size(a->type);
  const bool q8 = a->scale != nullptr;
  const bool vec = a->width % 8 == 0 && aligned(a->x, a->ld_x, es, 16) && aligned(a->residual, a->ld_residual, es, 16) && aligned(a->weight, 0, 1, 16) &&
                   aligned(a->post_weight, 0, 1, 16) && aligned(a->gate, a->gate ? a->ld_gate : 0, ops_type_size(a->gate_type), 16) &&
                   aligned(a->s, a->ld_s, es, 16) && (q8 ? aligned(a->y, a->ld_y, 1, 8) : aligned(a->y, a->ld_y, es, 16));
  if (a->type == ASD_TYPE_F32)
    q8 ? block_t<float, true>(o, n, vec, st) : block_t<float, false>(o, n, vec, st);
  else if (a->type == ASD_TYPE_F16)
    q8 ? block_t<__half, true>(o, n, vec, st) : block_t<__half, false>(o, n, vec, st);
  else
    q8 ? block_t<__nv_bfloat16, true>(o, n, vec, st) : block_t<__nv_bfloat16, false>(o, n, vec, st);
}

// The same plan whether the rows can be read in 16-byte pieces or not, but for shared memory.
int64_t block_rmsnorm_backward_bytes(const asd_ops* o, const asd_block_rmsnorm_backward_args* a) {
  if (a->rows == 0) return 0;
  return grad_space(plan_grad(o, a->rows, a->width, ops_type_size(a->type), false, 0), a).bytes;
}

void launch_block_rmsnorm_backward(const asd_ops* o, const asd_block_rmsnorm_backward_args* a, cudaStream_t st) {
  const int es = ops_type_size(a->type);
  const bool vec = grad_vec(a);
  const bool ring_gate = vec && a->gate && a->group == 1;
  const GradPlan p = plan_grad(o, a->rows, a->width, es, vec, ring_gate ? ops_type_size(a->gate_type) : 0);
  const GradSpace space = grad_space(p, a);
  BlockGradArgs n{};
  n.rows = a->rows, n.width = a->width, n.group = a->gate ? a->group : a->rows, n.post = a->post_norm, n.ranges = p.ranges;
  n.w_f32 = a->w_type == ASD_TYPE_F32, n.p_f32 = a->post_type == ASD_TYPE_F32, n.g_f32 = a->gate_type == ASD_TYPE_F32;
  n.stages = p.stages, n.pitch = p.pitch, n.stage_bytes = p.stage_bytes, n.ring_gate = p.ring_gate, n.err = o->err;
  n.ldp = (a->width + 3) / 4 * 4;
  n.eps = a->eps, n.alpha = a->alpha;
  n.dy = a->dy, n.ds = a->ds, n.x = a->x, n.s = a->s, n.w = a->weight, n.wp = a->post_weight, n.gate = a->gate;
  n.dx = a->dx, n.dr = a->dresidual, n.dgate = a->dgate;
  n.ld_dy = a->ld_dy, n.ld_ds = a->ld_ds, n.ld_x = a->ld_x, n.ld_s = a->ld_s, n.ld_g = a->ld_gate;
  n.ld_dx = a->ld_dx, n.ld_dr = a->ld_dresidual, n.ld_dg = a->ld_dgate;
  n.wide_dg = aligned(a->dgate, a->ld_dgate, es, 16);
  n.part_w = space.w, n.part_post = space.post, n.part_gate = space.gate, n.stats = space.stats;
  JoinArgs j{};
  j.width = a->width, j.ldp = n.ldp, j.blocks = p.blocks, j.rows = a->rows, j.ranges = p.ranges, j.group = n.group;
  j.part_w = space.w, j.part_post = space.post, j.part_gate = space.gate;
  j.dw = a->dweight, j.dp = a->dpost_weight, j.dgate = a->dgate, j.w_f32 = n.w_f32, j.p_f32 = n.p_f32, j.g_f32 = n.g_f32, j.ld_dg = a->ld_dgate;
  const int gates = a->rows / n.group;
  j.by_border = gates > p.ranges - 1;
  j.gate_jobs = space.gate ? std::min(gates, p.ranges - 1) : 0;
  j.split = j.gate_jobs <= 16;
  const int jobs = (space.w ? 1 : 0) + (space.post ? 1 : 0) + (j.split ? j.gate_jobs : (j.gate_jobs + kJoinWarps - 1) / kJoinWarps);
  const dim3 grid((a->width + 127) / 128, jobs);
  auto go = [&](auto zero) {
    using T = decltype(zero);
    vec ? grad_t<T, 8>(n, p, st) : grad_t<T, 1>(n, p, st);
    if (jobs) ops_launch(block_join_kernel<T>, grid, dim3(32 * kJoinWarps), 0, st, 1, j);
  };
  if (a->type == ASD_TYPE_F32)
    go(0.f);
  else if (a->type == ASD_TYPE_F16)
    go(__half());
  else
    go(__nv_bfloat16());
}

}  // namespace asd
