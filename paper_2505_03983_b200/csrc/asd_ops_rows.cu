// Operators that work on one row at a time: s = x + r with its root-mean-square norm (16 / 32 bits, or 8 bits with a scale
// per row), the norm's gradients, the row quantisation with or without the gate, and the copy that aligns an operand of a
// matrix product.
//
// All of them are bound by memory: a row is read once, kept in registers over its reductions, and written once.  A row
// belongs to 32, 128, 256 or 512 threads (rows of up to 1024, 4096, 8192, 16384), 32 elements to a thread, so that a thread has its
// 16-byte loads in flight together; longer rows are read a second time, and several narrow ones (up to 256) share a warp.
// Rows of more than 256 whose address, distance or length is not a multiple of 8 elements come into shared memory in the aligned
// 16-byte pieces that hold them, one row ahead, and are read from there element by element, neighbouring threads on neighbouring
// elements (read so from memory, 6001 rows of 2 x 2477 bf16 took 127 us to quantise).
//
// Measured (of 6.55 TB/s): norm 8192 x 4096 bf16 43 us = 6.2 TB/s, to int8 32768 x 1024 42.6 us = 5.5 TB/s, gradient 8192 x 4096 44 us =
// 6.1 TB/s, gate to int8 8192 x 8192 56.6 us = 5.9 TB/s with SiLU and 77 with GELU, whose instructions fill 79 % of
// the issue slots.  float32: norm 8192 x 4096 84 us = 6.4 TB/s, gradient 142 (3.8), rows to int8 without the gate 24, gate 8192 x 8192 90
// (6.7) and 93.  Rows of 16384, 4096 of them in bf16: norm 97, gradient 193 for dx, 118 for dw.  One row of 4096 takes 4 us, a kernel's start and end.
#include <type_traits>

#include "asd_ops_act.cuh"
#include "asd_ops_internal.h"

namespace asd {
namespace {

constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: the least magnitude that a row's scale is made from
constexpr int kPer = 32;                         // elements of a row that one thread keeps
constexpr int kStagedSmem = 220 * 1024;          // shared memory for staged rows

__device__ __forceinline__ void dep_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// VEC = 8 or 1 neighbouring elements; VEC = 8 asks for 16-byte aligned addresses (8 for int8).
template <int VEC, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    f[0] = to_f<T>(*p);
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_f<T>(e[i]);
  }
}
template <int VEC, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    *p = from_f<T>(f[0]);
  } else if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    uint4 v;
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = from_f<T>(f[i]);
    *reinterpret_cast<uint4*>(p) = v;
  }
}
// q = rint(f inv), |f inv| <= 127.  Adding 1.5 2^23 rounds to the nearest even integer and leaves it, as two's complement, in
// the low bits of the sum: three byte selections pack four of them, where conversions would take one slow instruction each.
__device__ __forceinline__ uint32_t rounded_bits(float f, float inv) { return __float_as_uint(fmaf(f, inv, 12582912.f)); }
template <int VEC>
__device__ __forceinline__ void store_q(int8_t* p, const float (&f)[VEC], float inv) {
  if constexpr (VEC == 1) {
    *p = (int8_t)rounded_bits(f[0], inv);
  } else {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[h] = __byte_perm(__byte_perm(rounded_bits(f[4 * h], inv), rounded_bits(f[4 * h + 1], inv), 0x0040),
                         __byte_perm(rounded_bits(f[4 * h + 2], inv), rounded_bits(f[4 * h + 3], inv), 0x0040), 0x5410);
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}
template <int VEC>
__device__ __forceinline__ void store_zero(int8_t* p) {
  if constexpr (VEC == 1)
    *p = 0;
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(0u, 0u);
}
template <int VEC, typename T>
__device__ __forceinline__ void load_weight(const void* w, int w_f32, int col, float (&f)[VEC]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = 1.f;
  } else if (w_f32) {
    load_vec<VEC, float>(reinterpret_cast<const float*>(w) + col, f);
  } else {
    load_vec<VEC, T>(reinterpret_cast<const T*>(w) + col, f);
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Sum and largest over the threads of a row (a warp, or the block).  `buf`: one word per warp; a block's call ends with
// the buffer free for the next one after another barrier, so alternate two buffers.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* buf) {
  v = warp_sum(v);
  if (TPR == 32) return v;
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < TPR / 32; ++i) t += buf[i];
  return t;
}
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* buf) {
  v = __reduce_max_sync(0xffffffffu, v);
  if (TPR == 32) return v;
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
  __syncthreads();
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < TPR / 32; ++i) t = max(t, buf[i]);
  return t;
}
// Magnitudes are compared as their bit patterns: the order of the numbers, with infinity above all of them and NaN above
// infinity, so that one maximum also tells whether the row can be represented.
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }
struct RowScale {
  float inv, scale;  // q = rint(y inv), y ~ q scale
  bool ok;           // false: the row has a NaN or an infinity; q = 0
};
__device__ __forceinline__ RowScale row_scale(uint32_t most) {
  if (most >= 0x7f800000u) return {0.f, __uint_as_float(0x7fffffffu), false};
  const float m = fmaxf(__uint_as_float(most), kTiny);
  return {127.f / m, m / 127.f, true};
}
template <int VEC>
__device__ __forceinline__ void put_q(int8_t* p, const float (&f)[VEC], const RowScale& rs) {
  if (rs.ok)
    store_q<VEC>(p, f, rs.inv);
  else
    store_zero<VEC>(p);
}

// The exponential and the reciprocal are the approximate instructions (relative error some 2^-22).
__device__ __forceinline__ float act_value(float g, int act) {
  if (act == ASD_ACT_SILU) {
    float e, p;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(1.f + e));
    return g * p;
  }
  return g * normal_cdf(g).x;
}

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 pa, pb, pc;\n\tmov.b64 pa, {%2, %3};\n\tmov.b64 pb, {%4, %5};\n\tmul.rn.f32x2 pc, pa, pb;\n\tmov.b64 {%0, %1}, pc;\n\t}"
      : "=f"(c.x), "=f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 pa, pb, pc, pd;\n\tmov.b64 pa, {%2, %3};\n\tmov.b64 pb, {%4, %5};\n\tmov.b64 pc, {%6, %7};\n\t"
      "fma.rn.f32x2 pd, pa, pb, pc;\n\tmov.b64 {%0, %1}, pd;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
// Pair i of elements that are held as they are stored.
template <typename T>
__device__ __forceinline__ float2 unpack(const uint32_t* e, int i) {
  if constexpr (sizeof(T) == 4)
    return make_float2(__uint_as_float(e[2 * i]), __uint_as_float(e[2 * i + 1]));
  else if constexpr (std::is_same<T, __nv_bfloat16>::value)
    return make_float2(__uint_as_float(e[i] << 16), __uint_as_float(e[i] & 0xffff0000u));
  else
    return __half22float2(*reinterpret_cast<const __half2*>(e + i));
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 pa, pb, pc;\n\tmov.b64 pa, {%2, %3};\n\tmov.b64 pb, {%4, %5};\n\tadd.rn.f32x2 pc, pa, pb;\n\tmov.b64 {%0, %1}, pc;\n\t}"
      : "=f"(c.x), "=f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}

struct NormArgs {
  int rows, width, w_f32;
  float eps;
  const void *x, *r, *w;
  void *sum, *y;
  float* scale;
  int64_t ld_x, ld_r, ld_s, ld_y;
};

// Threads of a block: the row's, or four rows of a warp each.
template <int TPR>
constexpr int block_of = TPR == 32 ? 128 : TPR;

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// A row of `bytes` into shared memory by T threads, in aligned pieces; it starts (address & 15) bytes into dst.  Nothing
// beyond the row's end is read.  The piece that holds its start begins in the row before; where there is none (`top`) one
// thread copies what there is of it.
__device__ __forceinline__ void stage_row(uint8_t* dst, const void* src, int bytes, int t, int T, bool top) {
  const int off = (int)((uintptr_t)src & 15), end = bytes + off;
  const uint8_t* p = reinterpret_cast<const uint8_t*>(src) - off;
  for (int at = 16 * t; at < end; at += 16 * T) {
    if (at == 0 && top && off) {
      for (int i = off; i < min(16, end); i += 2) *reinterpret_cast<uint16_t*>(dst + i) = *reinterpret_cast<const uint16_t*>(p + i);
    } else {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + at)), "l"(p + at), "r"(min(16, end - at))
                   : "memory");
    }
  }
}
template <typename T>
__device__ __forceinline__ const T* staged(const uint8_t* dst, const void* src) {
  return reinterpret_cast<const T*>(dst + ((uintptr_t)src & 15));
}
__host__ __device__ inline int stage_pitch(int64_t bytes) { return (int)((bytes + 15 + 15) / 16 * 16); }
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}
// The threads of a row.
template <int TPR>
__device__ __forceinline__ void row_sync() {
  if (TPR == 32)
    __syncwarp();
  else
    __syncthreads();
}
// How rows that are staged are walked over: `stride` rows side by side, each with `ahead` + 1 buffers of `pitch` bytes for each
// of its `parts`.
struct Walk {
  int stride, ahead, pitch, parts;
};
// Calls work(row, turn) for each of a row slot's rows with the row in the buffers of `turn`; fetch(row, turn) copies one.  The
// work has to read its buffers before a barrier of the row's threads that it takes itself.
template <int TPR, typename F, typename W>
__device__ __forceinline__ void walk_rows(int first, int rows, const Walk& k, F fetch, W work) {
  if (k.ahead) {
    if (first < rows) fetch(first, 0);
    commit_copies();
  }
  int turn = 0;
  for (int64_t row = first; row < rows; row += k.stride) {
    if (k.ahead) {
      if (row + k.stride < rows) fetch((int)(row + k.stride), turn ^ 1);
      commit_copies();
      wait_copies<1>();
    } else {
      fetch((int)row, 0);
      commit_copies();
      wait_copies<0>();
    }
    row_sync<TPR>();  // every thread's copies are in place
    work((int)row, turn);
    turn ^= k.ahead;
  }
}

// s and its norm for staged rows.
template <typename T, int TPR, bool Q8>
__global__ void __launch_bounds__(block_of<TPR>) rmsnorm_staged_kernel(const NormArgs a, const Walk k) {
  extern __shared__ __align__(16) uint8_t rows_smem[];
  __shared__ float buf_s[2][TPR / 32];
  __shared__ uint32_t buf_m[2][TPR / 32];
  dep_wait();
  dep_launch();
  const int t = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x, slot = TPR == 32 ? threadIdx.x >> 5 : 0;
  uint8_t* mine = rows_smem + slot * (k.ahead + 1) * k.parts * k.pitch;
  auto buffer = [&](int turn, int part) { return mine + (turn * k.parts + part) * k.pitch; };
  auto xrow = [&](int row) { return reinterpret_cast<const T*>(a.x) + row * a.ld_x; };
  auto rrow = [&](int row) { return reinterpret_cast<const T*>(a.r) + row * a.ld_r; };
  const int n = (a.width - t + TPR - 1) / TPR;  // this thread's elements t, t + TPR, ...
  int side = 0;
  walk_rows<TPR>(
      TPR == 32 ? blockIdx.x * 4 + slot : blockIdx.x, a.rows, k,
      [&](int row, int turn) {
        stage_row(buffer(turn, 0), xrow(row), a.width * (int)sizeof(T), t, TPR, row == 0);
        if (a.r) stage_row(buffer(turn, 1), rrow(row), a.width * (int)sizeof(T), t, TPR, row == 0);
      },
      [&](int row, int turn) {
        const T* x = staged<T>(buffer(turn, 0), xrow(row)) + t;
        const T* r = a.r ? staged<T>(buffer(turn, 1), rrow(row)) + t : nullptr;
        T* so = a.sum ? reinterpret_cast<T*>(a.sum) + row * a.ld_s + t : nullptr;
        float f[kPer], sq = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          f[i] = 0.f;
          if (i < n) {
            T v = x[i * TPR];
            if (r) v = from_f<T>(to_f<T>(v) + to_f<T>(r[i * TPR]));
            if (so) so[i * TPR] = v;
            f[i] = to_f<T>(v);
            sq = fmaf(f[i], f[i], sq);
          }
        }
        sq = row_sum<TPR>(sq, buf_s[side]);
        const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
        uint32_t most = 0;
        T* y = reinterpret_cast<T*>(a.y) + row * a.ld_y + t;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (i < n) {
            float w[1];
            load_weight<1, T>(a.w, a.w_f32, t + i * TPR, w);
            f[i] = f[i] * rho * w[0];
            if (Q8)
              most = max(most, mag(f[i]));
            else
              y[i * TPR] = from_f<T>(f[i]);
          }
        }
        if (Q8) {
          const RowScale rs = row_scale(row_max<TPR>(most, buf_m[side]));
          int8_t* q = reinterpret_cast<int8_t*>(a.y) + row * a.ld_y + t;
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (i < n) q[i * TPR] = rs.ok ? (int8_t)rounded_bits(f[i], rs.inv) : (int8_t)0;
          if (t == 0) a.scale[row] = rs.scale;
        }
        side ^= 1;
      });
}

// s and its norm.  TPR threads to a row, kPer elements each (LONG: any number, s read back or added up again for the
// second pass).
template <typename T, int VEC, int TPR, bool Q8, bool LONG>
__global__ void __launch_bounds__(block_of<TPR>) rmsnorm_kernel(const NormArgs a) {
  constexpr int NV = kPer / VEC;
  __shared__ float buf_s[TPR / 32];
  __shared__ uint32_t buf_m[TPR / 32];
  dep_wait();
  dep_launch();
  const int t = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x;
  const int row = TPR == 32 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= a.rows) return;  // whole warps: rows of a block do not share a barrier
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
  const T* r = a.r ? reinterpret_cast<const T*>(a.r) + row * a.ld_r : nullptr;
  T* so = a.sum ? reinterpret_cast<T*>(a.sum) + row * a.ld_s : nullptr;
  auto fetch = [&](int col, float(&f)[VEC]) {  // the rounded s
    load_vec<VEC, T>(x + col, f);
    if (r) {
      float g[VEC];
      load_vec<VEC, T>(r + col, g);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = to_f<T>(from_f<T>(f[i] + g[i]));
    }
  };
  if constexpr (!LONG) {
    float f[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width)
        fetch(col, f[v]);
      else
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[v][i] = 0.f;
    }
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (so && col < a.width) store_vec<VEC, T>(so + col, f[v]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sq = fmaf(f[v][i], f[v][i], sq);
    }
    sq = row_sum<TPR>(sq, buf_s);
    const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
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
    for (int col = t * VEC; col < a.width; col += TPR * VEC) {
      float f[VEC];
      fetch(col, f);
      if (so) store_vec<VEC, T>(so + col, f);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sq = fmaf(f[i], f[i], sq);
    }
    sq = row_sum<TPR>(sq, buf_s);
    const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
    // s once more: from where this thread has stored it (x or r may be gone by now), or added up again
    auto again = [&](int col, float(&f)[VEC]) {
      if (so)
        load_vec<VEC, T>(so + col, f);
      else
        fetch(col, f);
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

// act(g) u for two elements: the same operations as act_value's.
__device__ __forceinline__ float2 gated2(float2 g, float2 u, int act) {
  float2 a;
  if (act == ASD_ACT_SILU) {
    const float2 x = mul2(g, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    float2 e, p;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(x.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(x.y));
    e = add2(e, make_float2(1.f, 1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p.y) : "f"(e.y));
    a = mul2(g, p);
  } else {
    a = make_float2(act_value(g.x, act), act_value(g.y, act));
  }
  return mul2(a, u);
}

struct QuantArgs {
  int rows, width, act, stride;  // stride: rows that are worked on side by side
  const void* x;
  int8_t* q;
  float* scale;
  int64_t ld_x, ld_q;
};

// A row's threads walk over rows.  With the gate, 16-bit rows that can be read in 16-byte pieces come through shared memory
// one row ahead (cp.async; a thread reads back only what it has copied itself, so that takes no barrier): two transcendental
// instructions an element and the barrier of the row's maximum would leave memory idle otherwise.
template <typename T, int VEC>
constexpr bool row_ahead = VEC == 8 && sizeof(T) == 2;
template <typename T, int VEC, int TPR>
constexpr int quantize_smem = row_ahead<T, VEC> ? 2 * 2 * kPer * 2 * block_of<TPR> : 0;

template <typename T, int VEC, int TPR>
__global__ void __launch_bounds__(block_of<TPR>) quantize_kernel(const QuantArgs a) {
  constexpr int NV = kPer / VEC;
  constexpr bool AHEAD = row_ahead<T, VEC>;
  extern __shared__ __align__(16) uint4 ahead[];  // [2 rows][g, u][NV][threads]
  __shared__ uint32_t buf_m[2][TPR / 32];
  dep_wait();
  dep_launch();
  const int t = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x;
  const int first = TPR == 32 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  const bool gate = a.act != ASD_ACT_NONE;
  auto slot = [&](int turn, int part, int v) { return ahead + ((turn * 2 + part) * NV + v) * block_of<TPR> + threadIdx.x; };
  auto fetch = [&](int64_t row, int turn) {
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width) {
        copy_16((uint32_t)__cvta_generic_to_shared(slot(turn, 0, v)), x + col);
        if (gate) copy_16((uint32_t)__cvta_generic_to_shared(slot(turn, 1, v)), x + a.width + col);
      }
    }
  };
  if (AHEAD) {
    if (first < a.rows) fetch(first, 0);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int turn = 0;
  for (int64_t row = first; row < a.rows; row += a.stride, turn ^= 1) {
    if (AHEAD) {
      if (row + a.stride < a.rows) fetch(row + a.stride, turn ^ 1);
      asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
    }
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
    float f[NV][VEC];
    uint32_t most = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width) {
        if constexpr (AHEAD) {
          uint32_t g[4], u[4];
          *reinterpret_cast<uint4*>(g) = *slot(turn, 0, v);
          if (gate) *reinterpret_cast<uint4*>(u) = *slot(turn, 1, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2 h = unpack<T>(g, i);
            if (gate) h = gated2(h, unpack<T>(u, i), a.act);
            f[v][2 * i] = h.x;
            f[v][2 * i + 1] = h.y;
          }
        } else {
          load_vec<VEC, T>(x + col, f[v]);
          if (gate) {
            float u[VEC];
            load_vec<VEC, T>(x + a.width + col, u);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[v][i] = act_value(f[v][i], a.act) * u[i];
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) most = max(most, mag(f[v][i]));
      }
    }
    const RowScale rs = row_scale(row_max<TPR>(most, buf_m[turn]));
    int8_t* q = a.q + row * a.ld_q;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = (v * TPR + t) * VEC;
      if (col < a.width) put_q<VEC>(q + col, f[v], rs);
    }
    if (t == 0) a.scale[row] = rs.scale;
  }
}

// The same for staged rows.
template <typename T, int TPR>
__global__ void __launch_bounds__(block_of<TPR>) quantize_staged_kernel(const QuantArgs a, const Walk k) {
  extern __shared__ __align__(16) uint8_t rows_smem[];
  __shared__ uint32_t buf_m[2][TPR / 32];
  dep_wait();
  dep_launch();
  const int t = TPR == 32 ? (threadIdx.x & 31) : threadIdx.x, slot = TPR == 32 ? threadIdx.x >> 5 : 0;
  uint8_t* mine = rows_smem + slot * (k.ahead + 1) * k.pitch;
  const bool gate = a.act != ASD_ACT_NONE;
  auto xrow = [&](int row) { return reinterpret_cast<const T*>(a.x) + row * a.ld_x; };
  const int n = (a.width - t + TPR - 1) / TPR;
  int side = 0;
  walk_rows<TPR>(
      TPR == 32 ? blockIdx.x * 4 + slot : blockIdx.x, a.rows, k,
      [&](int row, int turn) { stage_row(mine + turn * k.pitch, xrow(row), (gate ? 2 : 1) * a.width * (int)sizeof(T), t, TPR, row == 0); },
      [&](int row, int turn) {
        const T* x = staged<T>(mine + turn * k.pitch, xrow(row)) + t;
        float f[kPer];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
          float2 g = make_float2(0.f, 0.f), u = g;
          if (i < n) g.x = to_f<T>(x[i * TPR]);
          if (i + 1 < n) g.y = to_f<T>(x[(i + 1) * TPR]);
          if (gate) {
            if (i < n) u.x = to_f<T>(x[a.width + i * TPR]);
            if (i + 1 < n) u.y = to_f<T>(x[a.width + (i + 1) * TPR]);
            g = gated2(g, u, a.act);
          }
          f[i] = g.x;
          f[i + 1] = g.y;
          most = max(most, max(mag(g.x), mag(g.y)));
        }
        const RowScale rs = row_scale(row_max<TPR>(most, buf_m[side]));
        int8_t* q = a.q + row * a.ld_q + t;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (i < n) q[i * TPR] = rs.ok ? (int8_t)rounded_bits(f[i], rs.inv) : (int8_t)0;
        if (t == 0) a.scale[row] = rs.scale;
        side ^= 1;
      });
}

// Rows of more than 16384, read twice.
template <typename T, int VEC>
__global__ void __launch_bounds__(512) quantize_long_kernel(const QuantArgs a) {
  __shared__ uint32_t buf_m[16];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
  int8_t* q = a.q + row * a.ld_q;
  auto fetch = [&](int col, float(&f)[VEC]) {
    load_vec<VEC, T>(x + col, f);
    if (a.act != ASD_ACT_NONE) {
      float u[VEC];
      load_vec<VEC, T>(x + a.width + col, u);
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = act_value(f[i], a.act) * u[i];
    }
  };
  uint32_t most = 0;
  for (int col = t * VEC; col < a.width; col += 512 * VEC) {
    float f[VEC];
    fetch(col, f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) most = max(most, mag(f[i]));
  }
  const RowScale rs = row_scale(row_max<512>(most, buf_m));
  for (int col = t * VEC; col < a.width; col += 512 * VEC) {
    float f[VEC];
    fetch(col, f);
    put_q<VEC>(q + col, f, rs);
  }
  if (t == 0) a.scale[row] = rs.scale;
}

struct NormGradArgs {
  int rows, width, w_f32, blocks;
  int pitch;    // of a staged row
  float eps;
  const void *dy, *s, *ds, *w;
  void* dx;     // or NULL
  float* part;  // [blocks, width] sums of dy z over a block's rows, or NULL
  float* rho;   // LONG: [rows]
  int64_t ld_dy, ld_s, ld_ds, ld_dx;
};

// Gradients.  One block walks over rows blockIdx.x, + blocks, ...; a thread keeps the same columns in every row, so the
// weights and the sums of dw over the block's rows stay in its registers; the sums are written once, to be added up by
// reduce_dw_kernel.  Both sums of a row, of s^2 and of dy w s, are taken together: mean(dy w z) = rho mean(dy w s).  Rows come
// through shared memory two rows ahead (32 bits: one), so that memory is busy over the barriers: where they can be read in
// 16-byte pieces a thread reads back only what it has copied itself, the others are staged.
template <typename T>
constexpr int grad_ahead = sizeof(T) == 2 ? 2 : 1;
template <typename T, int VEC, int TPR, int PER>
constexpr int grad_smem = VEC == 8 ? (grad_ahead<T> + 1) * 3 * PER * (int)sizeof(T) * TPR : 0;

template <typename T, int VEC, int TPR, int PER>
__global__ void __launch_bounds__(TPR) rmsnorm_grad_kernel(const NormGradArgs a) {
  // elements come in groups of E: VEC neighbouring ones, or (VEC = 1) two that are TPR apart
  constexpr int E = VEC == 1 ? 2 : VEC, NV = PER / E, NP = E / 2;  // NP: pairs; every product and sum is a two-way fp32 instruction
  constexpr bool AHEAD = VEC == 8;
  constexpr int kGradAhead = grad_ahead<T>;
  constexpr int PIECES = VEC * (int)sizeof(T) / 16;  // of 16 bytes to VEC elements
  extern __shared__ __align__(16) uint4 ahead[];      // [row][s, dy, ds][NV][pieces][threads]
  __shared__ float buf[2][2][TPR / 32];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x;
  auto column = [&](int v, int i) { return VEC == 1 ? (2 * v + i) * TPR + t : (v * TPR + t) * VEC + i; };
  float2 acc[NV][NP], w[NV][NP];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      float one[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float f[1];
        if (column(v, 2 * i + e) < a.width) {
          load_weight<1, T>(a.w, a.w_f32, column(v, 2 * i + e), f);
          one[e] = f[0];
        }
      }
      acc[v][i] = make_float2(0.f, 0.f);
      w[v][i] = make_float2(one[0], one[1]);
    }
  }
  const T* base[3] = {reinterpret_cast<const T*>(a.s), reinterpret_cast<const T*>(a.dy), reinterpret_cast<const T*>(a.ds)};
  const int64_t ld[3] = {a.ld_s, a.ld_dy, a.ld_ds};
  auto slot = [&](int turn, int part, int v, int piece) { return ahead + (((turn * 3 + part) * NV + v) * PIECES + piece) * TPR + t; };
  auto staged_at = [&](int turn, int part) { return reinterpret_cast<uint8_t*>(ahead) + (turn * 3 + part) * a.pitch; };
  auto fetch = [&](int64_t row, int turn) {
    if (!AHEAD && row < a.rows) {
      for (int part = 0; part < 3; ++part)
        if (part < 2 || a.ds) stage_row(staged_at(turn, part), base[part] + row * ld[part], a.width * (int)sizeof(T), t, TPR, row == 0);
    }
    if (AHEAD && row < a.rows) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = column(v, 0);
        if (col < a.width) {
#pragma unroll
          for (int part = 0; part < 3; ++part)
            if (part < 2 || a.ds) {
#pragma unroll
              for (int k = 0; k < PIECES; ++k)
                copy_16((uint32_t)__cvta_generic_to_shared(slot(turn, part, v, k)), base[part] + row * ld[part] + col + k * (16 / (int)sizeof(T)));
            }
        }
      }
    }
    commit_copies();
  };
  // VEC elements of s (0), dy (1) or ds (2) of the row that is worked on
  auto read = [&](int64_t row, int turn, int part, int v, int col, float2(&f)[NP]) {
    if constexpr (AHEAD) {
      uint32_t e[4 * PIECES];
#pragma unroll
      for (int k = 0; k < PIECES; ++k) reinterpret_cast<uint4*>(e)[k] = *slot(turn, part, v, k);
#pragma unroll
      for (int i = 0; i < NP; ++i) f[i] = unpack<T>(e, i);
    } else {
      const T* p = staged<T>(staged_at(turn, part), base[part] + row * ld[part]) + col;
      f[0] = make_float2(to_f<T>(p[0]), col + TPR < a.width ? to_f<T>(p[TPR]) : 0.f);
    }
  };
#pragma unroll
  for (int k = 0; k < kGradAhead; ++k) fetch(blockIdx.x + (int64_t)k * a.blocks, k);
  int turn = 0, side = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += a.blocks, side ^= 1) {
    const int64_t then = row + (int64_t)kGradAhead * a.blocks;
    const int free_turn = turn == 0 ? kGradAhead : turn - 1;
    if (AHEAD) {
      fetch(then, free_turn);
      wait_copies<kGradAhead>();
    } else {  // a thread reads what others have copied: all copies in place, and the row before no longer read
      wait_copies<kGradAhead - 1>();
      __syncthreads();
      fetch(then, free_turn);
    }
    float2 f[NV][NP], g[NV][NP], sq2 = make_float2(0.f, 0.f), dot2 = sq2;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = column(v, 0);
      if (col < a.width) {
        read(row, turn, 0, v, col, f[v]);
        read(row, turn, 1, v, col, g[v]);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          sq2 = fma2(f[v][i], f[v][i], sq2);
          dot2 = fma2(mul2(g[v][i], w[v][i]), f[v][i], dot2);
        }
      }
    }
    float sq = warp_sum(sq2.x + sq2.y), dot = warp_sum(dot2.x + dot2.y);
    if ((t & 31) == 0) {
      buf[side][0][t >> 5] = sq;
      buf[side][1][t >> 5] = dot;
    }
    __syncthreads();
    sq = dot = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) {
      sq += buf[side][0][i];
      dot += buf[side][1][i];
    }
    // dx = rho dy w - z (rho c) + ds with c = mean(dy w z) = rho dot / width; s times rho first: rho^2 c may leave the range of 32 bits
    const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
    const float k = -(rho * dot / (float)a.width) * rho;
    const float2 rho2 = make_float2(rho, rho), k2 = make_float2(k, k);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int col = column(v, 0);
      if (col < a.width) {
        float2 e[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) e[i] = make_float2(0.f, 0.f);
        if (a.ds) read(row, turn, 2, v, col, e);
        float d[2 * NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const float2 z = mul2(f[v][i], rho2);
          acc[v][i] = fma2(g[v][i], z, acc[v][i]);
          const float2 x = fma2(z, k2, fma2(mul2(g[v][i], w[v][i]), rho2, e[i]));
          d[2 * i] = x.x;
          d[2 * i + 1] = x.y;
        }
        if (a.dx) {
          T* p = reinterpret_cast<T*>(a.dx) + row * a.ld_dx + col;
          if constexpr (VEC == 1) {
            p[0] = from_f<T>(d[0]);
            if (col + TPR < a.width) p[TPR] = from_f<T>(d[1]);
          } else {
            store_vec<VEC, T>(p, d);
          }
        }
      }
    }
    if (++turn > kGradAhead) turn = 0;
  }
  if (a.part) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (column(v, i) < a.width) a.part[(size_t)blockIdx.x * a.width + column(v, i)] = i & 1 ? acc[v][i >> 1].y : acc[v][i >> 1].x;
  }
}

// Rows of more than 8192: dx row by row with rho kept per row, the sums of dw by columns afterwards.
template <typename T>
__global__ void __launch_bounds__(512) rmsnorm_grad_long_kernel(const NormGradArgs a) {
  __shared__ float buf[2][16];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.ld_dy;
  const T* s = reinterpret_cast<const T*>(a.s) + row * a.ld_s;
  float sq = 0.f, dot = 0.f, w[1], f[1], g[1];
  for (int col = t; col < a.width; col += 512) {
    load_vec<1, T>(s + col, f);
    load_vec<1, T>(dy + col, g);
    load_weight<1, T>(a.w, a.w_f32, col, w);
    sq = fmaf(f[0], f[0], sq);
    dot = fmaf(g[0] * w[0], f[0], dot);
  }
  sq = row_sum<512>(sq, buf[0]);
  dot = row_sum<512>(dot, buf[1]);
  const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
  const float c = rho * dot / (float)a.width;
  if (t == 0 && a.rho) a.rho[row] = rho;
  if (!a.dx) return;
  for (int col = t; col < a.width; col += 512) {
    load_vec<1, T>(s + col, f);
    load_vec<1, T>(dy + col, g);
    load_weight<1, T>(a.w, a.w_f32, col, w);
    float d = rho * (g[0] * w[0] - f[0] * rho * c);
    if (a.ds) d += to_f<T>(reinterpret_cast<const T*>(a.ds)[row * a.ld_ds + col]);
    reinterpret_cast<T*>(a.dx)[row * a.ld_dx + col] = from_f<T>(d);
  }
}
template <typename T>
__global__ void __launch_bounds__(128) columns_dw_kernel(const NormGradArgs a) {
  dep_wait();
  dep_launch();
  const int col = blockIdx.x * 128 + threadIdx.x;
  if (col >= a.width) return;
  float acc = 0.f;
  for (int64_t row = blockIdx.y; row < a.rows; row += a.blocks)
    acc = fmaf(to_f<T>(reinterpret_cast<const T*>(a.dy)[row * a.ld_dy + col]),
               to_f<T>(reinterpret_cast<const T*>(a.s)[row * a.ld_s + col]) * a.rho[row], acc);
  a.part[(size_t)blockIdx.y * a.width + col] = acc;
}

// dw[col] = sum over blocks of part[block, col], in a fixed order: 32 columns to a block, 32 threads to a column.
template <typename W>
__global__ void __launch_bounds__(1024) reduce_dw_kernel(const float* part, int blocks, int width, W* dw) {
  __shared__ float buf[32][33];
  dep_wait();
  dep_launch();
  const int col = blockIdx.x * 32 + threadIdx.x;
  float acc = 0.f;
  if (col < width) {
#pragma unroll 8
    for (int b = threadIdx.y; b < blocks; b += 32) acc += part[(size_t)b * width + col];
  }
  buf[threadIdx.y][threadIdx.x] = acc;
  __syncthreads();
  const float v = warp_sum(buf[threadIdx.x][threadIdx.y]);
  if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < width) dw[blockIdx.x * 32 + threadIdx.y] = from_f<W>(v);
}

// ---- narrow rows: up to 256 elements ----
// A row belongs to L = 8, 16 or 32 lanes with kNarrow elements each, so that a warp works on 32 / L rows at once and its sums
// are a few shuffles.  Lane `t` has the elements 8 t .. 8 t + 7 of rows in 16-byte pieces (VEC = 8), or t, t + L, ... of any
// others (VEC = 1), which neighbouring lanes read from the same sectors.
// Measured in bf16, with a warp to a row and 32 elements to a lane in brackets (a row of 64 then costs the instructions of
// one of 1024): 1048576 x 64 norm 89 us (391), to int8 107 (473), gradient 97 (824), to int8 without the norm 47 (231); these move
// 537, 470, 537 and 206 MB.  131072 x 100, rows that do not start on 16 bytes: 27 (115), 36 (188), 43 (171), 19 (84).
constexpr int kNarrow = 8;
constexpr int kNarrowWidth = 32 * kNarrow;
constexpr int kNarrowBlock = 128;       // of the norm and its gradient
constexpr int kNarrowQuantBlock = 256;  // 1048576 x 64: 47 us; with 128 threads 68, for blocks that end faster than they can be started

template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
#pragma unroll
  for (int o = L / 2; o; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int VEC, int L>
__device__ __forceinline__ int narrow_column(int t, int i) { return VEC == 8 ? kNarrow * t + i : t + L * i; }
// A lane's elements of a row; those beyond its end, and of a row that is not there, are zero.
template <int VEC, int L, typename T>
__device__ __forceinline__ void narrow_load(const T* p, int width, int t, bool live, float (&f)[kNarrow]) {
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) f[i] = 0.f;
  if constexpr (VEC == 8) {
    if (live && kNarrow * t < width) load_vec<8, T>(p + kNarrow * t, f);
  } else {
#pragma unroll
    for (int i = 0; i < kNarrow; ++i)
      if (live && t + L * i < width) f[i] = to_f<T>(p[t + L * i]);
  }
}
template <int VEC, int L, typename T>
__device__ __forceinline__ void narrow_store(T* p, int width, int t, const float (&f)[kNarrow]) {
  if constexpr (VEC == 8) {
    if (kNarrow * t < width) store_vec<8, T>(p + kNarrow * t, f);
  } else {
#pragma unroll
    for (int i = 0; i < kNarrow; ++i)
      if (t + L * i < width) p[t + L * i] = from_f<T>(f[i]);
  }
}
template <int VEC, int L>
__device__ __forceinline__ void narrow_put_q(int8_t* p, int width, int t, const float (&f)[kNarrow], const RowScale& rs) {
  if constexpr (VEC == 8) {
    if (kNarrow * t < width) put_q<8>(p + kNarrow * t, f, rs);
  } else {
#pragma unroll
    for (int i = 0; i < kNarrow; ++i)
      if (t + L * i < width) p[t + L * i] = rs.ok ? (int8_t)rounded_bits(f[i], rs.inv) : (int8_t)0;
  }
}
template <int VEC, int L, typename T>
__device__ __forceinline__ void narrow_weight(const void* w, int w_f32, int width, int t, float (&f)[kNarrow]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) f[i] = 1.f;
  } else if (w_f32) {
    narrow_load<VEC, L, float>(reinterpret_cast<const float*>(w), width, t, true, f);
  } else {
    narrow_load<VEC, L, T>(reinterpret_cast<const T*>(w), width, t, true, f);
  }
}

template <typename T, int VEC, int L, bool Q8>
__global__ void __launch_bounds__(kNarrowBlock) narrow_norm_kernel(const NormArgs a) {
  dep_wait();
  dep_launch();
  const int t = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * (kNarrowBlock / L) + threadIdx.x / L;
  const bool live = row < a.rows;  // the lanes of rows beyond the last take part in the shuffles
  float f[kNarrow], w[kNarrow];
  narrow_load<VEC, L, T>(reinterpret_cast<const T*>(a.x) + row * a.ld_x, a.width, t, live, f);
  if (a.r) {
    float r[kNarrow];
    narrow_load<VEC, L, T>(reinterpret_cast<const T*>(a.r) + row * a.ld_r, a.width, t, live, r);
#pragma unroll
    for (int i = 0; i < kNarrow; ++i) f[i] = to_f<T>(from_f<T>(f[i] + r[i]));
  }
  narrow_weight<VEC, L, T>(a.w, a.w_f32, a.width, t, w);
  if (a.sum && live) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.sum) + row * a.ld_s, a.width, t, f);
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) sq = fmaf(f[i], f[i], sq);
  sq = group_sum<L>(sq);
  const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) {
    // elements beyond the row's end are not there to make 0 inf of
    f[i] = narrow_column<VEC, L>(t, i) < a.width ? f[i] * rho * w[i] : 0.f;
    if (Q8) most = max(most, mag(f[i]));
  }
  if (!Q8) {
    if (live) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.y) + row * a.ld_y, a.width, t, f);
  } else {
    const RowScale rs = row_scale(group_max<L>(most));
    if (!live) return;
    narrow_put_q<VEC, L>(reinterpret_cast<int8_t*>(a.y) + row * a.ld_y, a.width, t, f, rs);
    if (t == 0) a.scale[row] = rs.scale;
  }
}

template <typename T, int VEC, int L>
__global__ void __launch_bounds__(kNarrowQuantBlock) narrow_quantize_kernel(const QuantArgs a) {
  dep_wait();
  dep_launch();
  const int t = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * (kNarrowQuantBlock / L) + threadIdx.x / L;
  const bool live = row < a.rows;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.ld_x;
  float f[kNarrow];
  narrow_load<VEC, L, T>(x, a.width, t, live, f);
  if (a.act != ASD_ACT_NONE) {
    float u[kNarrow];
    narrow_load<VEC, L, T>(x + a.width, a.width, t, live, u);
#pragma unroll
    for (int i = 0; i < kNarrow; i += 2) {
      const float2 h = gated2(make_float2(f[i], f[i + 1]), make_float2(u[i], u[i + 1]), a.act);
      f[i] = h.x;
      f[i + 1] = h.y;
    }
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) most = max(most, mag(f[i]));
  const RowScale rs = row_scale(group_max<L>(most));
  if (!live) return;
  narrow_put_q<VEC, L>(a.q + row * a.ld_q, a.width, t, f, rs);
  if (t == 0) a.scale[row] = rs.scale;
}

// A block walks over its rows, kNarrowBlock / L at once and two such steps with their loads in flight together; the sums of dw stay
// in a lane's registers and are joined over the block's row groups at the end.
template <typename T, int VEC, int L>
__global__ void __launch_bounds__(kNarrowBlock) narrow_grad_kernel(const NormGradArgs a) {
  constexpr int ROWS = kNarrowBlock / L, U = VEC == 8 ? 2 : 1;
  __shared__ float sums[kNarrowBlock / 32][kNarrowWidth];
  dep_wait();
  dep_launch();
  const int t = threadIdx.x % L;
  float w[kNarrow], acc[kNarrow];
  narrow_weight<VEC, L, T>(a.w, a.w_f32, a.width, t, w);
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) {
    if (narrow_column<VEC, L>(t, i) >= a.width) w[i] = 0.f;
    acc[i] = 0.f;
  }
  for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += (int64_t)a.blocks * ROWS * U) {
    float f[U][kNarrow], g[U][kNarrow], e[U][kNarrow];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = first + (int64_t)u * a.blocks * ROWS + threadIdx.x / L;
      const bool live = row < a.rows;
      narrow_load<VEC, L, T>(reinterpret_cast<const T*>(a.s) + row * a.ld_s, a.width, t, live, f[u]);
      narrow_load<VEC, L, T>(reinterpret_cast<const T*>(a.dy) + row * a.ld_dy, a.width, t, live, g[u]);
      narrow_load<VEC, L, T>(reinterpret_cast<const T*>(a.ds) + row * a.ld_ds, a.width, t, live && a.ds, e[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = first + (int64_t)u * a.blocks * ROWS + threadIdx.x / L;
      const bool live = row < a.rows;
      float sq = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) {
        sq = fmaf(f[u][i], f[u][i], sq);
        dot = fmaf(g[u][i] * w[i], f[u][i], dot);
      }
      sq = group_sum<L>(sq);
      dot = group_sum<L>(dot);
      const float rho = 1.f / sqrtf(sq / (float)a.width + a.eps);
      const float k = -(rho * dot / (float)a.width) * rho;
#pragma unroll
      for (int i = 0; i < kNarrow; ++i) {
        const float z = f[u][i] * rho;
        if (live) acc[i] = fmaf(g[u][i], z, acc[i]);
        e[u][i] = fmaf(z, k, fmaf(g[u][i] * w[i], rho, e[u][i]));
      }
      if (live && a.dx) narrow_store<VEC, L, T>(reinterpret_cast<T*>(a.dx) + row * a.ld_dx, a.width, t, e[u]);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < kNarrow; ++i) {
    for (int o = L; o < 32; o <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    if ((threadIdx.x & 31) < L) sums[threadIdx.x >> 5][narrow_column<VEC, L>(t, i)] = acc[i];
  }
  __syncthreads();
  for (int col = threadIdx.x; col < a.width; col += kNarrowBlock) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kNarrowBlock / 32; ++k) v += sums[k][col];
    a.part[(size_t)blockIdx.x * a.width + col] = v;
  }
}

// Calls f with the lanes of a narrow row as a constant.
template <typename F>
void with_lanes(int width, F f) {
  if (width <= 8 * kNarrow)
    f(std::integral_constant<int, 8>());
  else if (width <= 16 * kNarrow)
    f(std::integral_constant<int, 16>());
  else
    f(std::integral_constant<int, 32>());
}
unsigned narrow_grid(int rows, int lanes, int block) { return (unsigned)(((int64_t)rows * lanes + block - 1) / block); }

// Up to four matrices to rows of a multiple of 16 bytes, in one launch (blockIdx.y).  A thread makes 16 bytes of a row from
// the aligned words that hold them, each shifted by the row's misalignment; a row's last bytes, and elements of a row that
// does not start on a word, are read one by one where a word would reach outside the row.
constexpr int kMostPacks = 4;
struct PackArgs {
  struct One {
    const uint8_t* src;
    uint8_t* dst;
    int64_t rows, ld_src, ld_dst;  // bytes
    int bytes;                     // of a row
  } m[kMostPacks];
};
__global__ void __launch_bounds__(256) pack_rows_kernel(const PackArgs a) {
  dep_wait();
  dep_launch();
  const PackArgs::One m = a.m[blockIdx.y];
  const int pieces = (m.bytes + 15) / 16;
  const int64_t total = m.rows * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / pieces;
    const int at = (int)(i - row * pieces) * 16;
    const uint8_t* p = m.src + row * m.ld_src + at;
    const int off = (int)((uintptr_t)p & 3);
    uint32_t w[4];
    if (at >= off && at + 20 <= m.bytes) {  // the five words around the piece lie inside the row
      const uint32_t* q = reinterpret_cast<const uint32_t*>(p - off);
      uint32_t v[5];
#pragma unroll
      for (int k = 0; k < 5; ++k) v[k] = q[k];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(v[k], v[k + 1], 8 * off);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[k] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + 4 * k + e < m.bytes) w[k] |= (uint32_t)p[4 * k + e] << (8 * e);
      }
    }
    *reinterpret_cast<uint4*>(m.dst + row * m.ld_dst + at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

bool aligned(const void* p, int64_t ld, int es, int bytes) { return ((uintptr_t)p % bytes) == 0 && (ld * es) % bytes == 0; }

// Threads to a row.  A row of up to 1024 is a warp's, so that its sums need no barrier, unless there are too few rows to
// fill the SMs with warps; then, and beyond, a block's.
int row_threads(const asd_ops* o, int64_t rows, int width) {
  if (width <= 32 * kPer && rows >= 8 * o->num_sms) return 32;
  if (width <= 128 * kPer && (width <= 1024 || rows >= 4 * o->num_sms)) return 128;
  if (width <= 256 * kPer && rows >= 2 * o->num_sms) return 256;
  return 512;
}

// How staged rows of `parts` operands of `bytes` are walked over by blocks of `threads` with `slots` rows each: one row ahead
// where its buffers fit, and as many blocks as the SMs hold together.
struct WalkPlan {
  Walk k;
  int grid, smem;
};
WalkPlan plan_walk(const asd_ops* o, int rows, int64_t bytes, int parts, int slots, int threads) {
  WalkPlan p;
  p.k.pitch = stage_pitch(bytes);
  p.k.parts = parts;
  p.k.ahead = 2 * slots * parts * p.k.pitch <= kStagedSmem ? 1 : 0;
  p.smem = (p.k.ahead + 1) * slots * parts * p.k.pitch;
  int side = kStagedSmem / p.smem;
  if (side > 1024 / threads) side = 1024 / threads;
  const int blocks = (rows + slots - 1) / slots, most = o->num_sms * (side < 1 ? 1 : side);
  p.grid = blocks < most ? blocks : most;
  p.k.stride = p.grid * slots;
  return p;
}
template <typename T, int TPR, bool Q8>
void rmsnorm_staged(const asd_ops* o, const NormArgs& n, cudaStream_t st) {
  const WalkPlan p = plan_walk(o, n.rows, (int64_t)n.width * sizeof(T), n.r ? 2 : 1, TPR == 32 ? 4 : 1, block_of<TPR>);
  ops_launch(rmsnorm_staged_kernel<T, TPR, Q8>, dim3(p.grid), dim3(block_of<TPR>), (size_t)p.smem, st, 1, n, p.k);
}
template <typename T, bool Q8>
void rmsnorm_t(const asd_ops* o, const NormArgs& n, bool vec, cudaStream_t st) {
  if (n.width <= kNarrowWidth) {
    with_lanes(n.width, [&](auto lanes) {
      constexpr int L = decltype(lanes)::value;
      ops_launch(vec ? narrow_norm_kernel<T, 8, L, Q8> : narrow_norm_kernel<T, 1, L, Q8>, dim3(narrow_grid(n.rows, L, kNarrowBlock)),
                 dim3(kNarrowBlock), 0, st, 1, n);
    });
    return;
  }
  if (n.width > 512 * kPer) {
    if (vec)
      ops_launch(rmsnorm_kernel<T, 8, 512, Q8, true>, dim3(n.rows), dim3(512), 0, st, 1, n);
    else
      ops_launch(rmsnorm_kernel<T, 1, 512, Q8, true>, dim3(n.rows), dim3(512), 0, st, 1, n);
    return;
  }
  switch (row_threads(o, n.rows, n.width)) {
    case 32:
      if (!vec) return rmsnorm_staged<T, 32, Q8>(o, n, st);
      return ops_launch(rmsnorm_kernel<T, 8, 32, Q8, false>, dim3((n.rows + 3) / 4), dim3(128), 0, st, 1, n);
    case 128:
      if (!vec) return rmsnorm_staged<T, 128, Q8>(o, n, st);
      return ops_launch(rmsnorm_kernel<T, 8, 128, Q8, false>, dim3(n.rows), dim3(128), 0, st, 1, n);
    case 256:
      if (!vec) return rmsnorm_staged<T, 256, Q8>(o, n, st);
      return ops_launch(rmsnorm_kernel<T, 8, 256, Q8, false>, dim3(n.rows), dim3(256), 0, st, 1, n);
    default:
      if (!vec) return rmsnorm_staged<T, 512, Q8>(o, n, st);
      return ops_launch(rmsnorm_kernel<T, 8, 512, Q8, false>, dim3(n.rows), dim3(512), 0, st, 1, n);
  }
}
template <typename T>
void rmsnorm_type(const asd_ops* o, const NormArgs& n, bool vec, bool q8, cudaStream_t st) {
  q8 ? rmsnorm_t<T, true>(o, n, vec, st) : rmsnorm_t<T, false>(o, n, vec, st);
}

template <typename T, int TPR>
void quantize_rows(const asd_ops* o, QuantArgs n, bool vec, cudaStream_t st) {
  const int per_block = TPR == 32 ? 4 : 1;
  if (!vec) {
    const WalkPlan p = plan_walk(o, n.rows, (int64_t)n.width * sizeof(T) * (n.act != ASD_ACT_NONE ? 2 : 1), 1, per_block, block_of<TPR>);
    ops_launch(quantize_staged_kernel<T, TPR>, dim3(p.grid), dim3(block_of<TPR>), (size_t)p.smem, st, 1, n, p.k);
    return;
  }
  constexpr int smem = quantize_smem<T, 8, TPR>;
  // as many blocks as the SMs hold together
  const int blocks = (n.rows + per_block - 1) / per_block, most = o->num_sms * (smem ? 232448 / (smem + 1024) : 1024 / block_of<TPR>);
  const int grid = blocks < most ? blocks : most;
  n.stride = grid * per_block;
  ops_launch(quantize_kernel<T, 8, TPR>, dim3(grid), dim3(block_of<TPR>), (size_t)smem, st, 1, n);
}
template <typename T>
void quantize_t(const asd_ops* o, const QuantArgs& n, bool vec, cudaStream_t st) {
  if (n.width <= kNarrowWidth) {
    with_lanes(n.width, [&](auto lanes) {
      constexpr int L = decltype(lanes)::value;
      ops_launch(vec ? narrow_quantize_kernel<T, 8, L> : narrow_quantize_kernel<T, 1, L>, dim3(narrow_grid(n.rows, L, kNarrowQuantBlock)),
                 dim3(kNarrowQuantBlock), 0, st, 1, n);
    });
    return;
  }
  if (n.width > 512 * kPer) {
    if (vec)
      ops_launch(quantize_long_kernel<T, 8>, dim3(n.rows), dim3(512), 0, st, 1, n);
    else
      ops_launch(quantize_long_kernel<T, 1>, dim3(n.rows), dim3(512), 0, st, 1, n);
    return;
  }
  switch (row_threads(o, n.rows, n.width)) {
    case 32: return quantize_rows<T, 32>(o, n, vec, st);
    case 128: return quantize_rows<T, 128>(o, n, vec, st);
    case 256: return quantize_rows<T, 256>(o, n, vec, st);
    default: return quantize_rows<T, 512>(o, n, vec, st);
  }
}

constexpr int kGradWidth = 8192;  // the longest row whose sums of dw a block keeps in registers
// Blocks of the gradient: as many as the SMs hold together, so that each block's sums of dw are over as many rows as
// possible.
int grad_blocks(const asd_ops* o, int64_t rows, int width) {
  if (width <= kNarrowWidth) {  // of several rows at once
    const int64_t all = ((int64_t)narrow_grid((int)rows, width <= 64 ? 8 : width <= 128 ? 16 : 32, kNarrowBlock)), most = 5 * (int64_t)o->num_sms;
    return (int)(all < most ? all : most);
  }
  const int per_sm = width <= 1024 ? 8 : width <= 4096 ? 2 : width <= kGradWidth ? 1 : 2;
  const int64_t most = (int64_t)per_sm * o->num_sms;
  return (int)(rows < most ? rows : most);
}
template <typename T, int VEC, int TPR>
size_t grad_bytes(const NormGradArgs& n) {
  return VEC == 8 ? (size_t)grad_smem<T, VEC, TPR, 16> : (size_t)(grad_ahead<T> + 1) * 3 * n.pitch;
}
template <typename T, int VEC>
void grad_t(const asd_ops* o, const NormGradArgs& n, cudaStream_t st) {
  if (n.width <= kNarrowWidth)
    with_lanes(n.width, [&](auto lanes) {
      constexpr int L = decltype(lanes)::value;
      ops_launch(narrow_grad_kernel<T, VEC, L>, dim3(n.blocks), dim3(kNarrowBlock), 0, st, 1, n);
    });
  else if (n.width <= 1024)
    ops_launch(rmsnorm_grad_kernel<T, VEC, 64, 16>, dim3(n.blocks), dim3(64), grad_bytes<T, VEC, 64>(n), st, 1, n);
  else if (n.width <= 4096)
    ops_launch(rmsnorm_grad_kernel<T, VEC, 256, 16>, dim3(n.blocks), dim3(256), grad_bytes<T, VEC, 256>(n), st, 1, n);
  else if (n.width <= kGradWidth)
    ops_launch(rmsnorm_grad_kernel<T, VEC, 512, 16>, dim3(n.blocks), dim3(512), grad_bytes<T, VEC, 512>(n), st, 1, n);
  else {
    NormGradArgs stats = n;
    stats.dx = nullptr;
    const bool over_dy = n.part && n.dx == n.dy;  // dw needs dy, so dx comes after it
    ops_launch(rmsnorm_grad_long_kernel<T>, dim3(n.rows), dim3(512), 0, st, 1, over_dy ? stats : n);
    if (n.part) ops_launch(columns_dw_kernel<T>, dim3((n.width + 127) / 128, n.blocks), dim3(128), 0, st, 1, n);
    if (over_dy) ops_launch(rmsnorm_grad_long_kernel<T>, dim3(n.rows), dim3(512), 0, st, 1, n);
  }
}

}  // namespace

void launch_rmsnorm(const asd_ops* o, const asd_rmsnorm_args* a, cudaStream_t st) {
  NormArgs n{};
  n.rows = a->rows, n.width = a->width, n.w_f32 = a->w_type == ASD_TYPE_F32, n.eps = a->eps;
  n.x = a->x, n.r = a->residual, n.w = a->weight, n.sum = a->sum, n.y = a->y, n.scale = a->scale;
  n.ld_x = a->ld_x, n.ld_r = a->ld_residual, n.ld_s = a->ld_sum, n.ld_y = a->ld_y;
  const int es = ops_type_size(a->type);
  const bool q8 = a->scale != nullptr;
  const bool vec = a->width % 8 == 0 && aligned(a->x, a->ld_x, es, 16) && (!a->residual || aligned(a->residual, a->ld_residual, es, 16)) &&
                   (!a->weight || aligned(a->weight, 0, es, 16)) && (!a->sum || aligned(a->sum, a->ld_sum, es, 16)) &&
                   (q8 ? aligned(a->y, a->ld_y, 1, 8) : aligned(a->y, a->ld_y, es, 16));
  if (a->type == ASD_TYPE_F32)
    rmsnorm_type<float>(o, n, vec, q8, st);
  else if (a->type == ASD_TYPE_F16)
    rmsnorm_type<__half>(o, n, vec, q8, st);
  else
    rmsnorm_type<__nv_bfloat16>(o, n, vec, q8, st);
}

void launch_quantize(const asd_ops* o, const asd_quantize_args* a, cudaStream_t st) {
  QuantArgs n{};
  n.rows = a->rows, n.width = a->width, n.act = a->act, n.x = a->x, n.q = a->q, n.scale = a->scale, n.ld_x = a->ld_x, n.ld_q = a->ld_q;
  const bool vec = a->width % 8 == 0 && aligned(a->x, a->ld_x, ops_type_size(a->type), 16) && aligned(a->q, a->ld_q, 1, 8);
  if (a->type == ASD_TYPE_F32)
    quantize_t<float>(o, n, vec, st);
  else if (a->type == ASD_TYPE_F16)
    quantize_t<__half>(o, n, vec, st);
  else
    quantize_t<__nv_bfloat16>(o, n, vec, st);
}

namespace {
template <typename K>
cudaError_t allow_smem(K* kernel, int bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <typename T, int TPR>
cudaError_t prepare_staged() {
  for (cudaError_t e : {allow_smem(rmsnorm_staged_kernel<T, TPR, true>, kStagedSmem), allow_smem(rmsnorm_staged_kernel<T, TPR, false>, kStagedSmem),
                        allow_smem(quantize_staged_kernel<T, TPR>, kStagedSmem)})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}
template <typename T>
cudaError_t prepare_rows() {
  for (cudaError_t e : {prepare_staged<T, 32>(), prepare_staged<T, 128>(), prepare_staged<T, 256>(), prepare_staged<T, 512>(),
                        allow_smem(quantize_kernel<T, 8, 256>, quantize_smem<T, 8, 256>), allow_smem(quantize_kernel<T, 8, 512>, quantize_smem<T, 8, 512>),
                        allow_smem(rmsnorm_grad_kernel<T, 8, 256, 16>, grad_smem<T, 8, 256, 16>),
                        allow_smem(rmsnorm_grad_kernel<T, 8, 512, 16>, grad_smem<T, 8, 512, 16>),
                        allow_smem(rmsnorm_grad_kernel<T, 1, 64, 16>, kStagedSmem), allow_smem(rmsnorm_grad_kernel<T, 1, 256, 16>, kStagedSmem),
                        allow_smem(rmsnorm_grad_kernel<T, 1, 512, 16>, kStagedSmem)})
    if (e != cudaSuccess) return e;
  return cudaSuccess;
}
}  // namespace
asd_status ops_rows_prepare() {
  for (cudaError_t e : {prepare_rows<float>(), prepare_rows<__half>(), prepare_rows<__nv_bfloat16>()})
    if (e != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  return ASD_OK;
}

int64_t rmsnorm_backward_bytes(const asd_ops* o, const asd_rmsnorm_backward_args* a) {
  if (!a->dw || a->rows == 0) return 0;
  return 4 * ((int64_t)grad_blocks(o, a->rows, a->width) * a->width + (a->width > kGradWidth ? a->rows : 0));
}

void launch_rmsnorm_backward(const asd_ops* o, const asd_rmsnorm_backward_args* a, cudaStream_t st) {
  NormGradArgs n{};
  n.rows = a->rows, n.width = a->width, n.w_f32 = a->w_type == ASD_TYPE_F32, n.eps = a->eps;
  n.blocks = grad_blocks(o, a->rows, a->width);
  n.dy = a->dy, n.s = a->s, n.ds = a->ds, n.w = a->weight, n.dx = a->dx;
  n.ld_dy = a->ld_dy, n.ld_s = a->ld_s, n.ld_ds = a->ld_ds, n.ld_dx = a->ld_dx;
  if (a->dw) {
    n.part = reinterpret_cast<float*>(a->workspace);
    n.rho = n.part + (size_t)n.blocks * a->width;
  }
  const int es = ops_type_size(a->type);
  n.pitch = stage_pitch((int64_t)a->width * es);
  const bool vec = a->width % 8 == 0 && aligned(a->dy, a->ld_dy, es, 16) && aligned(a->s, a->ld_s, es, 16) &&
                   (!a->ds || aligned(a->ds, a->ld_ds, es, 16)) && (!a->weight || aligned(a->weight, 0, es, 16)) &&
                   (!a->dx || aligned(a->dx, a->ld_dx, es, 16));
  if (a->type == ASD_TYPE_F32)
    vec ? grad_t<float, 8>(o, n, st) : grad_t<float, 1>(o, n, st);
  else if (a->type == ASD_TYPE_F16)
    vec ? grad_t<__half, 8>(o, n, st) : grad_t<__half, 1>(o, n, st);
  else
    vec ? grad_t<__nv_bfloat16, 8>(o, n, st) : grad_t<__nv_bfloat16, 1>(o, n, st);
  if (!a->dw) return;
  const dim3 grid((a->width + 31) / 32), block(32, 32);
  if (a->w_type == ASD_TYPE_F32)
    ops_launch(reduce_dw_kernel<float>, grid, block, 0, st, 1, (const float*)n.part, n.blocks, n.width, reinterpret_cast<float*>(a->dw));
  else if (a->w_type == ASD_TYPE_F16)
    ops_launch(reduce_dw_kernel<__half>, grid, block, 0, st, 1, (const float*)n.part, n.blocks, n.width, reinterpret_cast<__half*>(a->dw));
  else
    ops_launch(reduce_dw_kernel<__nv_bfloat16>, grid, block, 0, st, 1, (const float*)n.part, n.blocks, n.width,
               reinterpret_cast<__nv_bfloat16*>(a->dw));
}

void launch_packs(const asd_ops* o, const Packs& packs, cudaStream_t st) {
  if (!packs.n) return;
  PackArgs a{};
  int64_t most = 0;
  for (int i = 0; i < packs.n; ++i) {
    const Mat& s = packs.src[i];
    const int bytes = (int)(s.cols * s.es);
    a.m[i] = {(const uint8_t*)s.p, (uint8_t*)packs.dst[i], s.rows, s.ld * s.es, packs.ld[i] * s.es, bytes};
    const int64_t blocks = (s.rows * ((bytes + 15) / 16) + 255) / 256;
    most = blocks > most ? blocks : most;
  }
  if (most > o->num_sms * 8) most = o->num_sms * 8;
  ops_launch(pack_rows_kernel, dim3((unsigned)most, packs.n), dim3(256), 0, st, 1, a);
}

}  // namespace asd
