// Device-side pieces shared by the operators' tensor-core kernels: shared-memory descriptors of both operand orders, the
// MMA of each operand kind, the gated activation with its gradient, and the 24-bit form in which a training step keeps
// the gate's two factors.  Everything here has internal linkage.
#pragma once

#include "asd_ops_act.cuh"
#include "asd_ops_internal.h"
#include "asd_tc.cuh"

namespace asd {
namespace {

// A tile in shared memory is made of 128-byte rows with the 128-byte swizzle, as the TMA writes them.
//   along k:  a row is an m or n index, 64 16-bit (128 8-bit) elements of k; groups of 8 rows are 1024 bytes apart
//             (stride offset).  One MMA's k is 32 bytes of a row: the next starts 32 bytes further.
//   along mn: a row is a k index, 64 elements of m or n; groups of 8 rows are 1024 bytes apart (stride offset) and
//             blocks of 64 elements of m or n are 64 rows = 8192 bytes apart (leading offset).  One MMA's k is 16
//             rows: the next starts 2048 bytes further.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn) {
  uint64_t d = smem_desc_sw128(addr);
  if (mn) d = (d & ~(0x3FFFull << 16)) | ((uint64_t)(8192 >> 4) << 16);
  return d;
}
__device__ __forceinline__ uint64_t desc_step(bool mn) { return mn ? 128u : 2u; }

template <bool I8, int CTAS>
__device__ __forceinline__ void tc_mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (!I8 && CTAS == 2)
    tc_mma_bf16_pair(d_tmem, a, b, idesc, accumulate);
  else if constexpr (!I8)
    tc_mma_bf16(d_tmem, a, b, idesc, accumulate);
  else if constexpr (CTAS == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, {%5, %5, %5, %5, %5, %5, %5, %5}, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, {%5, %5, %5, %5}, p;\n\t}" ::"r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(0u)
        : "memory");
}

// Two fp32 values rounded to a pair of 16-bit ones, the first in the low half.
__device__ __forceinline__ uint32_t pack16(float a, float b, bool f16) {
  uint32_t r;
  if (f16)
    asm("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(a), "f"(b));
  else
    asm("cvt.rn.bf16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint16_t round16(float a, bool f16) {
  return f16 ? __half_as_ushort(__float2half_rn(a)) : __bfloat16_as_ushort(__float2bfloat16_rn(a));
}

// act(g).  The exponential and reciprocal are the approximate instructions (relative error some 2^-22, far below the
// 16-bit rounding that follows).
__device__ __forceinline__ float sigmoid_approx(float g) { return rcp_approx(1.f + ex2_approx(g * kNegLog2e)); }
template <bool GELU>
__device__ __forceinline__ float gate_value(float g) {
  return g * (GELU ? normal_cdf(g).x : sigmoid_approx(g));
}
// act(g) and act'(g):  silu' = p (1 + g (1 - p)),  gelu' = Phi + g phi.
template <bool GELU>
__device__ __forceinline__ void gate_grad(float g, float& a, float& da) {
  if (!GELU) {
    const float p = sigmoid_approx(g);
    a = g * p;
    da = fmaf(a, 1.f - p, p);
  } else {
    const float2 p = normal_cdf(g);
    a = g * p.x;
    da = fmaf(g * 0.3989422804014327f, p.y, p.x);
  }
}

// N gated values: h = act(g) u, and (KEEP) g and u replaced by u act'(g) and act(g).  The activation is chosen once for all of
// them: a branch for each would keep the elements from being worked on side by side (a 256 x 128 tile of h: 11 against 4
// thousand clocks).
template <bool GELU, bool KEEP, int N>
__device__ __forceinline__ void gated_n(float (&g)[N], float (&u)[N], float (&h)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (KEEP) {
      float a, da;
      gate_grad<GELU>(g[i], a, da);
      h[i] = a * u[i];
      g[i] = u[i] * da;
      u[i] = a;
    } else {
      h[i] = gate_value<GELU>(g[i]) * u[i];
    }
  }
}
template <int N>
__device__ __forceinline__ void gated(float (&g)[N], float (&u)[N], float (&h)[N], bool gelu, bool keep) {
  if (gelu)
    keep ? gated_n<true, true>(g, u, h) : gated_n<true, false>(g, u, h);
  else
    keep ? gated_n<false, true>(g, u, h) : gated_n<false, false>(g, u, h);
}

// What a training step keeps of the gate.  h = act(g) u has the derivatives act(g) in u and u act'(g) in g, and it is these
// two factors that are kept: the backward pass then multiplies dh by them, without an exponential.  Rounding them to bf16
// would make the gradients' error half as large again as the roundings of dg, du and the result make it; fp32 would double
// the traffic.  Kept are the upper 24 bits of the fp32 value (truncated: sign, exponent and 15 bits, an error below 2^-15, always towards zero: a
// 128th of the rounding of dg and du to bf16, a 16th of that to fp16; rounding them would take an addition and a guard for NaN each),
// the upper 16 and the next 8 in separate vectors.  The order is that of the accumulator tiles, where a thread holds 32
// neighbouring columns of a row: a block is 32 rows x 32 columns of u act'(g), then of act(g), each as 4 + 2 vectors of 16
// bytes for every row, vector by vector, so that a warp's stores and loads are whole 512-byte runs.
constexpr int kKeptHalf = 32 * 32 * 3;
constexpr int kKeptBlock = 2 * kKeptHalf;
__device__ __forceinline__ void kept_store(uint8_t* block, int lane, const uint32_t (&v)[32]) {
  uint4* p = reinterpret_cast<uint4*>(block) + lane;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint4 h;
    h.x = __byte_perm(v[8 * i + 0], v[8 * i + 1], 0x7632);
    h.y = __byte_perm(v[8 * i + 2], v[8 * i + 3], 0x7632);
    h.z = __byte_perm(v[8 * i + 4], v[8 * i + 5], 0x7632);
    h.w = __byte_perm(v[8 * i + 6], v[8 * i + 7], 0x7632);
    p[32 * i] = h;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = 16 * i + 4 * j;
      w[j] = __byte_perm(__byte_perm(v[c], v[c + 1], 0x0051), __byte_perm(v[c + 2], v[c + 3], 0x0051), 0x5410);
    }
    p[32 * (4 + i)] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
__device__ __forceinline__ void kept_fetch(const uint8_t* block, int lane, uint4 (&r)[6]) {
  const uint4* p = reinterpret_cast<const uint4*>(block) + lane;
#pragma unroll
  for (int i = 0; i < 6; ++i) r[i] = p[32 * i];
}
// Column c (0..31) of a row's six vectors.
__device__ __forceinline__ float kept_value(const uint4 (&r)[6], int c) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r[0]);
  const uint32_t hi = w[c >> 1], lo = w[16 + (c >> 2)];
  // bytes of the value, low to high: 0, lo byte c & 3, the two of the upper half
  const uint32_t h = (c & 1) ? __byte_perm(hi, 0u, 0x3244) : __byte_perm(hi, 0u, 0x1044);
  return __uint_as_float(__byte_perm(h, lo, 0x3200 | ((4 + (c & 3)) << 4)));
}
// The same value by its place in the buffer, for the kernels whose threads do not hold rows of it.
__device__ __forceinline__ size_t kept_offset(int row, int col, int col_blocks) {
  return ((size_t)(row >> 5) * col_blocks + (col >> 5)) * kKeptBlock;
}
__device__ __forceinline__ void kept_put(uint8_t* half, int r, int c, float v) {
  const uint32_t b = __float_as_uint(v);
  *reinterpret_cast<uint16_t*>(half + ((c >> 3) * 32 + r) * 16 + (c & 7) * 2) = (uint16_t)(b >> 16);
  half[((4 + (c >> 4)) * 32 + r) * 16 + (c & 15)] = (uint8_t)(b >> 8);
}
// Four neighbouring columns from a multiple of four.
__device__ __forceinline__ void kept_put4(uint8_t* half, int r, int c, const float (&v)[4]) {
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(v[e]);
  *reinterpret_cast<uint2*>(half + ((c >> 3) * 32 + r) * 16 + (c & 7) * 2) = make_uint2(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632));
  *reinterpret_cast<uint32_t*>(half + ((4 + (c >> 4)) * 32 + r) * 16 + (c & 15)) =
      __byte_perm(__byte_perm(b[0], b[1], 0x0051), __byte_perm(b[2], b[3], 0x0051), 0x5410);
}
__device__ __forceinline__ void kept_get4(const uint8_t* half, int r, int c, float (&v)[4]) {
  const uint2 hi = *reinterpret_cast<const uint2*>(half + ((c >> 3) * 32 + r) * 16 + (c & 7) * 2);
  const uint32_t lo = *reinterpret_cast<const uint32_t*>(half + ((4 + (c >> 4)) * 32 + r) * 16 + (c & 15));
  v[0] = __uint_as_float((hi.x << 16) | ((lo & 0xffu) << 8));
  v[1] = __uint_as_float((hi.x & 0xffff0000u) | (lo & 0xff00u));
  v[2] = __uint_as_float((hi.y << 16) | ((lo >> 8) & 0xff00u));
  v[3] = __uint_as_float((hi.y & 0xffff0000u) | ((lo >> 16) & 0xff00u));
}

}  // namespace
}  // namespace asd
