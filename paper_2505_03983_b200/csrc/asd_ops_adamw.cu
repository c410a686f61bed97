// A step of AdamW over many tensors in one launch, with the moments in 32 bits or in 8:
//   g = grad scale,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: 28 bytes a parameter with moments and a master value in 32 bits and parameter and gradient in 16, 16 bytes with
// moments in 8 bits.  117M parameters: 504 us in 32 bits (6.5 TB/s), 336 in 8 (5.6 TB/s; some 50 instructions an element beside
// the memory's time; 508 us with integer conversions, types chosen at each operand and exact divisions), 357 with random bits for
// the codes (5.3 TB/s, 54 % of the issue slots where it was 44).  A warp works on 256 neighbouring elements at a time, eight to a lane,
// which is also the block of elements that shares a scale in 8 bits, so that its largest values are two warp-wide maxima.  The tensors'
// addresses are the launch's arguments (up to 32 KB of them): they need no copy of their own and a captured graph keeps them.
//
// 8 bits: m = M (q / 127) |q / 127| with M the block's largest |m|, sqrt(v) = R (q / 255)^2 with R its largest sqrt(v).  The square
// puts the steps where the values are: half a step is 0.4 % of the largest value there, 4 % of one that is a hundredth of
// it.  sqrt(v) is the denominator, so a v above 0 has a q of 1 at least.
//
// Codes are rounded to the nearest, or (ASD_ADAMW_UNBIASED) up with the probability of their fraction.  Half a step of v is 2 / q of it, a
// decay by beta2 = 0.999 only 0.001: rounded to the nearest, no code ever falls by decay while a large gradient lifts it, and sqrt(v)
// in a block of gradients of one size, beside that in 32 bits, has a mean of 1.04 after 1000 steps, 1.14 after 3000 and 1.33 after 10000
// (1.001, 1.002, 1.001 with the fraction's probability).  So it is with an m of less than 0.6 % of M at beta1 = 0.9, which then never
// comes to 0.  Both are rounded so or neither: an m that stays beside a v that falls would be a step that grows.  As a code goes with
// the root of m and the fourth root of v, roundings that leave its mean alone make v some 1.5 / q larger, which the mean of 1 / sqrt(v), the
// step, gets back from v's spread.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "asd_ops_rows.cuh"

namespace asd {
namespace {

constexpr int kUnit = 256;     // elements of a warp at a time, and of a scale
constexpr int kItem = 4;       // units that a warp takes in a row
constexpr int kAdamBlock = 256;
constexpr int kAdamSide = 3;  // blocks of an SM at a time
constexpr int kUnbiased = 8 | ASD_ADAMW_UNBIASED;  // a kernel's BITS: 32, 8 or this
// Blocks in all, for an SM.  In 32 bits memory is the time, and many blocks even out what the SMs get of it (117M parameters, 4: 604 us, 8:
// 520, 16: 521, 48: 503); in 8 bits it is not all of it, and blocks beyond those that run together only begin again (3: 336 us, 6: 351, 32: 367).
template <int BITS>
constexpr int kAdamBlocks = BITS == 32 ? 32 : kAdamSide;

struct AdamTensor {
  void* param;
  const void* grad;
  float* master;  // or NULL
  void *m, *v;
  float2* scales;  // (M, R)
  int64_t n;
  int first;       // number of its first item
  int16_t type, grad_type : 8, wide : 8;  // wide: every address can be read 8 elements at a time
};
template <int N>
struct AdamArgs {
  AdamTensor t[N];
  int count, items, advance;
  float b1, c1, b2, c2, eps, wd, lr;  // c = 1 - b
  float log_b1, log_b2;
  const float *lr_at, *grad_scale, *skip;
  int64_t* step;
};

__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Of numbers that may be taken for 0 where they are below 2^-126.
__device__ __forceinline__ float sqrt_fast(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A lane's eight elements of a unit: neighbouring ones (WIDE), or every 32nd with those from n on left out.
template <bool WIDE>
__device__ __forceinline__ int64_t element(int64_t base, int lane, int i) {
  return WIDE ? base + 8 * lane + i : base + lane + 32 * i;
}
template <bool WIDE, typename T>
__device__ __forceinline__ void load_8(const void* p, int64_t base, int lane, int64_t n, float (&f)[8]) {
  if constexpr (WIDE) {
    load_vec<8, T>(reinterpret_cast<const T*>(p) + base + 8 * lane, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = element<false>(base, lane, i) < n ? to_f<T>(reinterpret_cast<const T*>(p)[element<false>(base, lane, i)]) : 0.f;
  }
}
template <bool WIDE, typename T>
__device__ __forceinline__ void store_8(void* p, int64_t base, int lane, int64_t n, const float (&f)[8]) {
  if constexpr (WIDE) {
    store_vec<8, T>(reinterpret_cast<T*>(p) + base + 8 * lane, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (element<false>(base, lane, i) < n) reinterpret_cast<T*>(p)[element<false>(base, lane, i)] = from_f<T>(f[i]);
  }
}
template <bool WIDE>
__device__ __forceinline__ void store_8(void* p, int type, int64_t base, int lane, int64_t n, const float (&f)[8]) {
  if (type == ASD_TYPE_BF16)
    store_8<WIDE, __nv_bfloat16>(p, base, lane, n, f);
  else if (type == ASD_TYPE_F16)
    store_8<WIDE, __half>(p, base, lane, n, f);
  else
    store_8<WIDE, float>(p, base, lane, n, f);
}
// A lane's eight codes, as the bytes of two words.
template <bool WIDE>
__device__ __forceinline__ void load_codes(const void* p, int64_t base, int lane, int64_t n, uint32_t (&w)[2]) {
  if constexpr (WIDE) {
    const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(p) + base + 8 * lane);
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = w[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (element<false>(base, lane, i) < n) w[i >> 2] |= (uint32_t)reinterpret_cast<const uint8_t*>(p)[element<false>(base, lane, i)] << (8 * (i & 3));
  }
}
template <bool WIDE>
__device__ __forceinline__ void store_codes(void* p, int64_t base, int lane, int64_t n, const uint32_t (&w)[2]) {
  if constexpr (WIDE) {
    *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(p) + base + 8 * lane) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (element<false>(base, lane, i) < n) reinterpret_cast<uint8_t*>(p)[element<false>(base, lane, i)] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
  }
}
// 2^23 plus bytes i and i + 1 of w.
__device__ __forceinline__ float2 byte_pair(uint32_t w, int i) {
  return make_float2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7540 | i)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7541 + i)));
}
// The other way: the nearest integers to four numbers of -127 to 255, ties to even, as bytes.
__device__ __forceinline__ uint32_t round_4(float a, float b, float c, float d) {
  const float2 up = make_float2(12582912.f, 12582912.f), x = add2(make_float2(a, b), up), y = add2(make_float2(c, d), up);
  return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040), __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
}
// What is added to codes before they are rounded to the nearest, 16 bits of r to a code: -0.5 to 0.5, both left out, so that a whole
// number stays what it is.
__device__ __forceinline__ float2 dither_pair(uint32_t r) {
  constexpr float kIn = 1.f - 1.f / 32768.f;  // 128 + 16 bits, less 128.5, times this
  return fma2(make_float2(__uint_as_float(__byte_perm(r, 0x43000000u, 0x7610)), __uint_as_float(__byte_perm(r, 0x43000000u, 0x7632))),
              make_float2(kIn, kIn), make_float2(-128.5f * kIn, -128.5f * kIn));
}
// 64 random bits of eight neighbouring elements and a step by Philox-2x32 (7 rounds), and from them, by odd factors (digits of pi), 16 for
// each of their codes of v (the first four words) and of m: each code's own bits are uniform over the steps, and the same in every run.
__device__ __forceinline__ void dither_bits(int64_t at, int64_t step, uint32_t (&r)[8]) {
  uint32_t a = (uint32_t)at, b = (uint32_t)step, key = (uint32_t)(at >> 32) ^ ((uint32_t)(step >> 32) << 16);
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    const uint32_t high = __umulhi(a, 0xd256d193u), low = a * 0xd256d193u;
    a = high ^ key ^ b, b = low, key += 0x9e3779b9u;
  }
  r[0] = a, r[1] = b, r[2] = a * 0x243f6a89u, r[3] = b * 0x243f6a89u;
  r[4] = b * 0x85a308d3u, r[5] = a * 0x85a308d3u, r[6] = b * 0x13198a2fu, r[7] = a * 0x13198a2fu;
}
// The dithers of a lane's eight elements.  They go by the element's place alone, not by how its lane came to it.
template <bool WIDE>
__device__ __forceinline__ void dithers(int64_t base, int lane, int64_t step, float2 (&m)[4], float2 (&v)[4]) {
  uint32_t r[8];
  if constexpr (WIDE) {
    dither_bits(base / 8 + lane, step, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = dither_pair(r[i]), m[i] = dither_pair(r[4 + i]);
  } else {
    const int word = (lane & 7) >> 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dither_bits(element<false>(base, lane, i) / 8, step, r);
      const uint32_t rv = word & 2 ? (word & 1 ? r[3] : r[2]) : (word & 1 ? r[1] : r[0]), rm = word & 2 ? (word & 1 ? r[7] : r[6]) : (word & 1 ? r[5] : r[4]);
      const float2 pv = dither_pair(rv), pm = dither_pair(rm);
      const float fv = lane & 1 ? pv.y : pv.x, fm = lane & 1 ? pm.y : pm.x;
      i & 1 ? v[i >> 1].y = fv : v[i >> 1].x = fv;
      i & 1 ? m[i >> 1].y = fm : m[i >> 1].x = fm;
    }
  }
}
// The moments that a block's codes stand for.
__device__ __forceinline__ void moments_of(const uint32_t (&qm)[2], const uint32_t (&qv)[2], float2 scale, float (&fm)[8], float (&fv)[8]) {
  const float km = scale.x * (1.f / 16129.f), kv = scale.y * (1.f / 65025.f);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t wm = qm[i >> 2] ^ 0x80808080u, wv = qv[i >> 2];
    // a byte in the low bits of 2^23, which is then taken off (a conversion would be one of the slow instructions); signed ones 128 up
    const float2 a = add2(byte_pair(wm, i & 3), make_float2(-8388736.f, -8388736.f)), b = add2(byte_pair(wv, i & 3), make_float2(-8388608.f, -8388608.f));
    const float2 x = mul2(mul2(a, make_float2(fabsf(a.x), fabsf(a.y))), make_float2(km, km)), r = mul2(mul2(b, b), make_float2(kv, kv));
    const float2 y = mul2(r, r);
    fm[i] = x.x, fm[i + 1] = x.y, fv[i] = y.x, fv[i + 1] = y.y;
  }
}

struct Step {
  float b1, c1, b2, c2, eps, decay, size, root, scale;  // decay = lr wd, size = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
  int64_t number;
};
// A unit of a tensor whose gradient has type G and whose values have type V.  The types are known where the unit is compiled: behind
// a choice of type each operand's conversion would wait for it before the next one is asked for.
template <int BITS, bool WIDE, typename G, typename V>
__device__ __forceinline__ void adam_unit(const AdamTensor& t, int64_t base, int lane, const Step& s) {
  float g[8], p[8], m[8], v[8];
  void* value = t.master ? (void*)t.master : t.param;
  load_8<WIDE, G>(t.grad, base, lane, t.n, g);
  load_8<WIDE, V>(value, base, lane, t.n, p);
  if constexpr (BITS == 32) {
    load_8<WIDE, float>(t.m, base, lane, t.n, m);
    load_8<WIDE, float>(t.v, base, lane, t.n, v);
  } else {
    uint32_t qm[2], qv[2];
    const float2 scale = t.scales[base / kUnit];
    load_codes<WIDE>(t.m, base, lane, t.n, qm);
    load_codes<WIDE>(t.v, base, lane, t.n, qv);
    moments_of(qm, qv, scale, m, v);
  }
  float r[8];  // sqrt(v)
  auto two = [](float x) { return make_float2(x, x); };
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 gi = mul2(make_float2(g[i], g[i + 1]), two(s.scale));
    const float2 mi = fma2(two(s.b1), make_float2(m[i], m[i + 1]), mul2(two(s.c1), gi));
    const float2 vi = fma2(two(s.b2), make_float2(v[i], v[i + 1]), mul2(mul2(two(s.c2), gi), gi));
    const float2 ri = make_float2(sqrt_approx(vi.x), sqrt_approx(vi.y)), under = fma2(ri, two(s.root), two(s.eps));
    const float2 pi = make_float2(p[i], p[i + 1]), ratio = mul2(mi, make_float2(rcp_fast(under.x), rcp_fast(under.y)));
    // (1 - lr wd, rounded to 32 bits by itself, would make a decay of 1e-6 one of 0.95e-6)
    const float2 by = fma2(pi, two(s.decay), mul2(two(s.size), ratio));
    m[i] = mi.x, m[i + 1] = mi.y, v[i] = vi.x, v[i + 1] = vi.y, r[i] = ri.x, r[i + 1] = ri.y, p[i] -= by.x, p[i + 1] -= by.y;
  }
  store_8<WIDE, V>(value, base, lane, t.n, p);
  if (t.master) store_8<WIDE>(t.param, t.type, base, lane, t.n, p);
  if constexpr (BITS == 32) {
    store_8<WIDE, float>(t.m, base, lane, t.n, m);
    store_8<WIDE, float>(t.v, base, lane, t.n, v);
  } else {
    uint32_t most_m = 0, most_r = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most_m = max(most_m, mag(m[i])), most_r = max(most_r, mag(r[i]));
    most_m = __reduce_max_sync(0xffffffffu, most_m);
    most_r = __reduce_max_sync(0xffffffffu, most_r);
    // as in a row of 8-bit values: a NaN or an infinity among the moments makes the scale NaN
    const bool ok_m = most_m < 0x7f800000u, ok_r = most_r < 0x7f800000u;
    const float nan = __uint_as_float(0x7fffffffu);
    float M = ok_m ? __uint_as_float(most_m) : nan, R = ok_r ? __uint_as_float(most_r) : nan;
    if (M < kTiny) M = 0.f;
    if (R < kTiny) R = 0.f;
    // 127 sqrt(|m| / M) as sqrt(|m| (127^2 / M)); 0 where there is no scale
    const float km = ok_m && M > 0.f ? 16129.f * rcp_fast(M) : 0.f, kr = ok_r && R > 0.f ? 65025.f * rcp_fast(R) : 0.f;
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 x = mul2(make_float2(m[i], m[i + 1]), two(km)), y = mul2(make_float2(r[i], r[i + 1]), two(kr));
      a[i] = copysignf(sqrt_fast(fabsf(x.x)), x.x), a[i + 1] = copysignf(sqrt_fast(fabsf(x.y)), x.y);
      // sqrt(v) is 0 or above 10^-23
      b[i] = fmaxf(sqrt_fast(y.x), __saturatef(r[i] * 1e30f)), b[i + 1] = fmaxf(sqrt_fast(y.y), __saturatef(r[i + 1] * 1e30f));
    }
    if constexpr (BITS == kUnbiased) {
      float2 dm[4], dv[4];
      dithers<WIDE>(base, lane, s.number, dm, dv);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        // the block's largest are 127 and 255 but for the approximate root, and no dither may take them beyond
        const float2 x = add2(make_float2(fminf(fmaxf(a[i], -127.f), 127.f), fminf(fmaxf(a[i + 1], -127.f), 127.f)), dm[i / 2]);
        const float2 y = add2(make_float2(fminf(b[i], 255.f), fminf(b[i + 1], 255.f)), dv[i / 2]);
        a[i] = x.x, a[i + 1] = x.y, b[i] = y.x, b[i + 1] = y.y;
      }
    }
    uint32_t qm[2], qv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      qm[h] = km > 0.f ? round_4(a[4 * h], a[4 * h + 1], a[4 * h + 2], a[4 * h + 3]) : 0u;
      qv[h] = kr > 0.f ? round_4(b[4 * h], b[4 * h + 1], b[4 * h + 2], b[4 * h + 3]) : 0u;
    }
    store_codes<WIDE>(t.m, base, lane, t.n, qm);
    store_codes<WIDE>(t.v, base, lane, t.n, qv);
    if (lane == 0) t.scales[base / kUnit] = make_float2(M, R);
  }
}

template <int BITS, typename G, typename V>
__device__ __forceinline__ void adam_item(const AdamTensor& t, int64_t base, int lane, const Step& s) {
  for (int k = 0; k < kItem && base < t.n; ++k, base += kUnit) {
    if (t.wide && base + kUnit <= t.n)
      adam_unit<BITS, true, G, V>(t, base, lane, s);
    else
      adam_unit<BITS, false, G, V>(t, base, lane, s);
  }
}
template <int BITS, typename G>
__device__ __forceinline__ void adam_item(const AdamTensor& t, int64_t base, int lane, const Step& s) {
  if (t.master || t.type == ASD_TYPE_F32)
    adam_item<BITS, G, float>(t, base, lane, s);
  else if (t.type == ASD_TYPE_BF16)
    adam_item<BITS, G, __nv_bfloat16>(t, base, lane, s);
  else
    adam_item<BITS, G, __half>(t, base, lane, s);
}

template <int BITS, int N>
__global__ void __launch_bounds__(kAdamBlock, kAdamSide) adamw_kernel(const __grid_constant__ AdamArgs<N> a) {
  dep_wait();
  dep_launch();
  const int lane = threadIdx.x & 31;
  if (a.skip && *a.skip != 0.f) return;
  const int64_t steps = *reinterpret_cast<volatile int64_t*>(a.step) + 1;
  if (a.advance) {
    // the last block to have read the number of steps moves it on
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      unsigned long long* ticket = reinterpret_cast<unsigned long long*>(a.step + 1);
      if (atomicAdd(ticket, 1ull) == gridDim.x - 1) {
        *reinterpret_cast<volatile int64_t*>(a.step) = steps;
        *reinterpret_cast<volatile int64_t*>(a.step + 1) = 0;
      }
    }
  }
  Step s;
  const float lr = a.lr_at ? *a.lr_at : a.lr;
  s.b1 = a.b1, s.c1 = a.c1, s.b2 = a.b2, s.c2 = a.c2, s.eps = a.eps;
  s.decay = lr * a.wd;
  // 1 - b^t = -expm1(t log b): a relative error of a few 2^-24, where the power and the difference would lose 1 / (1 - b) of that
  s.size = lr / -expm1f((float)steps * a.log_b1);
  s.root = 1.f / sqrtf(-expm1f((float)steps * a.log_b2));
  s.scale = a.grad_scale ? *a.grad_scale : 1.f;
  s.number = steps;
  const int warps = gridDim.x * (kAdamBlock / 32);
  int low = 0;  // tensor of the item: they come in ascending order
  for (int64_t item = blockIdx.x * (kAdamBlock / 32) + (threadIdx.x >> 5); item < a.items; item += warps) {
    if (low + 1 < a.count && item >= a.t[low + 1].first) {
      int high = a.count;  // first of `low` <= item, first of `high` beyond it
      while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (a.t[mid].first <= item)
          low = mid;
        else
          high = mid;
      }
    }
    const AdamTensor t = a.t[low];
    const int64_t base = (item - t.first) * (kItem * kUnit);
    if (t.grad_type == ASD_TYPE_BF16)
      adam_item<BITS, __nv_bfloat16>(t, base, lane, s);
    else if (t.grad_type == ASD_TYPE_F16)
      adam_item<BITS, __half>(t, base, lane, s);
    else
      adam_item<BITS, float>(t, base, lane, s);
  }
}

// The moments that 8-bit codes stand for.
struct MomentArgs {
  int64_t n;
  const void *m, *v;
  const float2* scales;
  void *m_out, *v_out;
  int type, wide;
};
__global__ void __launch_bounds__(kAdamBlock) moments_kernel(const MomentArgs a) {
  dep_wait();
  dep_launch();
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * (kAdamBlock / 32);
  for (int64_t unit = (int64_t)blockIdx.x * (kAdamBlock / 32) + (threadIdx.x >> 5); unit * kUnit < a.n; unit += warps) {
    float m[8], v[8];
    uint32_t qm[2], qv[2];
    const int64_t base = unit * kUnit;
    const float2 scale = a.scales[unit];
    if (a.wide && base + kUnit <= a.n) {
      load_codes<true>(a.m, base, lane, a.n, qm);
      load_codes<true>(a.v, base, lane, a.n, qv);
      moments_of(qm, qv, scale, m, v);
      store_8<true>(a.m_out, a.type, base, lane, a.n, m);
      store_8<true>(a.v_out, a.type, base, lane, a.n, v);
    } else {
      load_codes<false>(a.m, base, lane, a.n, qm);
      load_codes<false>(a.v, base, lane, a.n, qv);
      moments_of(qm, qv, scale, m, v);
      store_8<false>(a.m_out, a.type, base, lane, a.n, m);
      store_8<false>(a.v_out, a.type, base, lane, a.n, v);
    }
  }
}

bool on(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

template <int BITS, int N>
void launch_list(const asd_ops* o, const asd_adamw_args* q, const asd_adamw_tensor* t, int count, bool last, cudaStream_t st) {
  static_assert(sizeof(AdamArgs<N>) <= 32764, "arguments of a launch");
  AdamArgs<N> a;
  int64_t items = 0;
  a.count = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].n == 0) continue;
    AdamTensor& d = a.t[a.count++];
    d.param = t[i].param, d.grad = t[i].grad, d.master = t[i].master, d.m = t[i].m, d.v = t[i].v, d.scales = (float2*)t[i].scales;
    d.n = t[i].n, d.first = (int)items;
    d.type = (int16_t)t[i].type, d.grad_type = t[i].grad_type;
    d.wide = on(d.param, 16) && on(d.grad, 16) && on(d.master, 16) && on(d.m, BITS == 32 ? 16 : 8) && on(d.v, BITS == 32 ? 16 : 8);
    items += (d.n + kItem * kUnit - 1) / (kItem * kUnit);
  }
  a.items = (int)items, a.advance = last;
  a.b1 = (float)q->beta1, a.c1 = (float)(1 - q->beta1), a.b2 = (float)q->beta2, a.c2 = (float)(1 - q->beta2);
  // the kernel's reciprocal takes what is below the least normal number for 0, and 0 / 0 is not what a gradient of 0 is to give
  a.eps = q->eps > 0 ? std::max((float)q->eps, FLT_MIN) : 0.f, a.wd = (float)q->weight_decay, a.lr = (float)q->lr;
  a.log_b1 = (float)log(q->beta1), a.log_b2 = (float)log(q->beta2);
  a.lr_at = q->lr_device, a.grad_scale = q->grad_scale, a.skip = q->skip, a.step = q->step;
  const int64_t blocks = (items + kAdamBlock / 32 - 1) / (kAdamBlock / 32), most = kAdamBlocks<BITS> * (int64_t)o->num_sms;
  ops_launch(adamw_kernel<BITS, N>, dim3((unsigned)std::max<int64_t>(1, std::min(blocks, most))), dim3(kAdamBlock), 0, st, 1, a);
}
template <int BITS>
void launch_bits(const asd_ops* o, const asd_adamw_args* q, cudaStream_t st) {
  constexpr int kMost = 480;  // tensors of a launch
  int at = 0;
  do {
    const int n = std::min(kMost, q->count - at);
    const bool last = at + n == q->count;
    if (n <= 16)
      launch_list<BITS, 16>(o, q, q->tensors + at, n, last, st);
    else if (n <= 96)
      launch_list<BITS, 96>(o, q, q->tensors + at, n, last, st);
    else
      launch_list<BITS, kMost>(o, q, q->tensors + at, n, last, st);
    at += n;
  } while (at < q->count);
}

}  // namespace

void launch_adamw(const asd_ops* o, const asd_adamw_args* a, cudaStream_t st) {
  a->bits == 32 ? launch_bits<32>(o, a, st) : a->bits == 8 ? launch_bits<8>(o, a, st) : launch_bits<kUnbiased>(o, a, st);
}

void launch_moments(const asd_ops* o, const asd_adamw_moments_args* q, cudaStream_t st) {
  MomentArgs a{};
  a.n = q->n, a.m = q->m, a.v = q->v, a.scales = (const float2*)q->scales, a.m_out = q->m_out, a.v_out = q->v_out, a.type = q->type;
  a.wide = on(a.m, 8) && on(a.v, 8) && on(a.m_out, 16) && on(a.v_out, 16);
  const int64_t blocks = (q->n + 8 * kUnit - 1) / (8 * kUnit);
  ops_launch(moments_kernel, dim3((unsigned)std::min<int64_t>(blocks, 16 * (int64_t)o->num_sms)), dim3(kAdamBlock), 0, st, 1, a);
}

}  // namespace asd
