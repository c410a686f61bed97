// Matrix products with too few tiles to fill the SMs: C[m, n] = sum_k A(m, k) B(n, k) for some tens to hundreds of rows.
//
// A CTA owns 128 columns of C (GATE: 64, with the gate's and the value's weights for them) and up to 256 rows, and a
// cluster of 1 to 8 CTAs shares the sum over k.  The operands change places: the weights are the 128-row operand of
// tcgen05.mma and the rows of A the narrow one, so that few rows cost no padded tensor work and the 32 lanes of a warp
// store 32 neighbouring columns of a row of C.  Each CTA parks its partial sums in its own shared memory as
// [row of C][column]; after one cluster barrier every CTA adds up its share of the rows over distributed shared memory in
// the order of the ranks (the same bits in every run), applies the epilogue and stores.
//
// Measured: the gated MLP of 16 rows, 4096 x 8192 in 16 bits, 201 MB of weights in 40 us (5.0 TB/s) against 80 with tiles; int8
// 64 x 4096 x 4096 7.9 us against 14.7, 256 x 4096 x 4096 11.3 against 15.5; at 512 x 1024 x 4096 both take 8 and the tiles go on
// from there.  What bounds it beside the weights is a kernel's start, the join and the way of the operands into shared memory.
#include <string.h>

#include <algorithm>

#include "asd_ops_tc.cuh"

namespace asd {
namespace {

constexpr int kSplitThreads = 64 + 256;  // a TMA warp, an MMA warp, eight epilogue warps
constexpr int kMostStages = 8;
constexpr int kSmSmem = 228 * 1024;  // shared memory of an SM; a block costs 1 KB beside its own

struct SplitMaps {
  CUtensorMap w[2], x[2];
};
struct SplitArgs {
  int m, n;
  int kb[2];   // k-blocks of the first and of the second sum
  int nb;      // rows of C to a CTA: a multiple of 16
  int split;   // CTAs of a cluster
  int stages;
  int w_mn;    // the weights are read across k
  int early;   // the weights may be read before the previous kernel has ended
  int wide;    // address and row distance of the outputs are multiples of four elements
  uint32_t idesc, tmem_cols;
  int out_type, gelu;
  void* c[2];
  int64_t ldc;
  uint8_t* kept;
  int kept_cols;
  const float* scale_a;
  const float* scale_b;
  const float* bias;
  int* err;
};

__host__ __device__ constexpr int split_stage_bytes(int nb) { return (BM + nb) * 128; }

__device__ __forceinline__ uint4 ld_cluster_v4(uint32_t addr) {
  uint4 v;
  asm("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
template <bool I8>
__device__ __forceinline__ uint32_t add_bits(uint32_t a, uint32_t b) {
  return I8 ? a + b : __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
}
template <bool I8>
__device__ __forceinline__ void add4(uint4& a, uint4 b) {
  a = make_uint4(add_bits<I8>(a.x, b.x), add_bits<I8>(a.y, b.y), add_bits<I8>(a.z, b.z), add_bits<I8>(a.w, b.w));
}
// Four neighbouring 16-bit outputs; `wide`: rows and address are multiples of four elements.
__device__ __forceinline__ void store4(void* c, int64_t at, const float (&y)[4], int cols, bool wide, bool f16) {
  uint16_t* p = reinterpret_cast<uint16_t*>(c) + at;
  if (wide && cols == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack16(y[0], y[1], f16), pack16(y[2], y[3], f16));
  } else {
    for (int e = 0; e < cols; ++e) p[e] = round16(y[e], f16);
  }
}

template <int EPI>
__global__ void __launch_bounds__(kSplitThreads, 3)
split_kernel(const __grid_constant__ SplitMaps maps, const __grid_constant__ SplitArgs g) {
  constexpr bool I8 = EPI == OPS_I8;
  constexpr int F = EPI == OPS_GATE ? 64 : 128;  // columns of C to a CTA
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  const int stage_bytes = split_stage_bytes(g.nb);
  uint8_t* tiles_ptr = smem_raw + (tiles - raw);
  const int S = g.stages;
  uint8_t* aux = tiles_ptr + max(S * stage_bytes, g.nb * BM * 4);
  uint64_t* bars = reinterpret_cast<uint64_t*>(aux);  // full[S], empty[S], acc_full
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aux + 8 * (2 * S + 1));
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* row_scale = reinterpret_cast<float*>(aux + 256);  // I8: scale_a of the CTA's rows
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
  const uint32_t accf_bar = bar0 + 8u * (2 * S);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int n0 = ((int)blockIdx.x / g.split) * F;
  const int row0 = (int)blockIdx.y * g.nb;
  const int num_kb = g.kb[0] + g.kb[1];
  const int per = (num_kb + g.split - 1) / g.split;  // k-blocks [kb0, kb1) belong to this rank
  const int kb0 = min(rank * per, num_kb), kb1 = min(kb0 + per, num_kb);
  const uint32_t tmem_cols = g.tmem_cols;

  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.w[0]);
    prefetch_tmap(&maps.x[0]);
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(accf_bar, 1);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  if (!g.early) {
    grid_dependency_wait();
    grid_launch_dependents();  // the next kernel may fetch its weights beside this one
  }

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    if (lane == 0) {
      auto load_w = [&](int stage, int kb) {
        const int part = kb >= g.kb[0] ? 1 : 0;
        const int k0 = (kb - part * g.kb[0]) * (I8 ? 128 : 64);
        const uint32_t sw = tiles + stage * stage_bytes;
        mbar_expect_tx(full_bar(stage), (uint32_t)stage_bytes);
        if (EPI == OPS_GATE) {
          tma_load_2d(sw, &maps.w[0], full_bar(stage), k0, n0);
          tma_load_2d(sw + 64 * 128, &maps.w[1], full_bar(stage), k0, n0);
        } else if (!g.w_mn) {
          tma_load_2d(sw, &maps.w[part], full_bar(stage), k0, n0);
        } else {
          tma_load_2d(sw, &maps.w[part], full_bar(stage), n0, k0);
          tma_load_2d(sw + 8192, &maps.w[part], full_bar(stage), n0 + 64, k0);
        }
      };
      auto load_x = [&](int stage, int kb) {
        const int part = kb >= g.kb[0] ? 1 : 0;
        tma_load_2d(tiles + stage * stage_bytes + BM * 128, &maps.x[part], full_bar(stage), (kb - part * g.kb[0]) * (I8 ? 128 : 64), row0);
      };
      // the first stages are free: weights now, rows of A once the kernel that makes them has ended
      const int pre = min(S, kb1 - kb0);
      for (int i = 0; i < pre; ++i) load_w(i, kb0 + i);
      if (g.early) grid_dependency_wait();
      for (int i = 0; i < pre; ++i) load_x(i, kb0 + i);
      int stage = pre == S ? 0 : pre;
      uint32_t phase = pre == S ? 1u : 0u;
      for (int kb = kb0 + pre; kb < kb1; ++kb) {
        mbar_wait(empty_bar(stage), phase ^ 1u, dead, g.err);
        load_w(stage, kb);
        load_x(stage, kb);
        if (++stage == S) {
          stage = 0;
          phase ^= 1u;
        }
      }
      drain_after_timeout(dead);
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (lane == 0) {
      if (g.early) grid_dependency_wait();  // the limits of the waits below do not run while the previous kernel does
      const uint64_t step_w = desc_step(g.w_mn);
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        mbar_wait(full_bar(stage), phase, dead, g.err);
        tc_fence_after();
        const uint32_t sw = tiles + stage * stage_bytes;
        const uint64_t da = smem_desc(sw, g.w_mn), db = smem_desc(sw + BM * 128, false);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          tc_mma<I8, 1>(tmem_base, da + step_w * k, db + (uint64_t)(2 * k), g.idesc, (kb > kb0 || k > 0) ? 1u : 0u);
        tc_commit(empty_bar(stage));
        if (++stage == S) {
          stage = 0;
          phase ^= 1u;
        }
      }
      if (kb1 > kb0)
        tc_commit(accf_bar);
      else
        mbar_arrive(accf_bar);  // no k-block of its own: the partial is zero
    }
  } else {
    // ---- park this rank's partial sums as part[row][column] ----
    const int quarter = warp & 3, half = (warp - kEpiWarp0) >> 2;  // the two warps of a lane quarter take alternate groups of 16 rows
    const int feat = quarter * 32 + lane;
    if (g.early) grid_dependency_wait();
    if (I8) {
      for (int r = (int)threadIdx.x - 64; r < min(g.nb, g.m - row0); r += 256) row_scale[r] = g.scale_a[row0 + r];
    }
    mbar_wait(accf_bar, 0u, dead, g.err);
    tc_fence_after();
    uint32_t* part = reinterpret_cast<uint32_t*>(tiles_ptr);  // the stages are idle now
    for (int c0 = half * 16; c0 < g.nb; c0 += 32) {
      uint32_t r[16];
      if (kb1 > kb0) {
        tc_ld16(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c0, r);
        tc_wait_ld();
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) r[e] = 0u;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) part[(c0 + e) * BM + feat] = r[e];
    }
    tc_fence_before();
  }
  __syncthreads();
  __syncwarp();
  cluster_sync_all();  // every rank's partial sums are in place
  if (g.early) grid_launch_dependents();  // after the wait above: what the next one may read early is then complete

  if (warp >= kEpiWarp0) {
    // a thread adds up and stores four neighbouring columns, a warp whole rows of the tile
    const int tid = (int)threadIdx.x - 64;
    constexpr int kAcross = F / 4, kRows = 256 / kAcross;  // threads to a row, rows side by side
    const int f = 4 * (tid % kAcross), col = n0 + f;
    const int m = min(g.m - row0, g.nb);
    const bool f16 = g.out_type == ASD_TYPE_F16, gelu = g.gelu != 0;
    if (col < g.n) {
      const int cols = min(4, g.n - col);
      float sb[4] = {}, bb[4] = {};
      if (I8) {
        for (int e = 0; e < cols; ++e) {
          sb[e] = g.scale_b[col + e];
          if (g.bias) bb[e] = g.bias[col + e];
        }
      }
      constexpr int R = 2;  // rows whose loads are in flight together
      for (int lr0 = rank + (tid / kAcross) * g.split; lr0 < m; lr0 += R * kRows * g.split) {
        uint4 v[R], u[R];
        float p[R][4], s[R][4];  // GATE_GRAD: the kept factors
#pragma unroll
        for (int i = 0; i < R; ++i) {
          v[i] = u[i] = make_uint4(0u, 0u, 0u, 0u);
          if (EPI == OPS_GATE_GRAD) {
            const int row = row0 + min(lr0 + i * kRows * g.split, m - 1);
            const uint8_t* b = g.kept + kept_offset(row, col, g.kept_cols);
            kept_get4(b, row & 31, col & 31, p[i]);
            kept_get4(b + kKeptHalf, row & 31, col & 31, s[i]);
          }
        }
        for (int q = 0; q < g.split; ++q) {
          const uint32_t base = map_to_cta(tiles, (uint32_t)q) + (uint32_t)(4 * f);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const int lr = min(lr0 + i * kRows * g.split, m - 1);  // rows beyond the last are added up and not stored
            add4<I8>(v[i], ld_cluster_v4(base + (uint32_t)(lr * BM * 4)));
            if (EPI == OPS_GATE) add4<false>(u[i], ld_cluster_v4(base + (uint32_t)(lr * BM * 4 + 256)));
          }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const int row = row0 + lr0 + i * kRows * g.split;
          if (row >= row0 + m) break;
          float y[4] = {__uint_as_float(v[i].x), __uint_as_float(v[i].y), __uint_as_float(v[i].z), __uint_as_float(v[i].w)};
          const int64_t at = row * g.ldc + col;
          if (EPI == OPS_STORE) {
            store4(g.c[0], at, y, cols, g.wide, f16);
          } else if (EPI == OPS_GATE) {
            float w[4] = {__uint_as_float(u[i].x), __uint_as_float(u[i].y), __uint_as_float(u[i].z), __uint_as_float(u[i].w)};
            float h[4];
            gated(y, w, h, gelu, g.kept != nullptr);
            if (g.kept) {
              uint8_t* b = g.kept + kept_offset(row, col, g.kept_cols);
              kept_put4(b, row & 31, col & 31, y);
              kept_put4(b + kKeptHalf, row & 31, col & 31, w);
            }
            store4(g.c[0], at, h, cols, g.wide, f16);
          } else if (EPI == OPS_GATE_GRAD) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[i][e] *= y[e];
              s[i][e] *= y[e];
            }
            store4(g.c[0], at, p[i], cols, g.wide, f16);
            store4(g.c[1], at, s[i], cols, g.wide, f16);
          } else {
            const float sa = row_scale[row - row0];
            const int k[4] = {(int)v[i].x, (int)v[i].y, (int)v[i].z, (int)v[i].w};
            float z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = fmaf((float)k[e] * sa, sb[e], bb[e]);
            if (g.out_type == ASD_TYPE_F32) {
              float* p = reinterpret_cast<float*>(g.c[0]) + at;
              if (g.wide && cols == 4)
                *reinterpret_cast<float4*>(p) = make_float4(z[0], z[1], z[2], z[3]);
              else
                for (int e = 0; e < cols; ++e) p[e] = z[e];
            } else {
              store4(g.c[0], at, z, cols, g.wide, f16);
            }
          }
        }
      }
    }
  }

  // no CTA leaves while a peer may still read its partial sums
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(tmem_cols) : "memory");
  }
}

uint32_t split_tmem_cols(int nb) { return nb <= 32 ? 32u : (nb <= 64 ? 64u : (nb <= 128 ? 128u : 256u)); }
// Shared memory of a CTA: at least as large a share of the SM's 228 KB as it takes of the 512 tensor-memory columns (452
// bytes a column next to the 1 KB that every block costs).  CTAs that fit an SM together then never wait for one another's
// tensor memory, which the members of a cluster, who wait for one another anyway, must not do.
int split_smem(int nb, int stages) {
  return std::max(std::max(stages * split_stage_bytes(nb), nb * BM * 4) + 1024 + 256 + 1024, (int)split_tmem_cols(nb) * 452);
}

template <int EPI>
asd_status launch_split(const asd_ops* o, const OpsGemm& q, const SplitPlan& p, bool early, cudaStream_t st) {
  constexpr bool I8 = EPI == OPS_I8;
  constexpr int F = EPI == OPS_GATE ? 64 : 128;
  SplitMaps maps;
  memset(&maps, 0, sizeof(maps));
  SplitArgs g{};
  const int ke = I8 ? 128 : 64;
  g.m = (int)q.m, g.n = (int)q.n;
  g.kb[0] = (int)((q.k[0] + ke - 1) / ke);
  g.kb[1] = q.parts == 2 ? (int)((q.k[1] + ke - 1) / ke) : 0;
  g.nb = p.nb, g.split = p.split, g.stages = p.stages;
  g.tmem_cols = split_tmem_cols(p.nb);
  g.w_mn = q.b[0].mn;
  g.early = early;
  const int es4 = 4 * ops_type_size(q.type);
  g.wide = q.ldc % 4 == 0 && (uintptr_t)q.c[0] % es4 == 0 && (uintptr_t)q.c[1] % es4 == 0;
  const uint32_t fmt = I8 ? 1u : (q.type == ASD_TYPE_BF16 ? 1u : 0u);
  g.idesc = (I8 ? 2u << 4 : 1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)g.w_mn << 15) | ((uint32_t)(p.nb >> 3) << 17) |
            ((uint32_t)(BM >> 4) << 24);
  g.out_type = q.type, g.gelu = q.act == ASD_ACT_GELU;
  g.c[0] = q.c[0], g.c[1] = q.c[1], g.ldc = q.ldc;
  g.kept = q.kept, g.kept_cols = (int)((q.n + 31) / 32);
  g.scale_a = q.scale_a, g.scale_b = q.scale_b, g.bias = q.bias;
  g.err = o->err;
  bool ok = true;  // only the maps that the kernel reads
  for (int i = 0; i < (EPI == OPS_GATE ? 2 : q.parts); ++i) ok = ok && encode_operand(&maps.w[i], q.b[i], q.type, I8, F);
  for (int i = 0; i < q.parts; ++i) ok = ok && encode_operand(&maps.x[i], q.a[i], q.type, I8, p.nb);
  if (!ok) return ops_fail(ASD_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  const dim3 grid((unsigned)((q.n + F - 1) / F * p.split), (unsigned)((q.m + p.nb - 1) / p.nb));
  ops_launch(split_kernel<EPI>, grid, dim3(kSplitThreads), (size_t)split_smem(p.nb, p.stages), st, p.split, maps, g);
  return ops_launched("split matrix product");
}

template <int EPI>
cudaError_t prepare_split() {
  return cudaFuncSetAttribute(split_kernel<EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448);
}

}  // namespace

// The cheapest way to split, by an estimate in clocks that was fitted to 13 shapes of 16 to 2000 rows (int8 and 16 bits, k
// 208 to 8192, out 1000 to 16384), each with every split; what it picks is within 10 % of the best of them.  A CTA's
// k-blocks cost the largest of its MMAs' time (2 clocks a row), its operands' way into shared memory (64 bytes a clock and
// SM) and the weights' way from memory (23 bytes a clock and SM that has a CTA).  Parking, adding up and storing cost 37
// clocks a row; a launch 3000 and each wave of CTAs 4000; joining a cluster 2500 more, and one of eight, which the GPU finds
// room for slowly, 9000 unless that is hidden under the kernel before (`early`).
SplitPlan plan_split(const asd_ops* o, const OpsGemm& q, bool early) {
  const int ke = q.epi == OPS_I8 ? 128 : 64, F = q.epi == OPS_GATE ? 64 : 128, m = (int)q.m, sms = o->num_sms;
  const int kb = (int)((q.k[0] + ke - 1) / ke + (q.parts == 2 ? (q.k[1] + ke - 1) / ke : 0));
  const int tiles_n = (int)((q.n + F - 1) / F);
  const float weights = (float)tiles_n * kb * (BM * 128);
  SplitPlan best{16, 1, 2, 1e30};
  int side_of_best = 1, share_of_best = kb;
  int last = 0;  // CTAs along the rows of the candidate before: of several heights with the same number the least one counts
  for (int nb = 16; nb <= 256; nb += 16) {
    const int tiles_m = (m + nb - 1) / nb;
    if (tiles_m == last) continue;
    last = tiles_m;
    for (int split = 1; split <= 8; split *= 2) {
      if (split > 1 && kb < 2 * split) break;
      const int64_t all = (int64_t)tiles_n * tiles_m * split;
      if (all > 1 << 20) break;
      const int ctas = (int)all, share = (kb + split - 1) / split;
      // CTAs that run side by side on an SM
      int side = std::min(3, (ctas + sms - 1) / sms);
      while (side > 1 && side * (split_smem(nb, 2) + 1024) > kSmSmem) --side;
      const int waves = (ctas + side * sms - 1) / (side * sms);
      const float fill = side * (BM + nb) * 2.f, math = side * std::max(128.f, 2.f * nb);
      const float stream = weights / (23.f * std::min(ctas, sms)) / waves;
      const float join = split == 8 && !early ? 9000.f : split > 1 ? 2500.f : 0.f;
      const float c = 3000.f + waves * (4000.f + join + std::max(stream, share * std::max(fill, math)) + 37.f * nb / split);
      if (c < best.clocks) {
        best = SplitPlan{nb, split, 2, c};
        side_of_best = side;
        share_of_best = share;
      }
    }
  }
  // few rows: no more than half of the SM's shared memory, which leaves room for the next kernel's first weights
  best.stages = std::min(best.nb <= 64 ? 112 * 1024 / split_stage_bytes(best.nb) : kMostStages, std::max(2, share_of_best));
  best.stages = std::min(best.stages, kMostStages);
  while (best.stages > 2 && side_of_best * (split_smem(best.nb, best.stages) + 1024) > kSmSmem) --best.stages;
  return best;
}

asd_status ops_gemm_split(const asd_ops* o, const OpsGemm& q, const SplitPlan& p, bool early, cudaStream_t st) {
  switch (q.epi) {
    case OPS_STORE: return launch_split<OPS_STORE>(o, q, p, early, st);
    case OPS_GATE: return launch_split<OPS_GATE>(o, q, p, early, st);
    case OPS_GATE_GRAD: return launch_split<OPS_GATE_GRAD>(o, q, p, early, st);
    default: return launch_split<OPS_I8>(o, q, p, early, st);
  }
}

asd_status ops_split_prepare() {
  for (cudaError_t e : {prepare_split<OPS_STORE>(), prepare_split<OPS_GATE>(), prepare_split<OPS_GATE_GRAD>(), prepare_split<OPS_I8>()})
    if (e != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  return ASD_OK;
}

}  // namespace asd
