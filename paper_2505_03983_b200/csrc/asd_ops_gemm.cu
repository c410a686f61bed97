// The matrix products of the gated MLP and of the 8-bit projection on the 5th-generation tensor cores:
//   C[m, n] = sum_k A(m, k) B(n, k)
// with either operand read along k (a row-major matrix [m or n, k]) or across it (the transpose of a row-major [k, m or n]),
// so that the three products of a gradient need no transposed copy.
//
// op_pair_kernel: a cluster of two CTAs computes a 256 x BN tile with tcgen05.mma.cta_group::2.  In each CTA one thread
// loads its own 128 rows of A and BN / 2 rows of B by TMA, one thread of the first CTA issues the MMAs, and eight warps
// take the CTA's 128 x BN accumulator out of tensor memory, which is double-buffered: a tile's epilogue runs under the next
// tile's MMAs.  Clusters are persistent and walk over the tiles in bands of eight tile rows, so that the tiles that are in
// flight together share their operands in L2.
//
// Epilogues, on the fp32 (8-bit products: int32) accumulator:
//   STORE      C rounded to 16 bits
//   GATE       the tile holds BN / 2 columns of g and the same columns of u (one CTA of the pair loads the gate's weights,
//              the other the value's): h = act(g) u, and its two derivatives kept for the backward pass
//   GATE_GRAD  C = dh: dg = dh u act'(g), du = dh act(g), from the two factors that were kept
//   I8         C scale_a[m] scale_b[n] + bias[n], rounded to the output's type
//   LINEAR     residual + act(C + bias[n]), act' kept for the backward pass.  The residual comes by TMA into the buffers that the
//              outputs leave from, the tile's first two pieces of it under the tile's MMAs
// Measured at 8192 x 2048 x 8192 in bf16, one launch at 1.6 GHz: gate 391 to 420 us with what is kept (1.3 PFLOP/s), h Wo 205 to 223
// (1.2 to 1.3), gate gradient 213 to 228, the three gradient products 1.0 ms (1.3 to 1.35); int8 8192 x 4096 x 8192 216 to 225 us
// (2.5 POP/s); a linear layer of 8192 x 4096 x 4096 190 us (1.45 PFLOP/s), with SiLU, residual and the kept act' 211, its two gradient
// products 404.  A k-block of a 256 x 256 tile takes some 650 clocks: its MMAs 512, but its 80 KB of shared memory traffic 640.  In
// a loop the power limit bounds all of them (988 W at 1.4 to 1.5 GHz).  Twice as high tiles (512 x 256) need fewer bytes and take
// longer (383 against 335 thousand clocks).
// An output whose address and row distance are multiples of 16 bytes leaves through shared memory by TMA stores of 128-byte
// row pieces; the others are staged in the same way and stored by lanes on neighbouring elements.
#include <limits.h>
#include <string.h>

#include <algorithm>

#include "asd_ops_tc.cuh"

namespace asd {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn();  // asd_gemm.cu

namespace {

constexpr int kStoreBytes = 32 * 128;  // a warp's staging buffer: 32 rows of 128 bytes
constexpr int kBand = 8;               // tile rows that are walked over together
constexpr int kPartBlock = 32 * 32;    // partial sums of a block

// One product of a launch.
struct PairProduct {
  int m, n;       // of C (GATE: n = hidden)
  int kb[2];      // k-blocks of the first and of the second sum
  int tiles_m, tiles_n;
  int first;      // number of its first unit in the launch: a tile, or one slice of a tile's sum
  int slices, per;  // slices of the sum, k-blocks of one
  float* part;      // slices > 1: [slice][32 rows of C][32 columns of C] blocks of partial sums
  int a_mn, b_mn;
  uint32_t idesc;
  int tma_store;
  void* c;
  int64_t ldc;
};
template <int N>
struct PairMaps {
  struct One {
    CUtensorMap a[2], b[2], c[2];
  } p[N];
};
template <int N>
struct PairArgs {
  PairProduct p[N];
  int units;      // of all products
  int out_type;   // asd_type
  int gelu;
  uint8_t* kept;
  int kept_cols;  // blocks of 32 columns
  const float* scale_a;
  const float* scale_b;
  const float* bias;
  const float* unscale;  // OPS_STORE: what the sums are multiplied by, or NULL
  int* err;
  // OPS_LINEAR
  int f16;        // the operands are F16, not BF16
  int b1_f32;
  const void* b1;
  const void* res;
  int64_t ldr;
  int res_tma;    // the residual can be read by TMA (map c[1])
};
// OPS_STORE products come in lists.
template <int EPI>
constexpr int products_of = EPI == OPS_STORE ? kMostProducts : 1;

template <int BN, int EPI>
struct OpPairCfg {
  static constexpr int kStageBytes = (BM + BN / 2) * 128;  // per CTA: 128 rows of A, BN / 2 of B, 128 bytes each
  static constexpr int kBufs = 2;  // staging buffers of a warp: one is filled while the other's store reads it
  // 4, 5 and 6 stages of 256 columns take the same time (8192 x 2048 x 8192: 386, 380 and 380 thousand clocks)
  static constexpr int kStages = BN == 256 ? (EPI == OPS_LINEAR ? 4 : 5) : 6;
  static constexpr int kBiasBytes = EPI == OPS_LINEAR ? kPairEpiWarps * (BN / 2) * 4 : 0;  // LINEAR: of every warp's columns
  static constexpr int kTmemCols = 2 * BN;
  static constexpr int kSmemBytes = kStages * kStageBytes + kPairEpiWarps * kBufs * kStoreBytes + kBiasBytes + 1024 + 512;
  static_assert(kSmemBytes <= 232448, "shared memory of a CTA");
};

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A warp's staging buffer, 32 rows of 128 bytes with the 128-byte swizzle of the store's tensor map: 16-byte piece `i` of
// row `lane`.  Eight neighbouring lanes write eight different pieces of the banks.
__device__ __forceinline__ void stage_put(uint8_t* buf, int lane, int i, uint4 v) {
  *reinterpret_cast<uint4*>(buf + lane * 128 + ((i ^ (lane & 7)) << 4)) = v;
}
// A warp's two buffers.  They change places whenever a store is issued from one, so that all but the last store have read
// theirs when the other is needed again.
struct Staging {
  uint8_t* first;
  uint32_t first_addr;
  int lane, cur;
  __device__ __forceinline__ uint8_t* buf() const { return first + cur * kStoreBytes; }
  __device__ __forceinline__ uint32_t addr() const { return first_addr + cur * kStoreBytes; }
  // The current buffer may be written (LEFT = 0: both).
  template <int LEFT = 1>
  __device__ __forceinline__ void free() const {
    if (lane == 0) bulk_wait_read<LEFT>();
    __syncwarp();
  }
  __device__ __forceinline__ void send(const CUtensorMap* map, int x, int y, bool any) {
    fence_async_shared();
    __syncwarp();
    if (!any) return;
    if (lane == 0) {
      tma_store_2d(map, addr(), x, y);
      bulk_commit();
    }
    cur ^= 1;
  }
};
// The staged rows for outputs that the TMA cannot address: a row at a time, lanes on neighbouring elements.  (Pairs of them
// as words, shifted by one where a row starts in the middle of a word, take longer: 45 against 41 us in a training step.)
__device__ __forceinline__ void rows_out16(const uint8_t* buf, void* c, int64_t ldc, int lane, int row0, int col0, int m, int n) {
  __syncwarp();
  uint16_t* p = reinterpret_cast<uint16_t*>(c) + row0 * ldc + col0 + lane;
  const int rows = min(32, m - row0);
  const bool first = col0 + lane < n, second = col0 + 32 + lane < n;
#pragma unroll 8
  for (int r = 0; r < rows; ++r, p += ldc) {
    const uint8_t* q = buf + r * 128 + 2 * (lane & 7);
    const int piece = lane >> 3;
    if (first) p[0] = *reinterpret_cast<const uint16_t*>(q + ((piece ^ (r & 7)) << 4));
    if (second) p[32] = *reinterpret_cast<const uint16_t*>(q + (((piece + 4) ^ (r & 7)) << 4));
  }
  __syncwarp();
}
__device__ __forceinline__ void rows_out32(const uint8_t* buf, void* c, int64_t ldc, int lane, int row0, int col0, int m, int n) {
  __syncwarp();
  uint32_t* p = reinterpret_cast<uint32_t*>(c) + row0 * ldc + col0;
  const int rows = min(32, m - row0);
#pragma unroll 8
  for (int r = 0; r < rows; ++r, p += ldc)
    if (col0 + lane < n) p[lane] = *reinterpret_cast<const uint32_t*>(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + 4 * (lane & 3));
  __syncwarp();
}
// The other way: 32 rows of 128 bytes from memory that the TMA cannot address into a staging buffer.
template <int ES>
__device__ __forceinline__ void rows_in(uint8_t* buf, const void* c, int64_t ldc, int lane, int row0, int col0, int m, int n) {
  const int rows = min(32, m - row0);
#pragma unroll 8
  for (int r = 0; r < rows; ++r) {
    if constexpr (ES == 4) {
      if (col0 + lane < n)
        *reinterpret_cast<uint32_t*>(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + 4 * (lane & 3)) =
            reinterpret_cast<const uint32_t*>(c)[(row0 + r) * ldc + col0 + lane];
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(c) + (row0 + r) * ldc + col0 + lane;
      uint8_t* q = buf + r * 128 + 2 * (lane & 7);
      const int piece = lane >> 3;
      if (col0 + lane < n) *reinterpret_cast<uint16_t*>(q + ((piece ^ (r & 7)) << 4)) = p[0];
      if (col0 + 32 + lane < n) *reinterpret_cast<uint16_t*>(q + (((piece + 4) ^ (r & 7)) << 4)) = p[32];
    }
  }
  __syncwarp();
}
__device__ __forceinline__ uint4 stage_get(const uint8_t* buf, int lane, int i) {
  return *reinterpret_cast<const uint4*>(buf + lane * 128 + ((i ^ (lane & 7)) << 4));
}
__device__ __forceinline__ void stage_half(uint8_t* buf, int lane, int half, const uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) stage_put(buf, lane, 4 * half + i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
}

// A unit of a launch: a tile, or the slice [kb0, kb1) of its sum.
struct Tile {
  int product, m0, n0, slice, kb0, kb1;
};
template <int BN, int N>
__device__ __forceinline__ Tile tile_at(const PairArgs<N>& g, int t) {
  Tile r;
  r.product = 0;
  for (int i = 1; i < N; ++i)
    if (t >= g.p[i].first) r.product = i;
  const PairProduct& p = g.p[r.product];
  t -= p.first;
  const int tiles = p.tiles_m * p.tiles_n;
  r.slice = p.slices > 1 ? t / tiles : 0;  // the tiles of one slice are in flight together
  t -= r.slice * tiles;
  r.kb0 = r.slice * p.per;
  r.kb1 = min(r.kb0 + p.per, p.kb[0] + p.kb[1]);
  const int band = t / (kBand * p.tiles_n), first = band * kBand;
  const int rows = min(p.tiles_m - first, kBand), in = t - first * p.tiles_n;
  r.m0 = (first + in % rows) * 2 * BM;
  r.n0 = (in / rows) * BN;
  return r;
}

// 64 columns of a warp's 32 rows of partial sums, as two blocks: float4 number `i` of row `lane` at 32 i + lane, so that both
// this store and the load of join_kernel are contiguous over the lanes.
__device__ __forceinline__ void part_out(const PairProduct& p, int slice, int row0, int col0, uint32_t acc, int lane) {
  const int blocks_m = (p.m + 31) / 32, blocks_n = (p.n + 31) / 32;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t r[32];
    tc_ld32(acc + 32 * h, r);
    tc_wait_ld();
    if (row0 >= p.m || col0 + 32 * h >= p.n) continue;
    const int64_t block = ((int64_t)slice * blocks_m + row0 / 32) * blocks_n + col0 / 32 + h;
    uint4* to = reinterpret_cast<uint4*>(p.part + block * kPartBlock) + lane;
#pragma unroll
    for (int i = 0; i < 8; ++i) to[32 * i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
  }
}

// ACT: the activation of LINEAR, whose epilogue takes 16 columns at a time in a loop that is not unrolled.
template <int BN, int EPI, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
op_pair_kernel(const __grid_constant__ PairMaps<products_of<EPI>> maps, const __grid_constant__ PairArgs<products_of<EPI>> g) {
  using C = OpPairCfg<BN, EPI>;
  constexpr int S = C::kStages;
  constexpr bool I8 = EPI == OPS_I8;
  // columns of C to a tile: half of the accumulator's where it holds g and u
  constexpr int CN = EPI == OPS_GATE ? BN / 2 : BN;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;
  uint8_t* stage_ptr = smem_raw + (tiles - raw) + S * C::kStageBytes;
  uint8_t* aux = stage_ptr + kPairEpiWarps * C::kBufs * kStoreBytes + C::kBiasBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(aux);  // full[S], empty[S], acc_full[2], acc_empty[2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(aux + 8 * (2 * S + 4));
  volatile int* dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t bar0 = smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
  auto accf_bar = [&](int b) { return bar0 + 8u * (2 * S + b); };
  auto acce_bar = [&](int b) { return bar0 + 8u * (2 * S + 2 + b); };
  auto res_bar = [&](int w, int b) { return bar0 + 8u * (2 * S + 6 + 2 * w + b); };  // LINEAR: a warp's buffers
  static_assert(8 * (2 * S + 6 + 2 * kPairEpiWarps) <= 512, "barriers");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
  const int n_tiles = g.units;

  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.p[0].a[0]);
    prefetch_tmap(&maps.p[0].b[EPI == OPS_GATE ? rank : 0]);
    for (int s = 0; s < S; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 2 * kPairEpiWarps);  // every epilogue warp of both CTAs
    }
    if (EPI == OPS_LINEAR)
      for (int w = 0; w < kPairEpiWarps; ++w) mbar_init(res_bar(w, 0), 1), mbar_init(res_bar(w, 1), 1);
    *dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"((uint32_t)C::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();  // the peer's barriers are initialised before anything arrives on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  grid_dependency_wait();
  grid_launch_dependents();

  if (warp == 0) {
    // ---------------- TMA producer (both CTAs) ----------------
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int t = pair; t < n_tiles; t += n_pairs) {
        const Tile tile = tile_at<CN>(g, t);
        const PairProduct& p = g.p[tile.product];
        const auto& mp = maps.p[tile.product];
        const bool a_mn = p.a_mn, b_mn = p.b_mn;
        const int m0 = tile.m0 + (int)rank * BM;
        const int n0 = EPI == OPS_GATE ? tile.n0 : tile.n0 + (int)rank * (BN / 2);
        for (int kb = tile.kb0; kb < tile.kb1; ++kb) {
          const int part = kb >= p.kb[0] ? 1 : 0;
          const int k0 = (kb - part * p.kb[0]) * (I8 ? 128 : 64);
          const CUtensorMap* ma = &mp.a[part];
          const CUtensorMap* mb = &mp.b[EPI == OPS_GATE ? (int)rank : part];
          mbar_wait(empty_bar(stage), phase ^ 1u, dead, g.err);
          const uint32_t sa = tiles + stage * C::kStageBytes;
          const uint32_t sb = sa + BM * 128;
          const uint32_t full0 = map_to_cta(full_bar(stage), 0);
          if (rank == 0) mbar_expect_tx(full_bar(stage), 2u * (uint32_t)C::kStageBytes);
          if (!a_mn) {
            tma_load_2d_pair(sa, ma, full0, k0, m0);
          } else {
            tma_load_2d_pair(sa, ma, full0, m0, k0);
            tma_load_2d_pair(sa + 8192, ma, full0, m0 + 64, k0);
          }
          if (!b_mn) {
            tma_load_2d_pair(sb, mb, full0, k0, n0);
          } else {
#pragma unroll
            for (int i = 0; i < BN / 128; ++i) tma_load_2d_pair(sb + 8192 * i, mb, full0, n0 + 64 * i, k0);
          }
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      drain_after_timeout(dead);
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (rank 0 only) ----------------
    if (rank == 0 && lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int it = 0;
      for (int t = pair; t < n_tiles; t += n_pairs, ++it) {
        const Tile tile = tile_at<CN>(g, t);
        const PairProduct& p = g.p[tile.product];
        const bool a_mn = p.a_mn, b_mn = p.b_mn;
        const uint64_t step_a = desc_step(a_mn), step_b = desc_step(b_mn);
        const uint32_t idesc = p.idesc;
        const int acc = it & 1;
        const uint32_t acc_phase = (uint32_t)(it >> 1) & 1u;
        mbar_wait(acce_bar(acc), acc_phase ^ 1u, dead, g.err);  // both CTAs' epilogues have drained it
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * BN);
        for (int kb = tile.kb0; kb < tile.kb1; ++kb) {
          mbar_wait(full_bar(stage), phase, dead, g.err);
          tc_fence_after();
          const uint32_t sa = tiles + stage * C::kStageBytes;
          const uint64_t da = smem_desc(sa, a_mn), db = smem_desc(sa + BM * 128, b_mn);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc_mma<I8, 2>(d_tmem, da + step_a * k, db + step_b * k, idesc, kb > tile.kb0 || k > 0 ? 1u : 0u);
          tc_commit_pair(empty_bar(stage));                 // frees the stage in this CTA ...
          tc_commit_pair(map_to_cta(empty_bar(stage), 1));  // ... and in the peer
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
        tc_commit_pair(accf_bar(acc));
        tc_commit_pair(map_to_cta(accf_bar(acc), 1));
      }
    }
  } else {
    // ---------------- epilogue warps (both CTAs, own 128 rows) ----------------
    const int quarter = warp & 3;
    const int half = (warp - kEpiWarp0) >> 2;  // of the tile's columns
    const bool f16 = g.out_type == ASD_TYPE_F16;
    const bool gelu = g.gelu != 0;
    const bool scales_wide = (((uintptr_t)g.scale_b | (uintptr_t)g.bias) & 15) == 0;
    uint8_t* const bufs = stage_ptr + (warp - kEpiWarp0) * C::kBufs * kStoreBytes;
    Staging out{bufs, smem_u32(bufs), lane, 0};
    constexpr int kUnits = CN / 64;  // of 64 columns; a tile of one is the first four warps'
    constexpr int kMine = kUnits >= 2 ? kUnits / 2 : 1;
    uint32_t res_phase = 0;  // LINEAR: a bit for each of the warp's buffers
    const bool out32 = EPI == OPS_LINEAR && g.out_type == ASD_TYPE_F32;
    float* const bias = reinterpret_cast<float*>(aux - C::kBiasBytes) + (warp - kEpiWarp0) * (BN / 2);  // LINEAR: of the warp's columns
    int it = 0;
    for (int t = pair; t < n_tiles; t += n_pairs, ++it) {
      const Tile tile = tile_at<CN>(g, t);
      const PairProduct& p = g.p[tile.product];
      const auto& mp = maps.p[tile.product];
      const int m = p.m, n = p.n;
      const bool tma = p.tma_store;
      const int row0 = tile.m0 + (int)rank * BM + quarter * 32;
      const int row = row0 + lane;
      const int acc = it & 1;
      const uint32_t acc_phase = (uint32_t)(it >> 1) & 1u;
      const uint32_t t0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * BN);
      const bool rows_any = row0 < m;
      float sa = 0.f;
      if (I8 && row < m) sa = g.scale_a[row];
      uint4 kept[2][6];  // GATE_GRAD: the factors of the 32 columns that come next
      auto fetch_kept = [&](int col) {
        if (rows_any && col < n) {
          const uint8_t* b = g.kept + kept_offset(row0, col, g.kept_cols);
          kept_fetch(b, lane, kept[0]);
          kept_fetch(b + kKeptHalf, lane, kept[1]);
        }
      };
      if (EPI == OPS_GATE_GRAD) fetch_kept(tile.n0 + half * kMine * 64);
      // LINEAR: piece i of the warp's columns is what a buffer holds, 64 columns in 16 bits or 32 in 32; those with a column of C take
      // the buffers in turn
      const int piece = out32 ? 32 : 64, pieces = kMine * 64 / piece;
      auto load_res = [&](int i, int b) {
        const int col = tile.n0 + half * kMine * 64 + i * piece;
        if (lane == 0 && i < pieces && col < n) {
          mbar_expect_tx(res_bar(warp - kEpiWarp0, b), kStoreBytes);
          tma_load_2d(out.first_addr + b * kStoreBytes, &mp.c[1], res_bar(warp - kEpiWarp0, b), col, row0);
        }
      };
      if (EPI == OPS_LINEAR) {
        if (g.res_tma && rows_any) {
          fence_async_shared();  // what was read from the buffers in the tile before
          out.free<0>();
          load_res(0, out.cur);
          load_res(1, out.cur ^ 1);
        }
        __syncwarp();  // the bias of the tile before has been read
#pragma unroll
        for (int i = 0; i < BN / 2; i += 32) {
          const int col = tile.n0 + half * kMine * 64 + i + lane;
          bias[i + lane] = g.b1 && col < n ? load_scalar(g.b1, col, g.b1_f32, g.f16) : 0.f;
        }
        __syncwarp();
      }
      mbar_wait(accf_bar(acc), acc_phase, dead, g.err);
      tc_fence_after();
      if constexpr (EPI == OPS_LINEAR) {
        const int first = tile.n0 + half * kMine * 64;  // the warp's columns
        const int per = out32 ? 2 : 4;                  // steps of 16 columns to a buffer
        uint32_t next_r[16];                            // the next columns' sums are on their way while these are worked on
        const uint32_t ta = t0 + half * kMine * 64;
        tc_ld16(ta, next_r);
#pragma unroll 1
        for (int i = 0; i < 4 * kMine; ++i) {
          const int col = first + 16 * i, in = i & (per - 1);
          const bool some = rows_any && first + 16 * (i - in) < n;  // of the buffer's columns
          float z[16], da[16];
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e] = __uint_as_float(next_r[e]);
          if (i + 1 < 4 * kMine) tc_ld16(ta + 16 * (i + 1), next_r);
          uint8_t* const buf = out.buf();
          if (in == 0) {
            if (g.res_tma) {
              if (some) {
                mbar_wait(res_bar(warp - kEpiWarp0, out.cur), (res_phase >> out.cur) & 1u, dead, g.err);
                res_phase ^= 1u << out.cur;
              }
            } else {
              if (tma) out.free();
              if (g.res && rows_any) {
                if (out32)
                  rows_in<4>(buf, g.res, g.ldr, lane, row0, col, m, n);
                else
                  rows_in<2>(buf, g.res, g.ldr, lane, row0, col, m, n);
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 b = *reinterpret_cast<const float4*>(bias + 16 * i + e);
            z[e] += b.x, z[e + 1] += b.y, z[e + 2] += b.z, z[e + 3] += b.w;
          }
          activated<ACT>(z, da, g.kept != nullptr);
          if (g.kept && rows_any && col < n) {
            float4* to = reinterpret_cast<float4*>(slope_block(reinterpret_cast<float*>(g.kept), row0, col, g.kept_cols)) + lane + 8 * (col & 31);
#pragma unroll
            for (int e = 0; e < 4; ++e) to[32 * e] = make_float4(da[4 * e], da[4 * e + 1], da[4 * e + 2], da[4 * e + 3]);
          }
          if (out32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint4 o = make_uint4(0u, 0u, 0u, 0u);
              if (g.res) o = stage_get(buf, lane, 4 * in + e);
              stage_put(buf, lane, 4 * in + e,
                        make_uint4(__float_as_uint(__uint_as_float(o.x) + z[4 * e]), __float_as_uint(__uint_as_float(o.y) + z[4 * e + 1]),
                                   __float_as_uint(__uint_as_float(o.z) + z[4 * e + 2]), __float_as_uint(__uint_as_float(o.w) + z[4 * e + 3])));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint32_t o[4] = {0u, 0u, 0u, 0u};
              if (g.res) *reinterpret_cast<uint4*>(o) = stage_get(buf, lane, 2 * in + e);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float2 x = unpack16(o[k], g.f16);
                o[k] = pack16(x.x + z[8 * e + 2 * k], x.y + z[8 * e + 2 * k + 1], g.f16);
              }
              stage_put(buf, lane, 2 * in + e, make_uint4(o[0], o[1], o[2], o[3]));
            }
          }
          if (in + 1 < per || !some) continue;
          const int from = col - 16 * in, b = out.cur;
          if (tma) {
            out.send(&mp.c[0], from, row0, true);
          } else {
            if (out32)
              rows_out32(buf, p.c, p.ldc, lane, row0, from, m, n);
            else
              rows_out16(buf, p.c, p.ldc, lane, row0, from, m, n);
            out.cur ^= 1;
          }
          const int next = (from - first) / piece + 2;
          if (g.res_tma && next < pieces) {
            fence_async_shared();
            out.free<0>();
            load_res(next, b);
          }
        }
      } else if (half < kUnits) {
#pragma unroll 1
        for (int u = 0; u < kMine; ++u) {
          const int c0 = (half * kMine + u) * 64;  // column in the tile
          const int col0 = tile.n0 + c0;
          const bool any = rows_any && col0 < n;
          if (EPI == OPS_STORE && p.part) {
            part_out(p, tile.slice, row0, col0, t0 + c0, lane);
          } else if (EPI == OPS_STORE || EPI == OPS_GATE) {
            if (tma) out.free();
            uint8_t* const buf = out.buf();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t w[16];
              const int col = col0 + 32 * h;
              if (EPI == OPS_STORE) {
                uint32_t r[32];
                tc_ld32(t0 + c0 + 32 * h, r);
                tc_wait_ld();
                if (g.unscale) {
                  const float by = *g.unscale;
#pragma unroll
                  for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * by);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack16(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]), f16);
              } else {
                uint32_t rg[32], ru[32];
                tc_ld32(t0 + c0 + 32 * h, rg);
                tc_ld32(t0 + CN + c0 + 32 * h, ru);
                tc_wait_ld();
#pragma unroll
                for (int q = 0; q < 32; q += 16) {
                  float gg[16], uu[16], hh[16];
#pragma unroll
                  for (int i = 0; i < 16; ++i) {
                    gg[i] = __uint_as_float(rg[q + i]);
                    uu[i] = __uint_as_float(ru[q + i]);
                  }
                  gated(gg, uu, hh, gelu, g.kept != nullptr);
#pragma unroll
                  for (int i = 0; i < 16; ++i) {
                    rg[q + i] = __float_as_uint(gg[i]);
                    ru[q + i] = __float_as_uint(uu[i]);
                    if (i & 1) w[(q + i) >> 1] = pack16(hh[i - 1], hh[i], f16);
                  }
                }
                if (g.kept && rows_any && col < n) {
                  uint8_t* b = g.kept + kept_offset(row0, col, g.kept_cols);
                  kept_store(b, lane, rg);
                  kept_store(b + kKeptHalf, lane, ru);
                }
              }
              stage_half(buf, lane, h, w);
            }
            if (tma)
              out.send(&mp.c[0], col0, row0, any);
            else
              rows_out16(buf, p.c, p.ldc, lane, row0, col0, m, n);
          } else if (EPI == OPS_GATE_GRAD) {
            out.free<0>();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t r[32], wg[16], wu[16];
              tc_ld32(t0 + c0 + 32 * h, r);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float d0 = __uint_as_float(r[2 * i]), d1 = __uint_as_float(r[2 * i + 1]);
                wg[i] = pack16(d0 * kept_value(kept[0], 2 * i), d1 * kept_value(kept[0], 2 * i + 1), f16);
                wu[i] = pack16(d0 * kept_value(kept[1], 2 * i), d1 * kept_value(kept[1], 2 * i + 1), f16);
              }
              if (h == 0 || u + 1 < kMine) fetch_kept(col0 + 32 * h + 32);
              stage_half(bufs, lane, h, wg);
              stage_half(bufs + kStoreBytes, lane, h, wu);
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0 && any) {
              tma_store_2d(&mp.c[0], out.first_addr, col0, row0);
              tma_store_2d(&mp.c[1], out.first_addr + kStoreBytes, col0, row0);
              bulk_commit();
            }
          } else {
            const bool f32 = g.out_type == ASD_TYPE_F32;
            if (tma) out.free();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint8_t* const buf = out.buf();
              const int col = col0 + 32 * h;
              uint32_t r[32];
              tc_ld32(t0 + c0 + 32 * h, r);
              tc_wait_ld();
              float f[32];
              if (col + 32 <= n && scales_wide) {  // every lane the same columns' scales, four at a time
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                  const float4 sb = *reinterpret_cast<const float4*>(g.scale_b + col + i);
                  const float4 bb = g.bias ? *reinterpret_cast<const float4*>(g.bias + col + i) : make_float4(0.f, 0.f, 0.f, 0.f);
                  f[i] = fmaf((float)(int)r[i] * sa, sb.x, bb.x);
                  f[i + 1] = fmaf((float)(int)r[i + 1] * sa, sb.y, bb.y);
                  f[i + 2] = fmaf((float)(int)r[i + 2] * sa, sb.z, bb.z);
                  f[i + 3] = fmaf((float)(int)r[i + 3] * sa, sb.w, bb.w);
                }
              } else {  // one load per lane, handed around
                const int mine = col + lane;
                const float sb = mine < n ? g.scale_b[mine] : 0.f;
                const float bb = g.bias && mine < n ? g.bias[mine] : 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  f[i] = fmaf((float)(int)r[i] * sa, __shfl_sync(0xffffffffu, sb, i), __shfl_sync(0xffffffffu, bb, i));
              }
              if (f32) {
                if (tma && h == 1) out.free();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  stage_put(buf, lane, i, make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]),
                                                     __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3])));
                if (tma)
                  out.send(&mp.c[0], col, row0, rows_any && col < n);
                else
                  rows_out32(buf, p.c, p.ldc, lane, row0, col, m, n);
              } else {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack16(f[2 * i], f[2 * i + 1], f16);
                stage_half(buf, lane, h, w);
              }
            }
            if (!f32) {
              if (tma)
                out.send(&mp.c[0], col0, row0, any);
              else
                rows_out16(out.buf(), p.c, p.ldc, lane, row0, col0, m, n);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_cta(acce_bar(acc), 0));
    }
    if (lane == 0) bulk_wait_all();  // the stores have left before the CTA does
  }

  // ---------------- tear-down: neither CTA leaves while the pair's MMAs may still touch it ----------------
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)C::kTmemCols) : "memory");
  }
}

// Joins the slices of sums, a block of 32 x 32 outputs to a block of threads: the partial sums in the order of the slices
// (the same bits in every run), rounded once.
struct JoinArgs {
  struct One {
    const float* part;
    uint16_t* c;
    int64_t ldc;
    int m, n, slices, first;  // number of its first block
  } p[kMostProducts];
  int f16;
  const float* unscale;  // or NULL
};
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ JoinArgs g) {
  __shared__ float tile[32][33];
  int j = 0;
  for (int i = 1; i < kMostProducts; ++i)
    if ((int)blockIdx.x >= g.p[i].first) j = i;
  const JoinArgs::One& p = g.p[j];
  const int block = (int)blockIdx.x - p.first, blocks_n = (p.n + 31) / 32;
  const int64_t slice = (int64_t)((p.m + 31) / 32) * blocks_n * (kPartBlock / 4);
  const float4* from = reinterpret_cast<const float4*>(p.part + (int64_t)block * kPartBlock) + threadIdx.x;
  grid_dependency_wait();
  grid_launch_dependents();
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int i = 0; i < p.slices; ++i) {
    const float4 v = from[i * slice];
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  if (g.unscale) {
    const float by = *g.unscale;
    s.x *= by, s.y *= by, s.z *= by, s.w *= by;
  }
  float* put = &tile[threadIdx.x & 31][4 * (threadIdx.x >> 5)];
  put[0] = s.x, put[1] = s.y, put[2] = s.z, put[3] = s.w;
  __syncthreads();
  const int r = threadIdx.x >> 3, c = 4 * (threadIdx.x & 7);
  const int row = block / blocks_n * 32 + r, col = block % blocks_n * 32 + c;
  if (row >= p.m || col >= p.n) return;
  uint16_t* to = p.c + row * p.ldc + col;
  const float* y = &tile[r][c];
  if (col + 4 <= p.n && ((uintptr_t)to & 7) == 0) {
    *reinterpret_cast<uint2*>(to) = make_uint2(pack16(y[0], y[1], g.f16), pack16(y[2], y[3], g.f16));
  } else {
    for (int e = 0; e < min(4, p.n - col); ++e) to[e] = round16(y[e], g.f16);
  }
}

// ---- host side --------------------------------------------------------------------------------

CUtensorMapDataType map_type(int type) {
  return type == ASD_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                              : type == ASD_TYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
}
// A row-major matrix [rows, cols], boxes of `box_rows` rows of 128 bytes, 128-byte swizzle.
bool encode(CUtensorMap* out, CUtensorMapDataType dt, int es, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)(ld * es)};
  cuuint32_t box[2] = {(cuuint32_t)(128 / es), (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  auto make = [&]() {
    return fn(out, dt, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (make()) return true;
  // A thread on which nothing of CUDA has run yet (autograd's, at the first backward pass) has a current device and no context, which
  // a call of the driver asks for.
  int dev = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && make()) return true;
  cudaGetLastError();
  return false;
}
}  // namespace

bool encode_operand(CUtensorMap* out, const Operand& x, int type, bool i8, int tile_rows) {
  const CUtensorMapDataType dt = i8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : map_type(type);
  return encode(out, dt, x.mat.es, x.mat.p, x.mat.rows, x.mat.cols, x.mat.ld, x.mn ? 64 : tile_rows);
}

namespace {

template <int BN, int EPI, int ACT>
asd_status launch_pair(const asd_ops* o, const OpsGemm* list, int count, cudaStream_t st) {
  using C = OpPairCfg<BN, EPI>;
  constexpr bool I8 = EPI == OPS_I8;
  constexpr int CN = EPI == OPS_GATE ? BN / 2 : BN, N = products_of<EPI>;
  PairMaps<N> maps;
  memset(&maps, 0, sizeof(maps));
  PairArgs<N> g{};
  const int ke = I8 ? 128 : 64;
  int64_t units = 0;
  for (int j = 0; j < N; ++j) {
    PairProduct& p = g.p[j];
    p.first = INT_MAX;
    if (j >= count) continue;
    const OpsGemm& q = list[j];
    p.m = (int)q.m, p.n = (int)q.n;
    p.kb[0] = (int)((q.k[0] + ke - 1) / ke);
    p.kb[1] = q.parts == 2 ? (int)((q.k[1] + ke - 1) / ke) : 0;
    p.tiles_m = (int)((q.m + 2 * BM - 1) / (2 * BM));
    p.tiles_n = (int)((q.n + CN - 1) / CN);
    p.first = (int)units;
    p.slices = std::max(1, q.slices);
    p.per = (p.kb[0] + p.kb[1] + p.slices - 1) / p.slices;
    p.part = p.slices > 1 ? q.part : nullptr;
    units += (int64_t)p.tiles_m * p.tiles_n * p.slices;
    p.a_mn = q.a[0].mn, p.b_mn = q.b[0].mn;
    const uint32_t fmt = I8 ? 1u : (q.type == ASD_TYPE_BF16 ? 1u : 0u);  // signed 8-bit; bf16 or fp16
    p.idesc = (I8 ? 2u << 4 : 1u << 4) | (fmt << 7) | (fmt << 10) | ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16) |
              ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((2 * BM) >> 4) << 24);
    p.c = q.c[0];
    p.ldc = q.ldc;
    const int ct = c_type(q), es = ops_type_size(ct), outs = EPI == OPS_GATE_GRAD ? 2 : 1;
    p.tma_store = 1;
    for (int i = 0; i < outs; ++i)
      if (((uintptr_t)q.c[i] & 15) || (q.ldc * es) % 16) p.tma_store = 0;
    bool ok = true;  // only the maps that the kernel reads
    for (int i = 0; i < q.parts; ++i) ok = ok && encode_operand(&maps.p[j].a[i], q.a[i], q.type, I8, BM);
    for (int i = 0; i < (EPI == OPS_GATE ? 2 : q.parts); ++i) ok = ok && encode_operand(&maps.p[j].b[i], q.b[i], q.type, I8, BN / 2);
    for (int i = 0; i < outs && p.tma_store; ++i) ok = ok && encode(&maps.p[j].c[i], map_type(ct), es, q.c[i], q.m, q.n, q.ldc, 32);
    if (EPI == OPS_LINEAR && q.res) {
      g.res_tma = ((uintptr_t)q.res & 15) == 0 && (q.ldr * es) % 16 == 0;
      if (g.res_tma) ok = ok && encode(&maps.p[j].c[1], map_type(ct), es, q.res, q.m, q.n, q.ldr, 32);
    }
    if (!ok) return ops_fail(ASD_ERR_CUDA, "cuTensorMapEncodeTiled failed");
  }
  const OpsGemm& q = list[0];
  g.units = (int)units;
  g.out_type = c_type(q);
  g.f16 = q.type == ASD_TYPE_F16;
  g.b1 = q.b1, g.b1_f32 = q.b1_f32, g.res = q.res, g.ldr = q.ldr;
  g.gelu = q.act == ASD_ACT_GELU;
  g.kept = q.kept;
  g.kept_cols = (int)((q.n + 31) / 32);
  g.scale_a = q.scale_a, g.scale_b = q.scale_b, g.bias = q.bias;
  g.unscale = q.unscale;  // the list's products have the same one
  g.err = o->err;
  const int pairs = (int)std::min<int64_t>(units, o->num_sms / 2);
  ops_launch(op_pair_kernel<BN, EPI, ACT>, dim3(2 * pairs), dim3(kPairThreads), (size_t)C::kSmemBytes, st, 1, maps, g);
  return ops_launched("matrix product");
}

// Clocks of a k-block (128 bytes of k) of a tile of width bn: the larger of its MMAs' time, 2 bn, and its operands' way
// into shared memory, 128 (128 + bn / 2) bytes at some 50 bytes a clock.
double kblock_clocks(int bn) { return std::max(2.0 * bn, (BM + bn / 2) * 128 / 50.0); }
int64_t pair_tiles(const OpsGemm& q, int bn) {
  const int cn = q.epi == OPS_GATE ? bn / 2 : bn;
  return ((q.m + 2 * BM - 1) / (2 * BM)) * ((q.n + cn - 1) / cn);
}
int64_t pair_kblocks(const OpsGemm& q) {
  const int ke = q.epi == OPS_I8 ? 128 : 64;
  return (q.k[0] + ke - 1) / ke + (q.parts == 2 ? (q.k[1] + ke - 1) / ke : 0);
}
// Clocks of a launch: the tiles go to the clusters in turn, and the longest row of them counts; some 10700 to start, drain
// the last tile and end (measured at 64 tiles of 2 to 32 k-blocks).
double list_clocks(const asd_ops* o, const OpsGemm* list, int count, int bn) {
  const int units = std::min(o->num_sms / 2, 256);
  double every = 0.0, more[256];  // of every cluster, and of some beyond that
  std::fill(more, more + units, 0.0);
  int next = 0;  // the cluster that the next product's first tile goes to
  for (int j = 0; j < count; ++j) {
    const int slices = std::max(1, list[j].slices);
    const int64_t tiles = pair_tiles(list[j], bn) * slices;
    const int rest = (int)(tiles % units);
    const double t = (double)((pair_kblocks(list[j]) + slices - 1) / slices) * kblock_clocks(bn);
    every += t * (double)(tiles / units);
    if (count == 1) return every + (rest ? t : 0.0) + 10700.0;
    for (int i = 0; i < rest; ++i) {
      more[next] += t;
      if (++next == units) next = 0;
    }
  }
  return every + *std::max_element(more, more + units) + 10700.0;
}
template <int EPI, int ACT = ASD_ACT_NONE>
asd_status launch_width(const asd_ops* o, const OpsGemm* list, int count, cudaStream_t st) {
  return list_clocks(o, list, count, 256) <= list_clocks(o, list, count, 128) ? launch_pair<256, EPI, ACT>(o, list, count, st)
                                                                             : launch_pair<128, EPI, ACT>(o, list, count, st);
}

template <int BN, int EPI, int ACT = ASD_ACT_NONE>
cudaError_t prepare_pair() {
  return cudaFuncSetAttribute(op_pair_kernel<BN, EPI, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, OpPairCfg<BN, EPI>::kSmemBytes);
}

}  // namespace

int64_t linear_kept_bytes(int64_t rows, int64_t out) { return (rows + 31) / 32 * ((out + 31) / 32) * (4 * kSlopeBlock); }
int64_t gated_kept_bytes(int64_t rows, int64_t hidden) { return (rows + 31) / 32 * ((hidden + 31) / 32) * kKeptBlock; }

namespace {
// Whether a product is better split than tiled; `plan` is how.
bool better_split(const asd_ops* o, const OpsGemm& q, bool early, SplitPlan* plan) {
  if (q.a[0].mn || q.m > kSplitMostRows) return false;
  *plan = plan_split(o, q, early);
  return plan->clocks < std::min(list_clocks(o, &q, 1, 256), list_clocks(o, &q, 1, 128));
}

asd_status launch_join(const OpsGemm* list, int count, cudaStream_t st) {
  JoinArgs g{};
  int64_t blocks = 0;
  int n = 0;
  for (int j = 0; j < count; ++j) {
    const OpsGemm& q = list[j];
    if (q.slices <= 1) continue;
    g.p[n++] = {q.part, (uint16_t*)q.c[0], q.ldc, (int)q.m, (int)q.n, q.slices, (int)blocks};
    blocks += (q.m + 31) / 32 * ((q.n + 31) / 32);
  }
  if (n == 0) return ASD_OK;
  for (int j = n; j < kMostProducts; ++j) g.p[j].first = INT_MAX;
  g.f16 = list[0].type == ASD_TYPE_F16;
  g.unscale = list[0].unscale;
  ops_launch(join_kernel, dim3((unsigned)blocks), dim3(256), 0, st, 1, g);
  return ops_launched("join of a sum's slices");
}
}  // namespace

asd_status ops_gemm(const asd_ops* o, const OpsGemm& q, bool early, cudaStream_t st) {
  if (use_stream(q)) return ops_gemm_stream(o, q, early, st);
  SplitPlan p;
  if (better_split(o, q, early, &p)) return ops_gemm_split(o, q, p, early, st);
  switch (q.epi) {
    case OPS_STORE: return launch_width<OPS_STORE>(o, &q, 1, st);
    case OPS_GATE: return launch_width<OPS_GATE>(o, &q, 1, st);
    case OPS_GATE_GRAD: return launch_width<OPS_GATE_GRAD>(o, &q, 1, st);
    case OPS_LINEAR:
      return q.act == ASD_ACT_SILU   ? launch_width<OPS_LINEAR, ASD_ACT_SILU>(o, &q, 1, st)
             : q.act == ASD_ACT_GELU ? launch_width<OPS_LINEAR, ASD_ACT_GELU>(o, &q, 1, st)
                                     : launch_width<OPS_LINEAR>(o, &q, 1, st);
    default: return launch_width<OPS_I8>(o, &q, 1, st);
  }
}

// One launch of tiles for all of the list, so that the last, partly filled wave of tiles comes once and not once for each
// product.  A first product (the one with the longest sum) that is better split goes by itself; whether it is does not
// depend on the others, so that a gradient has the same bits whichever are asked for.
asd_status ops_gemm_list(const asd_ops* o, const OpsGemm* list, int count, cudaStream_t st) {
  SplitPlan p;
  if (count && better_split(o, list[0], false, &p)) {
    const asd_status s = ops_gemm_split(o, list[0], p, false, st);
    if (s != ASD_OK) return s;
    ++list, --count;
  }
  if (!count) return ASD_OK;
  const asd_status s = launch_width<OPS_STORE>(o, list, count, st);
  return s == ASD_OK ? launch_join(list, count, st) : s;
}

// The gradient of a narrow weight is a few tiles with a sum over all rows, which a few pairs would walk along while the
// others are idle.  Up to a sixth of the pairs' number of tiles are therefore cut into as many slices as there are pairs, of
// 16 k-blocks at least.  All gradients of the gated MLP, with slices against without: 32768 x 256 x 512 (2 tiles) 96 us
// against 228, 131072 x 256 x 1024 (4) 565 against 1115, 32768 x 512 x 1280 (10) 273 against 356; with 12 tiles the
// two meet at some 4096 rows (512 x 1536: 2048 rows 51 against 49, 4096 65 against 63, 8192 97 against 111, 32768 332 against 447).
// Beyond that the input's gradient in the same launch keeps the pairs busy and the partial sums only cost: 4096 x
// 512 x 2048 (16) 80 against 70, 8192 x 768 x 2048 (24) 184 against 167.  It goes by the sizes of the one product alone, so
// that a gradient has the same bits whichever others are asked for.
// A linear layer has only one other product beside it, no longer than this one, and half of the pairs' number is the border there
// (part = 2), both products: 4096 x 1024 x 1024 (16 tiles) 43 to 29 us, 8192 72 to 43, 32768 262 to 115; 8192 x 1024 x 2048 (32) 84 to 68,
// 8192 x 1536 x 1536 (36) 88 to 74; where 16 k-blocks to a slice leave one, as at 2048 x 1536 x 1536, nothing changes, and
// with 8 k-blocks 1024 x 1024 x 1024 takes 28 instead of 25.
int sum_slices(const asd_ops* o, int64_t m, int64_t n, int64_t k, int part) {
  const int pairs = o->num_sms / 2;
  const int64_t tiles = ((m + 255) / 256) * ((n + 255) / 256), kb = (k + 63) / 64;
  if (part * tiles > pairs) return 1;
  const int64_t slices = std::min<int64_t>(pairs / tiles, kb / 16);
  if (slices < 2) return 1;
  const int64_t per = (kb + slices - 1) / slices;
  return (int)((kb + per - 1) / per);
}
int64_t part_bytes(int64_t m, int64_t n, int slices) {
  return slices > 1 ? (m + 31) / 32 * ((n + 31) / 32) * slices * (kPartBlock * 4) : 0;
}

asd_status ops_gemm_prepare() {
  const cudaError_t all[] = {prepare_pair<256, OPS_STORE>(),     prepare_pair<128, OPS_STORE>(), prepare_pair<256, OPS_GATE>(),
                             prepare_pair<128, OPS_GATE>(),      prepare_pair<256, OPS_GATE_GRAD>(),
                             prepare_pair<128, OPS_GATE_GRAD>(), prepare_pair<256, OPS_I8>(),    prepare_pair<128, OPS_I8>(),
                             prepare_pair<256, OPS_LINEAR>(),    prepare_pair<128, OPS_LINEAR>(),
                             prepare_pair<256, OPS_LINEAR, ASD_ACT_SILU>(), prepare_pair<128, OPS_LINEAR, ASD_ACT_SILU>(),
                             prepare_pair<256, OPS_LINEAR, ASD_ACT_GELU>(), prepare_pair<128, OPS_LINEAR, ASD_ACT_GELU>()};
  for (cudaError_t e : all)
    if (e != cudaSuccess) return ops_fail(ASD_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  return ASD_OK;
}

}  // namespace asd
