// What the gradients of a linear layer y = r + act(x w^T + bias) need beside its two products: dz = dy act'(z), rounded to 16
// bits for the tensor cores, and the bias's gradient, the sums of dz over the rows before that rounding.
//
// One pass over dy and the kept act'(z), which are in blocks of 32 rows by 32 columns (a lane a row): a warp has 32 columns and
// walks down a share of the rows, so that the sums of its columns stay in registers, 32 to a lane, and meet over the lanes once
// at its end.  The shares' sums are joined in their order by a second kernel: the same bits in every run.
//
// Bound by memory, 8 bytes an element with dy in 16 bits and 10 in 32: 8192 x 4096 42 and 48 us (6.4 and 7.0 TB/s, some of it from L2), with
// rows that are not on 16 bytes 70 and 57, by elements through shared memory, 16 of a lane's on their way at a time (8: 81, 63; all 32,
// which leave an SM one block: 178).
//
// A dy in 32 bits is a mean's gradient as often as not, 2e-6 a row and column, of which F16 has 32 steps.  With F16 operands dz is therefore
// written times the power of two that brings dy's largest finite magnitude to 2^14 to 2^15 (act' is 1.13 at most), and the products take it off their
// sums.  The largest magnitude is a pass over dy of its own: the whole backward pass of 8192 x 4096 x 4096 takes 502 us where BF16's, without
// it, takes 464, of 8192 x 1024 x 1024 80 and 70, of 1000 x 304 x 1001 37 and 33.
#include <algorithm>

#include "asd_ops_tc.cuh"

namespace asd {
namespace {

constexpr int kLinearWarps = 8;
constexpr int kPeakBlock = 256, kPeakReads = 8;  // reads of a thread that are on their way together

struct LinearArgs {
  int rows, out, blocks_n, shares;
  int wide;  // rows of dy are on 16 bytes
  const void* dy;
  int64_t ld_dy;
  const float* kept;
  uint16_t* dz;
  int64_t ld_dz;
  float* part;  // [shares, out]
  const uint32_t* peaks;  // the largest magnitudes of dy, block by block, or NULL
  int n_peaks;
  float* unscale;
};

// The 32 lanes' sums of 32 columns: lane l gets that of column l.  Each step halves the columns that a lane holds.
__device__ __forceinline__ float columns_sum(float (&v)[32], int lane) {
#pragma unroll
  for (int w = 16; w; w >>= 1) {
    const bool up = lane & w;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = up ? v[i + w] : v[i], give = up ? v[i] : v[i + w];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
    }
  }
  return v[0];
}

// The largest finite magnitude of a matrix in 32 bits, as far as a block has come: WIDE reads four columns at a time, of rows on 16 bytes.
template <bool WIDE>
__global__ void __launch_bounds__(kPeakBlock) linear_peak_kernel(const float* dy, int64_t ld, int rows, int out, uint32_t* peaks) {
  constexpr int V = WIDE ? 4 : 1;
  __shared__ uint32_t most[kPeakBlock / 32];
  grid_dependency_wait();
  grid_launch_dependents();
  const int across = (out + V - 1) / V;
  const int64_t threads = (int64_t)gridDim.x * kPeakBlock, at = (int64_t)blockIdx.x * kPeakBlock + threadIdx.x;
  int64_t row = at / across;
  int col = (int)(at - row * across);
  const int64_t down = threads / across;
  const int over = (int)(threads - down * across);
  uint32_t peak = 0;
  while (row < rows) {
    float f[kPeakReads][V];
#pragma unroll
    for (int i = 0; i < kPeakReads; ++i) {
      const float* p = dy + row * ld + V * col;
#pragma unroll
      for (int e = 0; e < V; ++e) f[i][e] = 0.f;
      if (row < rows) {
        if (WIDE && V * col + V <= out) {
          const float4 x = *reinterpret_cast<const float4*>(p);
          f[i][0] = x.x, f[i][V > 1 ? 1 : 0] = x.y, f[i][V > 2 ? 2 : 0] = x.z, f[i][V > 3 ? 3 : 0] = x.w;
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (V * col + e < out) f[i][e] = p[e];
        }
      }
      row += down, col += over;
      if (col >= across) col -= across, ++row;
    }
#pragma unroll
    for (int i = 0; i < kPeakReads; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const uint32_t m = __float_as_uint(f[i][e]) & 0x7fffffffu;
        peak = max(peak, m < 0x7f800000u ? m : 0u);
      }
  }
  peak = __reduce_max_sync(0xffffffffu, peak);
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = peak;
  __syncthreads();
  if (threadIdx.x < 32) {
    peak = __reduce_max_sync(0xffffffffu, threadIdx.x < kPeakBlock / 32 ? most[threadIdx.x] : 0u);
    if (threadIdx.x == 0) peaks[blockIdx.x] = peak;
  }
}
// The exponent, as fp32 has it, of the power of two that takes the largest of the peaks to 2^14 to 2^15.  All threads of the block.
__device__ __forceinline__ uint32_t scale_exponent(const uint32_t* peaks, int n) {
  __shared__ uint32_t most[kLinearWarps];
  uint32_t peak = 0;
  for (int i = threadIdx.x; i < n; i += 32 * kLinearWarps) peak = max(peak, peaks[i]);
  peak = __reduce_max_sync(0xffffffffu, peak);
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = peak;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kLinearWarps; ++i) peak = max(peak, most[i]);
  return min(268u - (peak >> 23), 253u);  // a peak of exponent 254 at most: 14 at least; and its reciprocal's is 1 at least
}

template <bool F32, bool F16>
__global__ void __launch_bounds__(32 * kLinearWarps, 2) linear_rows_kernel(const LinearArgs a) {
  __shared__ float turned[kLinearWarps][32][33];  // rows that are not aligned: read along the row, handed to their lanes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int block = blockIdx.x * kLinearWarps + warp, col0 = block * 32;
  grid_dependency_wait();
  grid_launch_dependents();
  float scale = 1.f;
  if (F32 && F16 && a.peaks) {
    const uint32_t e = scale_exponent(a.peaks, a.n_peaks);
    scale = __uint_as_float(e << 23);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.unscale = __uint_as_float((254u - e) << 23);
  }
  if (col0 >= a.out) return;
  const int cols = min(32, a.out - col0);
  float sum[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) sum[i] = 0.f;
  for (int64_t row0 = (int64_t)blockIdx.y * 32; row0 < a.rows; row0 += (int64_t)a.shares * 32) {
    const int64_t row = row0 + lane;
    const bool live = row < a.rows;
    float4 kept[8];
    if (a.kept) {
      const float4* p = reinterpret_cast<const float4*>(slope_block(const_cast<float*>(a.kept), (int)row0, col0, a.blocks_n)) + lane;
#pragma unroll
      for (int i = 0; i < 8; ++i) kept[i] = p[32 * i];
    }
    float d[32];
    if (!a.wide) {
      const int rows = (int)min((int64_t)32, a.rows - row0);
#pragma unroll 16
      for (int r = 0; r < 32; ++r)
        turned[warp][r][lane] = r < rows && lane < cols ? load_scalar(a.dy, (row0 + r) * a.ld_dy + col0 + lane, F32, F16) : 0.f;
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 32; ++i) d[i] = turned[warp][lane][i];
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
      if (!a.wide) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[i + j] = 0.f;
      if (live && i + 8 <= cols) {
        if constexpr (F32) {
          const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.dy) + row * a.ld_dy + col0 + i);
          const float4 x = p[0], y = p[1];
          d[i] = x.x, d[i + 1] = x.y, d[i + 2] = x.z, d[i + 3] = x.w, d[i + 4] = y.x, d[i + 5] = y.y, d[i + 6] = y.z, d[i + 7] = y.w;
        } else {
          const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.dy) + row * a.ld_dy + col0 + i);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 y = unpack16(w[j], F16);
            d[i + 2 * j] = y.x, d[i + 2 * j + 1] = y.y;
          }
        }
      } else if (live) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (i + j < cols) d[i + j] = load_scalar(a.dy, row * a.ld_dy + col0 + i + j, F32, F16);
      }
    }
    if (a.kept) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float4 k = kept[i >> 2];
        d[i] = live && i < cols ? d[i] * ((i & 3) == 0 ? k.x : (i & 3) == 1 ? k.y : (i & 3) == 2 ? k.z : k.w) : 0.f;  // what is kept beyond the matrix is not defined
      }
    }
    if (a.part) {
#pragma unroll
      for (int i = 0; i < 32; ++i) sum[i] += d[i];
    }
    if constexpr (F32 && F16) {
#pragma unroll
      for (int i = 0; i < 32; ++i) d[i] *= scale;
    }
    if (a.dz && live) {
      uint16_t* to = a.dz + row * a.ld_dz + col0;  // rows of a multiple of 8 elements
#pragma unroll
      for (int i = 0; i < 32; i += 8)
        if (i < cols)
          *reinterpret_cast<uint4*>(to + i) = make_uint4(pack16(d[i], d[i + 1], F16), pack16(d[i + 2], d[i + 3], F16), pack16(d[i + 4], d[i + 5], F16),
                                                         pack16(d[i + 6], d[i + 7], F16));
    }
  }
  if (a.part) {
    const float v = columns_sum(sum, lane);
    if (lane < cols) a.part[(size_t)blockIdx.y * a.out + col0 + lane] = v;
  }
}

// Shares of the rows: four blocks an SM between them and the columns, of two row blocks or more, so that the last step of the
// sums does not outweigh them; of one where they then find an SM each, as the time of a walk is all there is (256 x 512 x 512, the whole
// backward pass 24.5 to 22.4 us, 1000 x 304 x 1001 34.8 to 30.7, with cold inputs).
int row_shares(const asd_ops* o, int64_t rows, int64_t out) {
  const int64_t across = (out + 32 * kLinearWarps - 1) / (32 * kLinearWarps), down = (rows + 31) / 32;
  if (across * down <= o->num_sms) return (int)std::max<int64_t>(1, down);
  return (int)std::max<int64_t>(1, std::min<int64_t>((down + 1) / 2, (4 * o->num_sms + across - 1) / across));
}

}  // namespace

int64_t linear_part_bytes(const asd_ops* o, int64_t rows, int64_t out) { return (int64_t)row_shares(o, rows, out) * out * 4; }

// Blocks of the pass over dy: four an SM, or as many as read it element by element at once.
int linear_peaks(const asd_ops* o, int64_t rows, int64_t out) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(4 * (int64_t)o->num_sms, (rows * out + kPeakBlock * kPeakReads - 1) / (kPeakBlock * kPeakReads)));
}

asd_status launch_linear_rows(const asd_ops* o, const LinearRows& q, cudaStream_t st) {
  LinearArgs a{};
  a.rows = q.rows, a.out = q.out, a.blocks_n = (q.out + 31) / 32, a.shares = row_shares(o, q.rows, q.out);
  a.wide = ((uintptr_t)q.dy & 15) == 0 && (q.ld_dy * (q.dy_f32 ? 4 : 2)) % 16 == 0;
  a.dy = q.dy, a.ld_dy = q.ld_dy, a.kept = q.kept, a.dz = (uint16_t*)q.dz, a.ld_dz = q.ld_dz;
  a.part = q.dbias ? q.part : nullptr;
  const dim3 grid((unsigned)((q.out + 32 * kLinearWarps - 1) / (32 * kLinearWarps)), (unsigned)a.shares), block(32 * kLinearWarps);
  const bool f16 = q.type == ASD_TYPE_F16;
  if (q.peaks) {
    a.peaks = q.peaks, a.n_peaks = linear_peaks(o, q.rows, q.out), a.unscale = q.unscale;
    ops_launch(a.wide ? linear_peak_kernel<true> : linear_peak_kernel<false>, dim3((unsigned)a.n_peaks), dim3(kPeakBlock), 0, st, 1, (const float*)q.dy, q.ld_dy,
               q.rows, q.out, q.peaks);
  }
  if (q.dy_f32)
    f16 ? ops_launch(linear_rows_kernel<true, true>, grid, block, 0, st, 1, a) : ops_launch(linear_rows_kernel<true, false>, grid, block, 0, st, 1, a);
  else
    f16 ? ops_launch(linear_rows_kernel<false, true>, grid, block, 0, st, 1, a) : ops_launch(linear_rows_kernel<false, false>, grid, block, 0, st, 1, a);
  if (q.dbias) launch_column_join(q.part, a.shares, q.out, q.dbias, q.bias_type, st);
  return ops_launched("linear gradient");
}

}  // namespace asd
