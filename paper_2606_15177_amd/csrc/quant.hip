// Rows of bf16 to int8 with one scale per row, for the 8-bit expert products:
//   a = max_c |x[r][c]|,  scale[r] = a / 127,  q[r][c] = rint(127 x[r][c] / a),
// ties to even (scale 0 and q 0 where a = 0).  A row that holds a NaN or an
// infinity has no such scale: it gets scale NaN and q 0, so that every product
// with it is NaN rather than a plausible number.
//
// The arithmetic and why it is exact: quant_impl.h.
//
// Bound by HBM: 2 bytes read and 1 written per value, one pass, the row held
// in registers between its maximum and its rounding.
#include <algorithm>

#include "kernels.h"
#include "quant_impl.h"

namespace moe {
namespace {

constexpr int kQuantThreads = 256;
constexpr int kQuantWaves = kQuantThreads / kWave;
struct QuantPair {
  QuantArgs a, b;
  int blocks_a;
};

// Vector v of a row that is not read again: its lines leave the caches first
// (16384 x 7168: 65.3 us without the hint, 62.3 with it, 5.66 TB/s).
__device__ __forceinline__ u32x4 load_once(const uint16_t* row, int v, int cols) {
  const int c = v * kVec;
  return c + kVec <= cols ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(row + c)) : load_vec(row, v, cols);
}

// WPR waves per row, V vectors per lane held in registers (vectors past them
// are read twice), R rows at a time per wave (WPR 1): short rows need several
// in flight to cover the memory's latency.
template <int WPR, int V, int R>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(QuantPair p) {
  static_assert(WPR == 1 || R == 1, "several rows at a time: one wave each");
  constexpr int RPB = kQuantWaves / WPR * R;  // rows of a block at a time
  constexpr int STEP = WPR * kWave;           // vectors of a row at a time
  __shared__ uint32_t part[kQuantWaves];
  const bool second = static_cast<int>(blockIdx.x) >= p.blocks_a;
  const QuantArgs& a = second ? p.b : p.a;
  const int block = static_cast<int>(blockIdx.x) - (second ? p.blocks_a : 0);
  const int blocks = second ? static_cast<int>(gridDim.x) - p.blocks_a : p.blocks_a;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int at = static_cast<int>(threadIdx.x) % STEP;
  const int rows = a.n_rows ? min(a.rows, *a.n_rows) : a.rows;
  const int nvec = ceil_div(a.cols, 16) * 2;  // the padding to 16 values is written too, as zeros
  for (long long r0 = static_cast<long long>(block) * RPB + wave / WPR * R; r0 < rows; r0 += static_cast<long long>(blocks) * RPB) {
    u32x4 v[R][V];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[k][i] = u32x4{0u, 0u, 0u, 0u};
        if (r0 + k < rows && at + i * STEP < nvec) v[k][i] = load_once(a.x + (r0 + k) * a.ldx, at + i * STEP, a.cols);
      }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const long long r = r0 + k;
      if (r >= rows) break;
      const uint16_t* row = a.x + r * a.ldx;
      u16x2 m = {0, 0};
#pragma unroll
      for (int i = 0; i < V; ++i) m = max_bits(m, v[k][i]);
      for (int i = at + V * STEP; i < nvec; i += STEP) m = max_bits(m, load_vec(row, i, a.cols));
      uint32_t top = wave_max(max(static_cast<uint32_t>(m[0]), static_cast<uint32_t>(m[1])));
      if constexpr (WPR > 1) {
        if (lane_id() == 0) part[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantWaves; ++w) top = max(top, part[w]);
        __syncthreads();
      }
      const RowScale s = row_scale(top);
      if (at == 0) a.scale[r] = s.scale;
      int8_t* out = a.q + r * a.ldq;
      auto put = [&](int i, u32x4 x) { *reinterpret_cast<u32x2*>(out + static_cast<long long>(i) * kVec) = quantize_vec(x, s); };
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (at + i * STEP < nvec) put(at + i * STEP, v[k][i]);
      for (int i = at + V * STEP; i < nvec; i += STEP) put(i, load_vec(row, i, a.cols));
    }
  }
}

// Enough workgroups to fill the chip many times over; the rest by the loop
// over rows (a grid dimension holds 2^32 - 1 threads).
constexpr int kMaxBlocks = 1 << 20;

int quant_blocks(const QuantArgs& a, int rows_per_block) {
  return static_cast<int>(std::min<long long>((static_cast<long long>(a.rows) + rows_per_block - 1) / rows_per_block, kMaxBlocks));
}

template <int WPR, int V, int R>
hipError_t launch_rows(const QuantArgs& a, const QuantArgs* b, hipStream_t st) {
  constexpr int RPB = kQuantWaves / WPR * R;
  const QuantPair p{a, b ? *b : QuantArgs{}, quant_blocks(a, RPB)};
  const int grid = p.blocks_a + (b ? quant_blocks(*b, RPB) : 0);
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL((quantize_kernel<WPR, V, R>), dim3(grid), dim3(kQuantThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace

// A wave per row up to 4096 columns, several rows of up to 1024; a workgroup
// per row past that, and where there are no more rows than CUs (one row of
// 2048: latency alone).
hipError_t launch_quantize_rows(const QuantArgs& a, const QuantArgs* b, hipStream_t st) {
  const int cols = std::max(a.cols, b ? b->cols : 0);
  const long long rows = static_cast<long long>(a.rows) + (b ? b->rows : 0);
  if (cols > 4096 || (cols > 512 && rows <= 256)) return launch_rows<kQuantWaves, 8, 1>(a, b, st);
  if (cols > 2048) return launch_rows<1, 8, 1>(a, b, st);
  if (cols > 1024) return launch_rows<1, 4, 1>(a, b, st);
  return launch_rows<1, 2, 2>(a, b, st);
}

}  // namespace moe
