// Rows of bf16 to int8 with one scale per row, for the 8-bit expert products:
//   a = max_c |x[r][c]|,  scale[r] = a / 127,  q[r][c] = rint(127 x[r][c] / a),
// ties to even (scale 0 and q 0 where a = 0).  A row that holds a NaN or an
// infinity has no such scale: it gets scale NaN and q 0, so that every product
// with it is NaN rather than a plausible number.
//
// The integer is the one that exact arithmetic gives.  y = x * (127 / a) in
// fp32 is within 2^-22 of 127 x / a, relatively.  With x and a of 8
// significant bits, a quotient that is not exactly n + 1/2 lies at least 2^-16
// (relatively) from it, and n + 1/2 itself has 8 significant bits: so y,
// rounded to 18 significant bits, is n + 1/2 exactly where the quotient is,
// and on the quotient's side of it elsewhere.  That is two integer
// instructions; an IEEE division per element would be ten.  Adding 1.5 * 2^23
// then rounds to even and leaves the integer in the low byte.
//
// Bound by HBM: 2 bytes read and 1 written per value, one pass, the row held
// in registers between its maximum and its rounding.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace moe {
namespace {

constexpr int kQuantThreads = 256;
constexpr int kQuantWaves = kQuantThreads / kWave;
constexpr int kVec = 8;  // values per 16-byte load

// 16 bytes at any bf16 address: rows of odd length start at odd multiples of
// two bytes (global memory takes unaligned vector loads on this target).
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct QuantPair {
  QuantArgs a, b;
  int blocks_a;
};

// Vector v of a row (zeros past its end).
__device__ __forceinline__ u32x4 load_vec(const uint16_t* row, int v, int cols) {
  const int c = v * kVec;
  if (c + kVec <= cols) return *reinterpret_cast<const u32x4_a2*>(row + c);
  u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (c + i < cols) r[i / 2] |= static_cast<uint32_t>(row[c + i]) << (16 * (i & 1));
  return r;
}

// Largest magnitude of the 8 values, as bf16 bits in both halves' maxima: the
// order of the bits is the order of the magnitudes, infinity and NaN on top.
__device__ __forceinline__ u16x2 max_bits(u16x2 m, u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
  return m;
}

__device__ __forceinline__ uint32_t round_bits(float x, float pre, float c) {
  const uint32_t y = (__float_as_uint((x * pre) * c) + 32u) & ~63u;
  return __float_as_uint(__uint_as_float(y) + 12582912.0f);
}

__device__ __forceinline__ u32x2 quantize_vec(u32x4 v, float pre, float c) {
  u32x2 out;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pair = v[2 * h + i / 2];
      b[i] = round_bits(__uint_as_float((i & 1) ? (pair & 0xffff0000u) : (pair << 16)), pre, c);
    }
    const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
    out[h] = lo | (hi << 16);
  }
  return out;
}

// The largest of the 64 lanes' values, in all of them: within rows of 16 lanes
// by data-parallel moves, then across the rows.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#define MOE_DPP_MAX(ctrl) v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ctrl, 0xf, 0xf, true)))
  MOE_DPP_MAX(0xB1);   // quad_perm [1 0 3 2]
  MOE_DPP_MAX(0x4E);   // quad_perm [2 3 0 1]
  MOE_DPP_MAX(0x141);  // row_half_mirror
  MOE_DPP_MAX(0x140);  // row_mirror
#undef MOE_DPP_MAX
  const auto r16 = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(static_cast<uint32_t>(r16[0]), static_cast<uint32_t>(r16[1]));
  const auto r32 = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(static_cast<uint32_t>(r32[0]), static_cast<uint32_t>(r32[1]));
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
        if (r0 + k < rows && at + i * STEP < nvec) v[k][i] = load_vec(a.x + (r0 + k) * a.ldx, at + i * STEP, a.cols);
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
      const bool finite = top < 0x7f80u;
      const float amax = __uint_as_float(top << 16);
      // 127 / a leaves the range of fp32 for the smallest a: those rows are
      // scaled by 2^80 first (exact)
      const float pre = amax < 0x1p-60f ? 0x1p80f : 1.0f;
      const float c = (finite && top != 0u) ? 127.0f / (amax * pre) : 0.0f;
      if (at == 0) a.scale[r] = finite ? amax / 127.0f : __uint_as_float(0x7fc00000u);
      int8_t* out = a.q + r * a.ldq;
      // (a row that is not finite multiplies to NaN, whose bits are no integer)
      auto put = [&](int i, u32x4 x) {
        *reinterpret_cast<u32x2*>(out + static_cast<long long>(i) * kVec) = finite ? quantize_vec(x, pre, c) : u32x2{0u, 0u};
      };
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
