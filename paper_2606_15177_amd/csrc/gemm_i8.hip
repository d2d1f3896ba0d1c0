// Products of int8 rows with int8 weights, grouped by expert, with a scale per
// token and per output channel:
//   y[r][n] = bf16( (sum_c X[r][c] W[g][n][c]) * ws[g][n] * xs[r] )
// and the gated pair bf16( silu(gate) * up ) of two such products.  The sums
// are exact in int32 (K < 2^17); each value is rounded to bf16 once, the type
// that every output of the layer has.
//
// One workgroup of four waves per 64 rows x 64 columns of a group, each wave a
// 32 x 32 tile of v_mfma_i32_32x32x32_i8: lane l reads 16 bytes of row l % 32
// at k + 16 (l / 32) of either operand, and holds the results
// C[n = 8 (i / 4) + 4 (l / 32) + i % 4][r = l % 32].
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace moe {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kRows = 64, kCols = 64;

template <bool GATED>
__global__ __launch_bounds__(4 * kWave) void gemm_i8_kernel(GemmI8 a) {
  const int lane = lane_id(), wave = static_cast<int>(threadIdx.x) / kWave;
  const int lrow = lane & 31, lhalf = lane >> 5;
  // the group of this row tile: tiles are numbered by group
  int tile = static_cast<int>(blockIdx.y), g = 0, row_base = 0, m = a.static_rows;
  if (a.offsets) {
    for (;; ++g) {
      if (g == a.groups) return;
      row_base = a.offsets[g];
      m = a.offsets[g + 1] - row_base;
      const int t = m > 0 ? ceil_div(m, kRows) : 0;
      if (tile < t) break;
      tile -= t;
    }
  }
  const int r = tile * kRows + (wave & 1) * 32 + lrow;  // row within the group
  const int n0 = static_cast<int>(blockIdx.x) * kCols + (wave >> 1) * 32;
  const bool row_ok = r < m;
  const int row = row_base + (row_ok ? r : 0);
  int src = a.x_rows ? a.x_rows[row] : row;
  const bool src_ok = row_ok && (!a.x_rows || static_cast<unsigned>(src) < static_cast<unsigned>(a.x_count));
  if (!src_ok) src = 0;
  const int8_t* xp = a.x + static_cast<long long>(src) * a.ldx + 16 * lhalf;
  const int n = min(n0 + lrow, a.N - 1);
  const long long wofs = (static_cast<long long>(g) * a.N + n) * a.ldw + 16 * lhalf;
  i32x16 acc0 = {}, acc1 = {};
  const int kb = ceil_div(a.K, 16) * 16;
  for (int k = 0; k < kb; k += 32) {
    const bool ok = k + 16 * lhalf < kb;
    const i32x4 zero = {0, 0, 0, 0};
    const i32x4 xf = ok && src_ok ? *reinterpret_cast<const i32x4*>(xp + k) : zero;
    const i32x4 wf = ok ? *reinterpret_cast<const i32x4*>(a.w0 + wofs + k) : zero;
    acc0 = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf, xf, acc0, 0, 0, 0);
    if constexpr (GATED) {
      const i32x4 uf = ok ? *reinterpret_cast<const i32x4*>(a.w1 + wofs + k) : zero;
      acc1 = __builtin_amdgcn_mfma_i32_32x32x32_i8(uf, xf, acc1, 0, 0, 0);
    }
  }
  if (!row_ok) return;
  const float xs = src_ok ? a.x_scale[src] : 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int col = n0 + 8 * (i / 4) + 4 * lhalf + i % 4;
    if (col >= a.N) continue;
    const long long sc = static_cast<long long>(g) * a.N + col;
    float o = static_cast<float>(acc0[i]) * a.ws0[sc] * xs;
    if constexpr (GATED) o = silu(o) * (static_cast<float>(acc1[i]) * a.ws1[sc] * xs);
    a.out[static_cast<long long>(row) * a.ldo + col] = f32_to_bf16(o);
  }
}

hipError_t launch_one(const Segments& seg, const GemmI8& a, bool gated, hipStream_t st) {
  const int m_tiles = a.offsets ? seg.total_rows / kRows + std::min(seg.groups, seg.total_rows) : ceil_div(seg.static_rows, kRows);
  if (m_tiles == 0) return hipSuccess;
  const dim3 grid(ceil_div(a.N, kCols), m_tiles);
  if (gated)
    hipLaunchKernelGGL((gemm_i8_kernel<true>), grid, dim3(4 * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((gemm_i8_kernel<false>), grid, dim3(4 * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_i8(const Segments& seg, const GemmI8& a, const Segments* sh_seg, const GemmI8* sh, bool gated,
                          hipStream_t st) {
  hipError_t e = launch_one(seg, a, gated, st);
  if (e != hipSuccess || sh == nullptr) return e;
  return launch_one(*sh_seg, *sh, gated, st);
}

}  // namespace moe
