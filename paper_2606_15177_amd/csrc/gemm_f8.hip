// Products in e4m3 with a scale per 128 columns of a row and per 128 x 128 block of
// a matrix (see moe.h): the simplest kernel that is right for every size.
//
// A wave computes 32 rows of a group by 32 weight rows (gated: 16 gate rows and the
// 16 up rows of the same columns, which meet in one lane), its operands straight
// from memory.
#include <algorithm>

#include "f8_impl.h"

namespace moe {
namespace {

constexpr int kThreads = 4 * kWave;

struct PairF8 {
  GemmF8 g, sp;
  int rows;  // of g's result
};

// 32 bytes at byte k of a row of `bytes` (a multiple of 16); zeros past its end
// and where there is no row.
__device__ __forceinline__ i32x8 load32(const uint8_t* row, int k, int bytes) {
  u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
  if (row && k < bytes) lo = load16(row + k);
  if (row && k + 16 < bytes) hi = load16(row + k + 16);
  i32x8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = static_cast<int>(lo[i]);
    v[4 + i] = static_cast<int>(hi[i]);
  }
  return v;
}

template <bool GATED>
__global__ __launch_bounds__(kThreads) void simple_f8_kernel(PairF8 pa) {
  constexpr int COLS = GATED ? 16 : 32;
  const int lane = lane_id(), lrow = lane & 31, lhalf = lane >> 5;
  const int wave = static_cast<int>(threadIdx.x) / kWave;
  // the chunk of 32 rows: the shared rows' first, then group by group
  int chunk = static_cast<int>(blockIdx.x);
  const int sp_chunks = ceil_div(pa.sp.static_rows, 32);
  const bool shared = chunk < sp_chunks;
  const GemmF8& p = shared ? pa.sp : pa.g;
  int g = 0, base = 0, m = p.static_rows;
  if (!shared) {
    chunk -= sp_chunks;
    for (; g < p.groups; ++g) {
      base = row_at(p.offsets, g, pa.rows);
      m = max(row_at(p.offsets, g + 1, pa.rows) - base, 0);
      if (chunk < ceil_div(m, 32)) break;
      chunk -= ceil_div(m, 32);
    }
    if (g == p.groups) return;
  }
  const int n0 = (static_cast<int>(blockIdx.y) * 4 + wave) * COLS;
  if (n0 >= p.N) return;
  const int r = base + 32 * chunk + lrow, kb = ceil_div(p.K, kF8Block), bytes = ceil_div(p.K, 16) * 16;
  const bool row_in = 32 * chunk + lrow < m;
  const int src = row_in && p.x_rows ? p.x_rows[r] : r;
  const bool in = row_in && (!p.x_rows || static_cast<unsigned>(src) < static_cast<unsigned>(p.x_count));
  const uint8_t* x = in ? p.x + static_cast<long long>(src) * p.ldx : nullptr;
  const int col = n0 + (GATED ? lrow & 15 : lrow);
  const bool up = GATED && (lrow & 16);
  const uint8_t* w = col < p.N ? (up ? p.w1 : p.w0) + (static_cast<long long>(g) * p.N + col) * p.ldw : nullptr;
  const long long sc = (static_cast<long long>(g) * ceil_div(p.N, kF8Block) + n0 / kF8Block) * kb;
  f32x16 acc = {};
  for (int b = 0; b < kb; ++b) {
    f32x16 part = {};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = b * kF8Block + 64 * h + 32 * lhalf;
      part = mfma_f8(load32(w, k, bytes), load32(x, k, bytes), part);
    }
    const float xs = in ? p.x_scale[static_cast<long long>(src) * kb + b] : 0.0f;
    const float s0 = xs * p.ws0[sc + b], s1 = GATED ? xs * p.ws1[sc + b] : s0;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = fmaf(part[i], i < 8 ? s0 : s1, acc[i]);
  }
  if (!row_in) return;
  uint16_t* out = p.out + static_cast<long long>(r) * p.ldo;
#pragma unroll
  for (int i = 0; i < (GATED ? 8 : 16); ++i) {
    const int c = n0 + 8 * (i / 4) + 4 * lhalf + i % 4;
    const float v = GATED ? silu(acc[i]) * acc[8 + i] : acc[i];
    if (c < p.N) out[c] = f32_to_bf16(v);
  }
}

// Chunks of 32 rows, however the rows are spread over the groups.
long long simple_chunks(const Segments& seg, const GemmF8& a, const GemmF8* sh) {
  const long long own = a.offsets ? seg.total_rows / 32 + std::min(seg.groups, seg.total_rows) : ceil_div(a.static_rows, 32);
  return own + (sh ? ceil_div(sh->static_rows, 32) : 0);
}

int simple_columns(const GemmF8& a, const GemmF8* sh, bool gated) {
  return ceil_div(std::max(a.N, sh ? sh->N : 0), gated ? 64 : 128);
}

bool takes_tiles(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  const int cols = gated ? 128 : 256;
  auto tiles = [&](int rows, int N) { return static_cast<long long>(ceil_div(rows, 192)) * ceil_div(N, cols); };
  if (!a.offsets) return tiles(a.static_rows, a.N) >= 80;
  if (seg.groups * tiles(seg.mean_rows, a.N) + (sh ? tiles(sh->static_rows, sh->N) : 0) < 128) return false;
  return seg.mean_rows >= 75;
}

}  // namespace

bool gemm_f8_supported(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  return simple_chunks(seg, a, sh) <= kMaxItemBlocks && simple_columns(a, sh, gated) <= 65535;
}

hipError_t launch_gemm_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated, hipStream_t st) {
  if (takes_tiles(seg, a, sh, gated)) return launch_tiled_f8(seg, a, sh, gated, st);
  PairF8 pa{a, sh ? *sh : GemmF8{}, seg.total_rows};
  if (!a.offsets) pa = PairF8{GemmF8{}, a, 0};  // a product of static rows alone
  const dim3 grid(static_cast<unsigned>(simple_chunks(seg, a, sh)), simple_columns(a, sh, gated));
  if (grid.x == 0) return hipSuccess;
  if (gated) hipLaunchKernelGGL(simple_f8_kernel<true>, grid, dim3(kThreads), 0, st, pa);
  else hipLaunchKernelGGL(simple_f8_kernel<false>, grid, dim3(kThreads), 0, st, pa);
  return hipGetLastError();
}

}  // namespace moe
