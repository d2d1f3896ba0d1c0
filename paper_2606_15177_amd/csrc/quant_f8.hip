// Rows and matrices of bf16 to e4m3 with one scale per 128 columns of a row, or
// per 128 x 128 block of a matrix (the arithmetic: quant_f8_impl.h).
//
// Bound by HBM: 2 bytes read and 1 written per value, one pass; a group of 128
// is 16 lanes' registers, so rows need no reduction over more lanes than that.
#include <algorithm>

#include "kernels.h"
#include "quant_f8_impl.h"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kThreads / kF8Lanes;  // groups of a workgroup at a time
constexpr int kAhead = 4;                     // times that, their loads in flight together

struct QuantF8Pair {
  QuantF8Args a, b;
  int blocks_a;
};

__device__ __forceinline__ u32x4 load_once(const uint16_t* row, int v, int cols) {
  const int c = v * kVec;
  return c + kVec <= cols ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(row + c)) : load_vec(row, v, cols);
}

// Groups are numbered row by row; a workgroup takes kGroups * kAhead of them at a
// time.
__global__ __launch_bounds__(kThreads) void quantize_rows_f8_kernel(QuantF8Pair p) {
  const bool second = static_cast<int>(blockIdx.x) >= p.blocks_a;
  const QuantF8Args& a = second ? p.b : p.a;
  const int block = static_cast<int>(blockIdx.x) - (second ? p.blocks_a : 0);
  const int blocks = second ? static_cast<int>(gridDim.x) - p.blocks_a : p.blocks_a;
  const int rows = a.n_rows ? min(a.rows, max(*a.n_rows, 0)) : a.rows;
  const int kb = ceil_div(a.cols, kF8Block);
  const long long groups = static_cast<long long>(rows) * kb;
  const int at = static_cast<int>(threadIdx.x) / kF8Lanes, lane16 = static_cast<int>(threadIdx.x) % kF8Lanes;
  for (long long g0 = static_cast<long long>(block) * (kGroups * kAhead); g0 < groups;
       g0 += static_cast<long long>(blocks) * (kGroups * kAhead)) {
    const long long r0 = g0 / kb;
    const int b0 = static_cast<int>(g0 - r0 * kb);
    u32x4 v[kAhead];
    long long row[kAhead];
    int vec[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int b = b0 + i * kGroups + at;  // of row r0, or past its end
      row[i] = r0 + b / kb;
      vec[i] = b % kb * kF8Lanes + lane16;
      v[i] = u32x4{0u, 0u, 0u, 0u};
      if (row[i] < rows && vec[i] * kVec < a.cols) v[i] = load_once(a.x + row[i] * a.ldx, vec[i], a.cols);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const F8Scale s = f8_scale(group_max(max_bits_f32(v[i])));
      if (row[i] >= rows) continue;
      if (lane16 == 0) a.scale[row[i] * kb + vec[i] / kF8Lanes] = s.scale;
      if (vec[i] * kVec < ceil_div(a.cols, 16) * 16)  // the padding to 16 values too, as zeros
        *reinterpret_cast<u32x2*>(a.q + row[i] * a.ldq + vec[i] * kVec) = quantize_f8_vec(v[i], s);
    }
  }
}

// A workgroup per 128 x 128 block, four loads per thread (32 matrices of 2048 x 7168
// 243 us, 5.8 TB/s; with 256 threads and eight loads 4 % more, with 1024 and two 2 %).
// Workgroups in turn on other XCDs each fetched the lines that two blocks share: 24
// matrices of 520 x 1000 12.7 us, 9.9 now.
constexpr int kBlockThreads = 512, kXcds = 8;
__global__ __launch_bounds__(kBlockThreads) void quantize_blocks_f8_kernel(int blocks, int rows, int cols, const uint16_t* x, long long ldx,
                                                                      uint8_t* q, long long ldq, float* scale) {
  constexpr int kRows = kBlockThreads / kF8Lanes, kPasses = kF8Block / kRows;  // rows at a time, and of a thread
  __shared__ uint32_t part[kBlockThreads / kWave];
  const int kb = ceil_div(cols, kF8Block), nb = ceil_div(rows, kF8Block);
  // neighbours, which share lines where rows are not whole lines, on one XCD
  const int per = static_cast<int>(gridDim.x) / kXcds;
  const int block = static_cast<int>(blockIdx.x) % kXcds * per + static_cast<int>(blockIdx.x) / kXcds;
  if (block >= blocks) return;
  const int b = block % kb, n = block / kb % nb, g = block / kb / nb;
  const int at = static_cast<int>(threadIdx.x) / kF8Lanes, vec = b * kF8Lanes + static_cast<int>(threadIdx.x) % kF8Lanes;
  u32x4 v[kPasses];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int r = n * kF8Block + i * kRows + at;
    v[i] = u32x4{0u, 0u, 0u, 0u};
    if (r < rows && vec * kVec < cols) v[i] = load_once(x + (static_cast<long long>(g) * rows + r) * ldx, vec, cols);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) top = max(top, max_bits_f32(v[i]));
  top = wave_max(top);
  if (lane_id() == 0) part[threadIdx.x / kWave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kBlockThreads / kWave; ++w) top = max(top, part[w]);
  const F8Scale s = f8_scale(top);
  if (threadIdx.x == 0) scale[block] = s.scale;
  if (vec * kVec >= ceil_div(cols, 16) * 16) return;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int r = n * kF8Block + i * kRows + at;
    if (r < rows)
      *reinterpret_cast<u32x2*>(q + (static_cast<long long>(g) * rows + r) * ldq + vec * kVec) = quantize_f8_vec(v[i], s);
  }
}

// Enough workgroups to fill the chip many times over; the rest by the loop.
constexpr int kMaxBlocks = 1 << 20;

int quant_blocks(const QuantF8Args& a) {
  const long long groups = static_cast<long long>(a.rows) * ceil_div(a.cols, kF8Block);
  return static_cast<int>(std::min<long long>((groups + kGroups * kAhead - 1) / (kGroups * kAhead), kMaxBlocks));
}

}  // namespace

hipError_t launch_quantize_rows_f8(const QuantF8Args& a, const QuantF8Args* b, hipStream_t st) {
  const QuantF8Pair p{a, b ? *b : QuantF8Args{}, quant_blocks(a)};
  const int grid = p.blocks_a + (b ? quant_blocks(*b) : 0);
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(quantize_rows_f8_kernel, dim3(grid), dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

// A grid dimension holds 2^32 - 1 threads.
bool quantize_blocks_f8_supported(int G, int rows, int cols) {
  auto blocks = [](int n) { return (static_cast<long long>(n) + kF8Block - 1) / kF8Block; };
  const long long per = blocks(rows) * blocks(cols), most = 0xffffffffll / kBlockThreads / kXcds * kXcds;
  return per <= most && G <= most / per;
}

hipError_t launch_quantize_blocks_f8(int G, int rows, int cols, const uint16_t* x, long long ldx, uint8_t* q, long long ldq,
                                     float* scale, hipStream_t st) {
  const long long blocks = static_cast<long long>(G) * ceil_div(rows, kF8Block) * ceil_div(cols, kF8Block);
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(quantize_blocks_f8_kernel, dim3(static_cast<unsigned>((blocks + kXcds - 1) / kXcds * kXcds)), dim3(kBlockThreads), 0, st,
                     static_cast<int>(blocks), rows, cols, x, ldx, q, ldq, scale);
  return hipGetLastError();
}

}  // namespace moe
