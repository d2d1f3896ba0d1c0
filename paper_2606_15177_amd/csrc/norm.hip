// The norms around a block, with its gate and the residual (see moe.h), row by row:
//   z = y * rsqrt(mean y^2 + eps) * w_post (or y);  h' = rho h + gate z;
//   x = h' * rsqrt(mean h'^2 + eps) * w;  q, scale: x in e4m3 per 128 columns.
// y is read, or is the weighted sum of the experts' outputs of a token (combine.hip),
// which then is not written and read again.
//
// Bound by HBM: y and h read once, h', x and q written once; the row stays in
// registers, in fp32, from its first load to its last store.  The two means are
// the only exchanges between a row's waves.
#include <algorithm>

#include "kernels.h"
#include "quant_f8_impl.h"

namespace moe {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

__device__ __forceinline__ void unpack(u32x4 v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(v[i] << 16);
    f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}

// Vector v of a row of n values, or those of its values before n.
__device__ __forceinline__ void store_vec(uint16_t* row, int v, int n, const float (&f)[8]) {
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
  const int c = v * kVec;
  if (c + kVec <= n) {
    *reinterpret_cast<u32x4_a2*>(row + c) = o;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (c + i < n) row[c + i] = static_cast<uint16_t>(o[i / 2] >> (16 * (i & 1)));
  }
}

__device__ __forceinline__ u32x4 load_row(const uint16_t* row, int v, int n) {
  return v * kVec < n ? load_vec(row, v, n) : u32x4{0u, 0u, 0u, 0u};
}

// THREADS threads per row, V vectors of 8 columns each; ROWS rows per block at a
// time (THREADS 64: a wave each).
template <int THREADS, int V, bool COMBINE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(NormArgs a) {
  constexpr int WAVES = THREADS / kWave;                        // of a row
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  static_assert(WAVES == 1 || ROWS == 1, "rows of a block: one wave each, or one row");
  __shared__ float part[2][2][WAVES];
  const int tid = static_cast<int>(threadIdx.x) % THREADS;
  const int lane = lane_id();
  // the row's sum of its threads' values, in all of them (two places, taken in
  // turns by rows: a place is written again after every wave has read it)
  int turn = 0;
  auto row_sum = [&](float v, int which) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
      if (lane == 0) part[turn][which][tid / kWave] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += part[turn][which][w];
    }
    return v;
  };
  constexpr bool KEEP = THREADS * V <= 1024 * 2;  // the weights are read once for all rows (the registers hold no more)
  auto weights = [&](const uint16_t* w, int i) { return w ? load_row(w, tid + i * THREADS, a.H) : u32x4{0u, 0u, 0u, 0u}; };
  u32x4 pw[V], nw[V];
  if constexpr (KEEP) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      pw[i] = weights(a.post_weight, i);
      nw[i] = weights(a.weight, i);
    }
  }
  const int nvec = ceil_div(a.H, kVec);
  const float inv_h = 1.0f / static_cast<float>(a.H);
  for (long long t = static_cast<long long>(blockIdx.x) * ROWS + threadIdx.x / THREADS; t < a.T;
       t += static_cast<long long>(gridDim.x) * ROWS, turn ^= 1) {
    float z[V][8];
    u32x4 h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = load_row(a.h + t * a.ldh, tid + i * THREADS, a.H);
    if constexpr (COMBINE) {
      // the weighted sum as launch_combine takes it: j ascending, then the shared term
      constexpr int kAhead = !KEEP ? 1 : V >= 4 || THREADS * V > 1024 ? 2 : V == 2 ? 4 : 8;  // rows whose loads are in flight together
      int pos = -1;
      float w = 0.0f;
      if (lane < a.k) {
        pos = a.inv_pos[t * a.k + lane];
        w = a.topk_w[t * a.k + lane];
      }
      u32x4 sh[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        sh[i] = a.y_shared ? load_row(a.y_shared + t * a.H, tid + i * THREADS, a.H) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] = 0.0f;
      }
      uint64_t left = __ballot(pos >= 0);
      while (left != 0) {
        u32x4 y[kAhead][V];
        float g[kAhead];
        int n = 0;
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          g[q] = 0.0f;
          if (left != 0) {
            const int j = __ffsll(static_cast<long long>(left)) - 1;
            left &= left - 1;
            g[q] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j));
            const uint16_t* row = a.y_perm + static_cast<long long>(__builtin_amdgcn_readlane(pos, j)) * a.H;
#pragma unroll
            for (int i = 0; i < V; ++i) y[q][i] = load_row(row, tid + i * THREADS, a.H);
            n = q + 1;
          }
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          if (q >= n) break;
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float f[8];
            unpack(y[q][i], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[i][e] = fmaf(g[q], f[e], z[i][e]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float f[8];
        unpack(sh[i], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] += f[e];
        if (a.out && tid + i * THREADS < nvec) store_vec(a.out + t * a.H, tid + i * THREADS, a.H, z[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) unpack(a.y ? load_row(a.y + t * a.ldy, tid + i * THREADS, a.H) : u32x4{0u, 0u, 0u, 0u}, z[i]);
    }
    if (a.post_weight) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(z[i][e], z[i][e], s);
      const float post = rsqrtf(row_sum(s, 0) * inv_h + a.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float w[8];
        unpack(KEEP ? pw[i] : weights(a.post_weight, i), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] = z[i][e] * post * (w[e] + a.add);
      }
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int v = tid + i * THREADS;
      if (a.gate && v < nvec) {
        const uint16_t* gate = a.gate + t * a.gate_row;
        float w[8];
        if (a.gate_col) {
          unpack(load_vec(gate, v, a.H), w);
        } else {
          const float one = bf16_to_f32(*gate);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = one;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] *= w[e];
      }
      float hv[8];
      unpack(h[i], hv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[i][e] = v * kVec + e < a.H ? fmaf(a.rho, hv[e], z[i][e]) : 0.0f;
        sum = fmaf(z[i][e], z[i][e], sum);
      }
      if (a.h_out && v < nvec) store_vec(a.h_out + t * a.ldho, v, a.H, z[i]);
    }
    if (!a.x && !a.q) continue;
    const float pre = rsqrtf(row_sum(sum, 1) * inv_h + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int v = tid + i * THREADS;
      float w[8];
      unpack(KEEP ? nw[i] : weights(a.weight, i), w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[i][e] *= pre;
        if (a.weight) z[i][e] = v * kVec + e < a.H ? z[i][e] * (w[e] + a.add) : 0.0f;
      }
      if (a.x && v < nvec) store_vec(a.x + t * a.ldx, v, a.H, z[i]);
      if (a.q) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(z[i][e]) & 0x7fffffffu);
        top = group_max(top);
        const F8Scale s = f8_scale(top);
        if (tid % kF8Lanes == 0 && v < nvec) a.scale[t * ceil_div(a.H, kF8Block) + v / kF8Lanes] = s.scale;
        if (v * kVec < ceil_div(a.H, 16) * 16) {
          u32x2 o = {0u, 0u};
          if (s.finite) {
            const float rest = f8_rest(top, s);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = f8_quotient(z[i][e], rest, s);
            o = u32x2{pack_f8x4(y[0], y[1], y[2], y[3]), pack_f8x4(y[4], y[5], y[6], y[7])};
          }
          *reinterpret_cast<u32x2*>(a.q + t * a.ldq + v * kVec) = o;
        }
      }
    }
  }
}

constexpr int kMaxBlocks = 1 << 20;  // the rest by the loop over rows
constexpr int kFewRowsNorm = 512;    // rows that run at once with 1024 threads each

template <int THREADS, int V>
hipError_t launch_rows(const NormArgs& a, int blocks, hipStream_t st) {
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
  const int grid = norm_blocks(a.T, ROWS, blocks);
  const dim3 threads(ROWS * THREADS);
  if (a.inv_pos) hipLaunchKernelGGL((norm_kernel<THREADS, V, true>), dim3(grid), threads, 0, st, a);
  else hipLaunchKernelGGL((norm_kernel<THREADS, V, false>), dim3(grid), threads, 0, st, a);
  return hipGetLastError();
}

}  // namespace

int norm_blocks(int T, int rows, int most) {
  return static_cast<int>(std::min<long long>((static_cast<long long>(T) + rows - 1) / rows, most));
}

// A wave per row up to 1024 columns, 256 threads past that, more past 8192; where
// there are few rows, as many threads as a row has vectors (us, 1 row of 7168: 4.9
// with 1024 threads, 6.4 with 256; 16384 rows: 236 and 191.  16384 rows of 1000: 24.4
// with a wave, 32.6 with 256 threads; of 4096: 106 with 256, 113 with 512, 150 with a
// wave).  With the combine, whose rows take several rounds of loads, four
// workgroups of the widest kind per CU take rows in turn (16384 of 7168: 251 us a
// workgroup each, 234 in turn).
hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  const bool few = a.T <= kFewRowsNorm;
  if (a.H <= kWave * kVec) return launch_rows<kWave, 1>(a, kMaxBlocks, st);
  if (a.H <= kWave * kVec * 2) return launch_rows<kWave, 2>(a, kMaxBlocks, st);
  if (a.H <= 256 * kVec) return launch_rows<256, 1>(a, kMaxBlocks, st);
  if (a.H <= 512 * kVec) return few ? launch_rows<512, 1>(a, kMaxBlocks, st) : launch_rows<256, 2>(a, kMaxBlocks, st);
  if (a.H <= 1024 * kVec)
    return few ? launch_rows<1024, 1>(a, kMaxBlocks, st) : launch_rows<256, 4>(a, a.inv_pos ? 4 * device_cu_count() : kMaxBlocks, st);
  if (a.H <= 2048 * kVec) return launch_rows<1024, 2>(a, kMaxBlocks, st);
  return launch_rows<1024, 4>(a, kMaxBlocks, st);
}

}  // namespace moe
