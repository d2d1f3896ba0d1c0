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

// THREADS threads per row, V vectors of 8 columns each.
template <int THREADS, int V, bool COMBINE>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a) {
  constexpr int WAVES = THREADS / kWave;
  __shared__ float part[2][WAVES];
  const int tid = static_cast<int>(threadIdx.x);
  const int nvec = ceil_div(a.H, kVec);
  // the row's sum of its threads' values, in all of them
  auto row_sum = [&](float v, int which) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
      if (lane_id() == 0) part[which][tid / kWave] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v += part[which][w];
    }
    return v;
  };
  for (int t = static_cast<int>(blockIdx.x); t < a.T; t += static_cast<int>(gridDim.x)) {
    float z[V][8];
    u32x4 h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int v = tid + i * THREADS;
      h[i] = v < nvec ? load_vec(a.h + t * a.ldh, v, a.H) : u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (COMBINE) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] = 0.0f;
      for (int j = 0; j < a.k; ++j) {
        const int r = a.inv_pos[static_cast<long long>(t) * a.k + j];
        if (r < 0) continue;
        const float w = a.topk_w[static_cast<long long>(t) * a.k + j];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int v = tid + i * THREADS;
          if (v >= nvec) continue;
          float f[8];
          unpack(load16(a.y_perm + static_cast<long long>(r) * a.H + v * kVec), f);
#pragma unroll
          for (int e = 0; e < 8; ++e) z[i][e] = fmaf(w, f[e], z[i][e]);
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int v = tid + i * THREADS;
        if (v >= nvec) continue;
        if (a.y_shared) {
          float f[8];
          unpack(load16(a.y_shared + static_cast<long long>(t) * a.H + v * kVec), f);
#pragma unroll
          for (int e = 0; e < 8; ++e) z[i][e] += f[e];
        }
        if (a.out) store_vec(a.out + static_cast<long long>(t) * a.H, v, a.H, z[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int v = tid + i * THREADS;
        unpack(a.y && v < nvec ? load_vec(a.y + t * a.ldy, v, a.H) : u32x4{0u, 0u, 0u, 0u}, z[i]);
      }
    }
    float post = 1.0f;
    if (a.post_weight) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(z[i][e], z[i][e], s);
      post = rsqrtf(row_sum(s, 0) / static_cast<float>(a.H) + a.eps);
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int v = tid + i * THREADS;
      float w[8], hv[8];
      unpack(h[i], hv);
      if (a.post_weight) {
        unpack(v < nvec ? load_vec(a.post_weight, v, a.H) : u32x4{0u, 0u, 0u, 0u}, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] = z[i][e] * post * (w[e] + a.add);
      }
      if (a.gate && v < nvec) {
        const uint16_t* gate = a.gate + t * a.gate_row;
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
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        z[i][e] = v * kVec + e < a.H ? fmaf(a.rho, hv[e], z[i][e]) : 0.0f;
        sum = fmaf(z[i][e], z[i][e], sum);
      }
      if (a.h_out && v < nvec) store_vec(a.h_out + t * a.ldho, v, a.H, z[i]);
    }
    if (!a.x && !a.q) {
      if constexpr (WAVES > 1) __syncthreads();  // (the sums' place is free)
      continue;
    }
    const float pre = rsqrtf(row_sum(sum, 1) / static_cast<float>(a.H) + a.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int v = tid + i * THREADS;
      float w[8];
      if (a.weight) unpack(v < nvec ? load_vec(a.weight, v, a.H) : u32x4{0u, 0u, 0u, 0u}, w);
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
        const F8Scale s = f8_scale(group_max(top));
        if (tid % kF8Lanes == 0 && v < nvec) a.scale[static_cast<long long>(t) * ceil_div(a.H, kF8Block) + v / kF8Lanes] = s.scale;
        if (v * kVec < ceil_div(a.H, 16) * 16) {
          u32x2 o = {0u, 0u};
          if (s.finite) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = z[i][e] * s.pre * s.c;
            o = u32x2{pack_f8x4(y[0], y[1], y[2], y[3]), pack_f8x4(y[4], y[5], y[6], y[7])};
          }
          *reinterpret_cast<u32x2*>(a.q + t * a.ldq + v * kVec) = o;
        }
      }
    }
    // the row's sums have been read by all (the next row's first exchange comes
    // after another barrier only where y is normed)
    if constexpr (WAVES > 1) __syncthreads();
  }
}

template <int THREADS, int V>
hipError_t launch_rows(const NormArgs& a, hipStream_t st) {
  const int grid = std::min(a.T, 1 << 20);
  if (a.inv_pos) hipLaunchKernelGGL((norm_kernel<THREADS, V, true>), dim3(grid), dim3(THREADS), 0, st, a);
  else hipLaunchKernelGGL((norm_kernel<THREADS, V, false>), dim3(grid), dim3(THREADS), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  if (a.H <= kWave * kVec) return launch_rows<kWave, 1>(a, st);
  if (a.H <= 256 * kVec) return launch_rows<256, 1>(a, st);
  if (a.H <= 1024 * kVec) return launch_rows<1024, 1>(a, st);
  return launch_rows<1024, 4>(a, st);
}

}  // namespace moe
