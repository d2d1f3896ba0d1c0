// Quantisation of a row of bf16 values to int8: its largest magnitude, and the
// integers 127 x / a rounded to nearest, ties to even.
//
// The integer is the one that exact arithmetic gives.  y = x * (127 / a) in
// fp32 is within 2^-22 of 127 x / a, relatively.  With x and a of 8
// significant bits, a quotient that is not exactly n + 1/2 lies at least 2^-16
// (relatively) from it, and n + 1/2 itself has 8 significant bits: so y,
// rounded to 18 significant bits, is n + 1/2 exactly where the quotient is,
// and on the quotient's side of it elsewhere.  That is two integer
// instructions; an IEEE division per element would be ten.  Adding 1.5 * 2^23
// then rounds to even and leaves the integer in the low byte.
#pragma once

#include "common.h"

namespace moe {

constexpr int kVec = 8;  // values per 16-byte load

// 16 bytes at any bf16 address: rows of odd length start at odd multiples of
// two bytes (global memory takes unaligned vector loads on this target).
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

// What a row's maximum (bf16 bits) makes of it.
struct RowScale {
  bool finite;
  float scale, pre, c;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  RowScale s;
  s.finite = top < 0x7f80u;
  const float amax = __uint_as_float(top << 16);
  // 127 / a leaves the range of fp32 for the smallest a: those rows are
  // scaled by 2^80 first (exact)
  s.pre = amax < 0x1p-60f ? 0x1p80f : 1.0f;
  s.c = (s.finite && top != 0u) ? 127.0f / (amax * s.pre) : 0.0f;
  s.scale = s.finite ? amax / 127.0f : __uint_as_float(0x7fc00000u);
  return s;
}

// Eight values' integers (zeros in a row that is not finite: NaN's bits are no
// integer).
__device__ __forceinline__ u32x2 quantize_vec(u32x4 v, const RowScale& s) {
  if (!s.finite) return u32x2{0u, 0u};
  const float pre = s.pre, c = s.c;
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

}  // namespace moe
