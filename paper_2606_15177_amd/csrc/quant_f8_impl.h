// Quantisation to e4m3 with one scale per 128 columns: the largest magnitude a of
// the 128, and the e4m3 values nearest to 448 x / a, ties to even.
//
// From bf16 the e4m3 value is the one that exact arithmetic gives.  y = x * (448 /
// a) in fp32 is within 2^-22 of 448 x / a, relatively.  A tie m between two e4m3
// values has 5 significant bits at most, x and a have 8 and 448 = 7 * 2^6 has 3: so
// 7 x and m a, scaled to integers, are below 2^13, and a quotient that is not m
// lies 2^-13 or more (relatively) from it.  Rounded to 18 significant bits y is m
// exactly where the quotient is, and on the quotient's side of it elsewhere; the
// conversion then rounds to even.
//
// Sixteen lanes hold 128 columns, 8 each: a row of the wave's data-parallel
// moves.
#pragma once

#include "quant_impl.h"

namespace moe {

constexpr int kF8Block = 128;    // columns (and rows of a matrix) that share a scale
constexpr float kF8Max = 448.0f; // largest e4m3 value
constexpr int kF8Lanes = kF8Block / kVec;

// The largest of the values of the 16 lanes that hold a group, in all of them.
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
#define MOE_DPP_MAX(ctrl) v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ctrl, 0xf, 0xf, true)))
  MOE_DPP_MAX(0xB1);   // quad_perm [1 0 3 2]
  MOE_DPP_MAX(0x4E);   // quad_perm [2 3 0 1]
  MOE_DPP_MAX(0x141);  // row_half_mirror
  MOE_DPP_MAX(0x140);  // row_mirror
#undef MOE_DPP_MAX
  return v;
}

// What a group's maximum (fp32 bits of the magnitude) makes of it.
struct F8Scale {
  bool finite;
  float scale, pre, c;
};
__device__ __forceinline__ F8Scale f8_scale(uint32_t top) {
  F8Scale s;
  s.finite = top < 0x7f800000u;
  const float amax = __uint_as_float(top);
  // 448 / a leaves the range of fp32 for the smallest a: those groups are scaled
  // by 2^80 first (exact, but for subnormal fp32 inputs' own spacing)
  s.pre = amax < 0x1p-60f ? 0x1p80f : 1.0f;
  s.c = (s.finite && top != 0u) ? kF8Max / (amax * s.pre) : 0.0f;
  s.scale = s.finite ? amax / kF8Max : __uint_as_float(0x7fc00000u);
  return s;
}

// Of any fp32 values 448 x / a is rounded to fp32 once, and then to e4m3: c is 448 / a
// rounded, f8_rest what that leaves of it, and x c + x rest, added in one operation,
// lies within 2^-47 of the quotient before it is rounded (2^-29 for a past 2^100, whose
// rest is subnormal).  So ties between e4m3 values stay ties, which x c alone, rounded
// twice, leaves in either direction.
__device__ __forceinline__ float f8_rest(uint32_t top, const F8Scale& s) {
  return fmaf(-s.c, __uint_as_float(top) * s.pre, kF8Max) * (s.c * (1.0f / kF8Max));
}
__device__ __forceinline__ float f8_quotient(float x, float rest, const F8Scale& s) {
  const float v = x * s.pre;
  return fmaf(v, s.c, v * rest);
}

// Four scaled values to e4m3.  (A value past 448 by fp32's rounding is still
// nearest to 448: no clamp is needed.)
__device__ __forceinline__ uint32_t pack_f8x4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

// Four bf16 values' e4m3 (zeros in a group that is not finite).
__device__ __forceinline__ uint32_t quantize_f8_4(uint32_t lo, uint32_t hi, const F8Scale& s) {
  if (!s.finite) return 0u;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t v = i < 2 ? lo : hi;
    const float x = __uint_as_float((i & 1) ? (v & 0xffff0000u) : (v << 16));
    y[i] = __uint_as_float((__float_as_uint((x * s.pre) * s.c) + 32u) & ~63u);
  }
  return pack_f8x4(y[0], y[1], y[2], y[3]);
}
__device__ __forceinline__ u32x2 quantize_f8_vec(u32x4 v, const F8Scale& s) {
  return u32x2{quantize_f8_4(v[0], v[1], s), quantize_f8_4(v[2], v[3], s)};
}

// Largest magnitude of eight bf16 values, as fp32 bits.
__device__ __forceinline__ uint32_t max_bits_f32(u32x4 v) {
  const u16x2 m = max_bits(u16x2{0, 0}, v);
  return static_cast<uint32_t>(max(m[0], m[1])) << 16;
}

}  // namespace moe
