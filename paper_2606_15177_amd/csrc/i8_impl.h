// Shared definitions of the 8-bit product kernels (gemm_i8.hip's launchers
// choose among them).
#pragma once

#include "ffn_impl.h"
#include "quant_impl.h"

namespace moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
constexpr uint32_t kPastEnd = 0x80000000u;  // an offset past a descriptor's range: reads zeros, no traffic
constexpr int kXcds = 8;
constexpr int kWaitLds = 15 | (3 << 14) | (7 << 4);  // s_waitcnt immediate (see wait_vm): LDS accesses done

// Lane l holds A[row l % 32][16 (l / 32) ..] and B[col l % 32][16 (l / 32) ..]
// (16 bytes), and C[8 (i / 4) + 4 (l / 32) + i % 4][l % 32] in element i.
__device__ __forceinline__ i32x16 mfma_i8(i32x4 a, i32x4 b, i32x16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00020000);
}

// Row offsets as the kernels use them: whatever the array holds, they stay
// within the rows that the caller's buffers have.
__device__ __forceinline__ int row_at(const int32_t* offsets, int g, int rows) { return min(max(offsets[g], 0), rows); }

// load_lds16 of data that no other workgroup reads: its lines leave the L2
// first, and what is shared stays.  Only for whole lines: of a line that two
// loads share the second fetches it again.
constexpr int kLine = 128;
__host__ __device__ __forceinline__ bool whole_lines(const int8_t* rows, long long stride) {
  return ((reinterpret_cast<uintptr_t>(rows) | static_cast<uintptr_t>(stride)) & (kLine - 1)) == 0;
}
__device__ __forceinline__ void load_lds16_once(__amdgpu_buffer_rsrc_t rs, unsigned char* lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)lds, 16, off, 0, 0, 2);
}

// A scalar load: its wait leaves the vector-memory counter, and so the tile
// loads in flight, alone.
typedef const int __attribute__((address_space(4)))* ConstIntPtr;
__device__ __forceinline__ int load_scalar(const int* p, int i) { return ((ConstIntPtr)(uintptr_t)p)[i]; }

// Eight consecutive results, or those of them before N.
__device__ __forceinline__ void store_cols(uint16_t* p, u32x4 v, int col, int N) {
  if (col + 8 <= N) {
    *reinterpret_cast<u32x4_a2*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (col + i < N) p[i] = static_cast<uint16_t>(v[i / 2] >> (16 * (i & 1)));
  }
}

// a over seg and sh (nullable, static rows) in one launch: 256-row tiles (K of
// either past kTiledMinK), or items of up to 128 rows.
constexpr int kTiledMinK = 384;
int tiled_grid(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated);
// In how many parts each of the `rest` tiles past a grid's last whole round runs.
constexpr int kMaxParts = 4;
__host__ __device__ __forceinline__ int last_round_parts(int rest, int grid) {
  return kMaxParts * rest <= grid ? kMaxParts : 2 * rest <= grid ? 2 : 1;
}
hipError_t launch_tiled_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st);
hipError_t launch_items_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st);
// How a launch of items cuts its products: K in `parts`, chunks of `rows` rows.
struct Cut {
  int parts, rows;
  bool half;  // 16 weight rows per wave, not 32
  bool pair = false;  // two workgroups per CU
};
Cut items_cut(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated);
// Bf16 rows (xb), few of them per group (any number is computed): each
// workgroup quantises the rows that it multiplies.
constexpr int kFewRows = 8;
bool few_supported(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated);
Cut few_cut(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated);
hipError_t launch_few_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st);
// Workgroups of launch_items_i8, and how many a grid dimension holds (2^32 - 1
// threads).
long long items_blocks(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated);
constexpr long long kMaxItemBlocks = 0xffffffffll / (4 * kWave);

}  // namespace moe
