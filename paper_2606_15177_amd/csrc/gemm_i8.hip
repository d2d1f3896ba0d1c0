// Which kernel an 8-bit product takes: 256-row tiles (i8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128
// rows (i8_mid.hip).
#include "i8_impl.h"

namespace moe {
namespace {

// Time of the tiles over that of the items (gate/up and down, kernel trace):
// long K: Mixtral 1.04 and 1.34 at 200 tokens (a mean of 50 rows), 0.86 and
// 0.90 at 300 (75); DSV3 share 1.19 and 1.11 at 1500 (47), 0.99 and 0.94 at
// 2048 (64); shorter: DSV2-Lite 1.10 and 1.35 at 800 (75), 1.00 and 1.05 at
// 1500 (140), 0.92 and 0.85 at 4096 (384); Qwen3 1.07 and 1.05 at 1500 (93),
// 0.99 and 1.02 at 2048 (128).
constexpr int kLongBytes = 4096, kMeanLong = 60, kMeanShort = 130;

bool takes_tiles(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  if (items_blocks(seg, a, sh, gated) > kMaxItemBlocks) return true;
  // few tiles leave CUs idle (16 experts of H 1024, I 512, 3000 tokens: 1.14
  // and 1.12 with 128 tiles)
  const int cols = gated ? 128 : 256;
  const long long tiles = (a.offsets ? static_cast<long long>(seg.groups) * ceil_div(seg.mean_rows, 256) : ceil_div(a.static_rows, 256)) *
                          ceil_div(a.N, cols);
  if (3 * tiles < 2 * device_cu_count()) return false;
  return seg.mean_rows >= (a.K >= kLongBytes ? kMeanLong : kMeanShort);
}

}  // namespace

hipError_t launch_gemm_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  return takes_tiles(seg, a, sh, gated) ? launch_tiled_i8(seg, a, sh, gated, st) : launch_items_i8(seg, a, sh, gated, st);
}

bool gemm_i8_supported(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  return items_blocks(seg, a, sh, gated) <= kMaxItemBlocks || takes_tiles(seg, a, sh, gated);
}

}  // namespace moe
