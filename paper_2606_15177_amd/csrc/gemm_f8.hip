// Which kernel an e4m3 product takes: tiles of 192 rows (f8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128 rows
// (f8_mid.hip).
#include "f8_impl.h"

namespace moe {
namespace {

// TODO-COMMENT
constexpr int kMeanRows = 75, kMeanMany = 300;
constexpr int kMany = 64, kManyK = 2048;
constexpr int kShortK = 1500;
constexpr long long kFewTiles = 128, kFewShort = 400, kFewStatic = 80, kFewStaticShort = 128;

bool takes_tiles(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  if (items_f8_blocks(seg, a, sh, gated) > kMaxItemBlocks) return true;
  const int cols = gated ? 128 : 256;
  const bool brief = a.K < kShortK;
  auto tiles = [&](int rows, int N) { return static_cast<long long>(ceil_div(rows, 192)) * ceil_div(N, cols); };
  if (!a.offsets) return tiles(a.static_rows, a.N) >= (brief ? kFewStaticShort : kFewStatic);
  if (seg.groups * tiles(seg.mean_rows, a.N) + (sh ? tiles(sh->static_rows, sh->N) : 0) < (brief ? kFewShort : kFewTiles)) return false;
  return seg.mean_rows >= (seg.groups >= kMany && a.K <= kManyK ? kMeanMany : kMeanRows);
}

}  // namespace

hipError_t launch_gemm_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated, hipStream_t st) {
  return takes_tiles(seg, a, sh, gated) ? launch_tiled_f8(seg, a, sh, gated, st) : launch_items_f8(seg, a, sh, gated, st);
}

bool gemm_f8_quantizes(const Segments& seg, const GemmF8& a, const GemmF8* sh) { return takes_tiles(seg, a, sh, true); }

bool gemm_f8_supported(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  return items_f8_blocks(seg, a, sh, gated) <= kMaxItemBlocks || takes_tiles(seg, a, sh, gated);
}

}  // namespace moe
