// Which kernel an 8-bit product takes: 256-row tiles (i8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128
// rows (i8_mid.hip).
#include "i8_impl.h"

namespace moe {
namespace {

// 256-row tiles want rows that fill them and tiles for a good part of the CUs;
// fewer on short K, where an item's turnaround is short too.  Over 400 random
// layers (65 to 8192 tokens, even to Zipf 1 routing, K 392 to 14336) these lines
// choose the faster kernel within 8 % for all but 31 of 760 grouped products
// (1.29 at worst, 0.7 % on average), and over 297 random products of static rows
// for all but 5 (1.38, 0.4 %).  Both sides, us (items, tiles):
//   rows: Qwen3 of 3000 tokens (a mean of 187, 128 groups) gate/up 143 and 136,
//     1500 tokens 115 and 123; DSV2-Lite of 3000 (281) 210 and 187, of 1500 126
//     and 132; 8 experts of K 14336, N 4096 at a mean of 84 110 and 148;
//   many groups of short K, whose last tiles are mostly padding: Qwen3 gate/up
//     at a mean of 358, Zipf 1, 241 and 281, at 312, Zipf 0.6, 203 and 170;
//   few tiles, grouped: 150 of K 896 17 and 23, 85 of K 2960 53 and 47; static:
//     84 of K 5033 72 and 60, 117 of K 1142 18 and 25, 264 of K 796 29 and 34.
constexpr int kMeanRows = 85, kMeanMany = 300;
constexpr int kMany = 64, kManyK = 2048;
constexpr int kShortK = 1500;
constexpr long long kFewTiles = 110, kFewShort = 300, kFewStatic = 80, kFewStaticShort = 128;

bool takes_tiles(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  if (items_blocks(seg, a, sh, gated) > kMaxItemBlocks) return true;
  const int cols = gated ? 128 : 256;
  const bool brief = a.K < kShortK;
  auto tiles = [&](int rows, int N) { return static_cast<long long>(ceil_div(rows, 256)) * ceil_div(N, cols); };
  if (!a.offsets) return tiles(a.static_rows, a.N) >= (brief ? kFewStaticShort : kFewStatic);
  if (seg.groups * tiles(seg.mean_rows, a.N) + (sh ? tiles(sh->static_rows, sh->N) : 0) < (brief ? kFewShort : kFewTiles)) return false;
  return seg.mean_rows >= (seg.groups >= kMany && a.K <= kManyK ? kMeanMany : kMeanRows);
}

}  // namespace

hipError_t launch_gemm_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  if (a.xb) return launch_few_i8(seg, a, sh, gated, st);
  return takes_tiles(seg, a, sh, gated) ? launch_tiled_i8(seg, a, sh, gated, st) : launch_items_i8(seg, a, sh, gated, st);
}

bool gemm_i8_supported(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  return items_blocks(seg, a, sh, gated) <= kMaxItemBlocks || takes_tiles(seg, a, sh, gated);
}

bool gemm_i8_quantizes(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  return seg.max_rows <= kFewRows && (!sh || sh->static_rows <= kFewRows) && few_supported(seg, a, sh, gated);
}

GemmI8Plan plan_gemm_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  if (!a.xb && takes_tiles(seg, a, sh, gated)) return {1, 1, 256};
  const Cut c = a.xb ? few_cut(seg, a, sh, gated) : items_cut(seg, a, sh, gated);
  return {a.xb ? 2 : 0, c.parts, c.rows};
}

}  // namespace moe
