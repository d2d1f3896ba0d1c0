// Which kernel an 8-bit product takes: 256-row tiles (i8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128
// rows (i8_mid.hip).
#include "i8_impl.h"

namespace moe {
namespace {

// 256-row tiles want rows that fill them and tiles for half of the CUs; more on
// short K, where an item's turnaround is short too.  Over 800 random layers (65 to
// 8192 tokens, even to Zipf 1 routing, K 392 to 14336) these lines choose the
// faster kernel within 8 % for all but 75 of 1600 grouped products (1.39 at worst,
// 0.9 % on average), and over 297 random products of static rows for all but 5
// (1.38, 0.4 %).  Both sides, us (items, tiles):
//   rows: 8 experts of K 4096, N 14336 at a mean of 67 178 and 186, of 81 225 and
//     196; K 3128, N 904, 34 groups of 80 54 and 40;
//   many groups of short K, whose last tiles are mostly padding: Qwen3 gate/up at a
//     mean of 193 147 and 163, of 252 172 and 206; DSV2-Lite's at 281 216 and 247,
//     at 308 235 and 235, its down at 381 168 and 152;
//   few tiles, grouped: 116 of K 2936 26 and 39, 126 of K 2408 37 and 29; short K:
//     384 of K 712 28 and 38, 435 of K 1296 86 and 81; static: 84 of K 5033 72 and
//     60, 117 of K 1142 18 and 25, 264 of K 796 29 and 34.
constexpr int kMeanRows = 75, kMeanMany = 300;
constexpr int kMany = 64, kManyK = 2048;
constexpr int kShortK = 1500;
constexpr long long kFewTiles = 128, kFewShort = 400, kFewStatic = 80, kFewStaticShort = 128;

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
  if (!a.xb && takes_tiles(seg, a, sh, gated)) return {1, 1, 256, 0};
  const Cut c = a.xb ? few_cut(seg, a, sh, gated) : items_cut(seg, a, sh, gated);
  return {a.xb ? 2 : 0, c.parts, c.rows, c.half};
}

}  // namespace moe
