// Which kernel an 8-bit product takes: 256-row tiles (i8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128
// rows (i8_mid.hip).
#include "i8_impl.h"

namespace moe {
namespace {

// 256-row tiles want rows that fill them and tiles for half of the CUs; more on
// short K, where an item's turnaround is short too.  Over 320 random layers (65 to
// 8192 tokens, even to Zipf 1 routing, K 392 to 14336) these lines choose the
// faster kernel within 8 % for all but 34 of 640 grouped products (1.36 at worst,
// 1.1 % on average), and over 300 random products of static rows for all but 17
// (1.49, 1.1 %).  Both sides, us (items, tiles):
//   rows: 8 experts of K 4096, N 14336 at a mean of 67 178 and 186, of 81 225 and
//     196; K 3128, N 904, 34 groups of 80 35 and 29;
//   many groups of short K, whose last tiles are mostly padding: Qwen3 gate/up at a
//     mean of 193 147 and 163, of 252 172 and 206; DSV2-Lite's at 281 216 and 247,
//     at 308 235 and 235, its down at 381 168 and 152;
//   few tiles, grouped: 112 of K 3080 47 and 45, 128 of K 14336 157 and 143; short
//     K: 324 of K 888 24 and 34, 408 of K 1208 52 and 60, 456 of K 480 64 and 54;
//   static: 48 of K 5000 34 and 38, 64 of K 7168 50 and 43, 70 of K 1500 21 and 19,
//     84 of K 5033 71 and 46; short K: 102 of K 844 20 and 17, 117 of K 1142 21 and
//     18, 264 of K 796 35 and 31, 528 of K 829 48 and 55.  (These lines stand a
//     little high: tiles win from about 64 on since an only round runs in parts.)
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

GemmI8Round round_gemm_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, int tiles) {
  const int grid = tiled_grid(seg, a, sh, gated);
  return {grid, grid > 0 ? last_round_parts(tiles % grid, grid) : 0};
}

}  // namespace moe
