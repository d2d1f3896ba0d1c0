// Which kernel an 8-bit product takes: 256-row tiles (i8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128
// rows (i8_mid.hip).
#include "i8_impl.h"

namespace moe {
namespace {

// 256-row tiles want rows that fill them and tiles for a good part of the CUs.
// Over 160 random layers (65 to 8192 tokens, even to Zipf 1 routing; K 392 to
// 14336) and 249 random products of static rows these lines choose the kernel
// that is within 8 % of the faster one for all but 9 of 300 grouped products
// (1.31 at worst, 0.7 % on average; another 160 layers 0.6 %) and all but 4 of
// the others (1.44, 0.5 %).
// Both sides, us (items, tiles):
//   long K (kLongK bytes): Mixtral gate/up at a mean of 50 rows 180 and 190, at
//     75 212 and 199; the DSV3 share's down at 62 rows 171 and 161;
//   shorter: 122 rows of K 1416, N 3432 108 and 92, 97 rows of K 1656 35 and 39;
//   many groups of short K, whose last tiles are mostly padding: Qwen3 gate/up
//     at a mean of 309 rows 214 and 258, at 512 335 and 308, down at 315 149 and
//     165, at 406 205 and 193;
//   few tiles: 593 x 9972 x 1142 (117) 18.0 and 24.2, 11380 x 485 x 6294 (90)
//     94 and 82, 3941 x 2301 x 2281 (144) 57 and 38.
constexpr int kMeanLong = 60, kMeanShort = 110, kMeanMany = 350, kMeanManyGated = 420;
constexpr int kMany = 64, kManyK = 2048;
constexpr long long kFewTiles = 128, kFewStaticTiles = 96;

bool takes_tiles(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  if (items_blocks(seg, a, sh, gated) > kMaxItemBlocks) return true;
  const int cols = gated ? 128 : 256;
  auto tiles = [&](int rows, int N) { return static_cast<long long>(ceil_div(rows, 256)) * ceil_div(N, cols); };
  if (!a.offsets) return tiles(a.static_rows, a.N) >= kFewStaticTiles;
  if (seg.groups * tiles(seg.mean_rows, a.N) + (sh ? tiles(sh->static_rows, sh->N) : 0) < kFewTiles) return false;
  if (a.K >= kLongK) return seg.mean_rows >= kMeanLong;
  if (seg.groups < kMany || a.K > kManyK) return seg.mean_rows >= kMeanShort;
  return seg.mean_rows >= (gated ? kMeanManyGated : kMeanMany);
}

}  // namespace

hipError_t launch_gemm_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  return takes_tiles(seg, a, sh, gated) ? launch_tiled_i8(seg, a, sh, gated, st) : launch_items_i8(seg, a, sh, gated, st);
}

bool gemm_i8_supported(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  return items_blocks(seg, a, sh, gated) <= kMaxItemBlocks || takes_tiles(seg, a, sh, gated);
}

}  // namespace moe
