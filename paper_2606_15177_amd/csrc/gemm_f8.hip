// Which kernel an e4m3 product takes: tiles of 192 rows (f8_tiled.hip) where the
// groups' rows fill them and the tiles fill the chip, else items of up to 128 rows
// (f8_mid.hip).
#include "f8_impl.h"

namespace moe {
namespace {

// Tiles want rows that fill them (routed and shared ones, each by the share of the weights
// that it multiplies), and more of them than items with K in two parts run at
// once (both sides of that in f8_mid.hip); where rows fill them less, on short K, many.  A
// gated tile also saves the launch that quantises the hidden rows (3 to 12 us).  Both
// sides, us (items, tiles):
//   rows of a group: 8 experts of K 4096, N 14336 gated at a mean of 64 179 and 190, of
//     80 233 and 196; 32 of K 7168, N 2048 gated at 80 222 and 227, at 96 299 and 229;
//     64 of K 2048, N 1408 gated at 96 87 and 104, at 128 112 and 107; 128 of K 2048, N
//     768 gated at 96 104 and 106; 32 of K 2048, N 7168 at 80 102 and 111, at 96 130 and 114;
//   past two items per CU: 16 of K 4096, N 520 at 260 43 and 32; 3 of K 7168, N 3000 at 260 70
//     and 56; 24 of K 700, N 1024 at 90 14.4 and 13.7; 4 of K 7168, N 2048 gated at 130 71 and
//     58; 8 of K 1000, N 1000 gated at 130 15.5 and 17.2;
//   short K, many tiles, not gated: 128 of K 768, N 2048 at 24 53 and 48, at 96 62 and 57,
//     at 256 130 and 97; 64 of K 1408, N 2048 at 64 46 and 47, at 96 58 and 48;
//   static: 64 x 30000 x 4096 31 and 40; 70 x 30000 x 4096 46 and 41, 100 x 33000 x 8200 173
//     and 109, 80 x 40000 x 1000 21 and 17;
//   shared rows (T of them) beside the routed ones, by the rows of a weight row over the
//     whole launch, the layer's us (both products in items, in tiles): 32 groups of K 7168, N
//     2048 with a shared one like them at 61 357 and 376, at 85 397 and 388, at 121 525 and 417,
//     at 158 615 and 468; 64 of K 2048, N 1408, shared 2816, at 73 175 and 187, at 109 222
//     and 200; 8 of K 7168, N 2048, shared 8192, at 168 253 and 259, at 336 383 and 284, at
//     2690 2172 and 1400; 8 of K 2048, N 1024, shared 4096, at 150 98 and 81, at 300 114 and
//     83; 32 of K 4096, N 1536 with one like them at 38 157 and 172, at 61 174 and 174, at 83
//     229 and 189; 20 of K 2056, N 776, shared 2320, at 110 93 and 84;
//   short K of the routed rows alone (items, down in tiles): 64 of K 1408 with a shared K of
//     2816 at 48 161 and 161, with uneven rows 162 and 168, at 73 175 and 180, 174 and 187.
//   Of 475 random layers with shared experts the routed rows alone chose another kernel for
//   44; by all rows 43 of those are faster, 9 % on average, and one 1 % slower.
constexpr int kMeanRows = 85, kMeanShort = 24;
constexpr int kShortK = 1500;
constexpr long long kFewShort = 400;
constexpr int kOneChunk = 64;

bool takes_tiles(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  if (a.K <= kTiledMinK || (sh && sh->K <= kTiledMinK)) return false;
  if (items_f8_blocks(seg, a, sh, gated) > kMaxItemBlocks) return true;
  const bool many = !items_f8_fit(seg, a, sh, gated);
  if (!a.offsets) return a.static_rows > kOneChunk && many;
  // rows of a weight row, over the launch (routed rows alone: their mean)
  const double w = static_cast<double>(a.N) * a.K, w_sh = sh ? static_cast<double>(sh->N) * sh->K : 0.0;
  const double rows = static_cast<double>(seg.mean_rows) * seg.groups * w + (sh ? sh->static_rows * w_sh : 0.0);
  if (rows >= kMeanRows * (seg.groups * w + w_sh)) return many;
  auto tiles = [&](int rows, int N) { return static_cast<long long>(ceil_div(rows, 192)) * ceil_div(N, 256); };
  return !gated && a.K < kShortK && (!sh || sh->K < kShortK) && seg.mean_rows >= kMeanShort &&
         seg.groups * tiles(seg.mean_rows, a.N) + (sh ? tiles(sh->static_rows, sh->N) : 0) >= kFewShort;
}

}  // namespace

hipError_t launch_gemm_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated, hipStream_t st) {
  if (a.xb) return launch_few_f8(seg, a, sh, gated, st);
  return takes_tiles(seg, a, sh, gated) ? launch_tiled_f8(seg, a, sh, gated, st) : launch_items_f8(seg, a, sh, gated, st);
}

bool gemm_f8_quantizes(const Segments& seg, const GemmF8& a, const GemmF8* sh) { return takes_tiles(seg, a, sh, true); }

bool gemm_f8_supported(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  return items_f8_blocks(seg, a, sh, gated) <= kMaxItemBlocks || takes_tiles(seg, a, sh, gated);
}

bool gemm_f8_takes_bf16(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  return seg.max_rows <= kFewRows && (!sh || sh->static_rows <= kFewRows) && few_f8_supported(seg, a, sh, gated);
}

GemmF8Plan plan_gemm_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  if (!a.xb && takes_tiles(seg, a, sh, gated)) return {1, 1, 192, 0, 0};
  const Cut c = a.xb ? few_f8_cut(seg, a, sh, gated) : items_f8_cut(seg, a, sh, gated);
  return {a.xb ? 2 : 0, c.parts, c.rows, c.half, c.pair};
}

}  // namespace moe
