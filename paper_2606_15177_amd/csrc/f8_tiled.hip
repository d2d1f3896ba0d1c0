// e4m3 products for prefill-sized batches: persistent tiles of 256 weight rows x 192
// token rows on v_mfma_f32_16x16x128_f8f6f4, operands straight into LDS, one wave per
// SIMD.
//
// Mathematics.  A stage is 128 columns, one block of scales: a result's MFMA starts
// from zero and is added to its accumulator times the row's and the matrix block's
// scale, four fused multiply-adds per lane for the 16 x 16 results of an MFMA of 32
// cycles.  So the accumulators are ordinary registers (192 of 512), the fragments
// accumulation registers.  (32 x 32 x 64 MFMAs have as many additions, 16 at a time
// behind two of them: dense 16384 x 4096 x 7168 467 us where these take 435.)  A result
// is added three MFMAs after it was begun; the weights' scales of a wave's block are one
// (gated two) per stage, held across the lanes for 64 stages, the rows' come with the
// stage.
//
// Bound: the board's power, and issue.  In a row (12000 of them, 5 s) 401 to 411 us (2.4
// PFLOP/s); the first 30 after the card idled up to 575, in turn with other work 425
// to 443 at 1.7 to 1.9 GHz, with the MFMAs busy 53 % of the time; the library's product
// of e4m3 with one scale per tensor, which adds nothing beside its MFMAs, 303.  Of a stage's 1.48 us (256
// workgroups; 1.09 with 64, whose clock is higher) copies with a part left out take
// 1.00 without the loads into LDS, 1.39 without the fragments' reads, 1.22 without the
// additions, 0.88 with the loads alone, 0.82 with the MFMAs alone: what moves costs
// clock.  Without gain: fragments in two sets (430), a second barrier to load earlier
// (1.53 us per stage), row scales four stages at a time, 4, 6 or 16 row tiles to a block,
// weights a stage earlier, all loads behind the barrier (32 experts of gate and up 7168 x
// 2048 with 1000 rows each 925 us, 1040).  A gated tile's end, of vector work alone, is
// 4 to 5 us (a launch without it: 64 experts of 2048 x 1408 with 96 rows 103 and 89).
//
// Tiles.  192 token rows x 256 weight rows of one group, four waves two by two, 96 x
// 128 each: 256 rows would leave no registers for the additions.  Gated products take
// 128 gate and the 128 up rows of the same columns, so that both sums of an output
// meet in one lane, and the tile's 128 hidden columns share a scale: the tile quantises
// them, its rows' largest magnitudes meet in LDS.  (bf16 hidden rows and a launch that
// quantises them: 3 to 12 us more.)  Tile ids go group by group; within a group by
// blocks of 8 row tiles, column tiles within a block, row tiles fastest: the 32 tiles
// that run on one XCD at a time share weight tiles and token tiles in its L2.  Each
// round of the grid is dealt to the XCDs in contiguous shares, the last partly filled
// one too.  The shared experts (static rows) are one more group, first, with operands
// of its own.
//
// Last round.  Where the tiles past the last whole round of the grid are at most
// half (a quarter) of the workgroups, each is run in two (four) parts of its rows on as
// many CUs.  So is an only round: the grid is sized for the parts.
//
// A group's last tile: rows past its end cost no traffic (their loads lie past the
// descriptor's range), and a tile of up to 96 or 64 rows takes half or a third of the
// MFMAs, the four waves side by side along the weights.
//
// Stages and pipeline.  A stage is an X and a W part [192 and 256 rows x 128 bytes] and
// the rows' scales; rings of two X and three W parts take 147 KB of LDS.  16-byte chunk
// c of row r sits at slot c ^ ((r / 2) % 8).  One barrier per stage, before its last two
// row tiles, once the wave's loads of the next stage have landed and its LDS reads
// are done; past it the next stage's fragments take the place of those that are done
// with, and X of two stages on goes into the slot of this one; W of two on went out
// before it, into the slot of the stage before.  Stages run on across tiles.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "f8_impl.h"

namespace moe {
namespace {

constexpr int kTileW = 256, kTileX = 192;
constexpr int kTiledThreads = 4 * kWave;
constexpr int kRow = kF8Block;            // bytes of an LDS row: K per stage
constexpr int kXPart = kTileX * kRow, kWPart = kTileW * kRow;
constexpr int kXSlots = 2, kWSlots = 3;
constexpr int kScaleSlot = 4 * kWave * 4;              // a stage's scales of the rows (the last wave's share unused)
constexpr int kScales = kXSlots * kXPart + kWSlots * kWPart;
constexpr int kTops = kScales + kXSlots * kScaleSlot;  // largest magnitudes of a gated tile's rows, by wave
constexpr int kTiledLds = kTops + 4 * 96 * 4;
static_assert(kTiledLds <= 160 * 1024, "the rings fit");
constexpr int kXLoads = 6, kWLoads = 8;   // per part and wave: 8 rows each
constexpr int kXRows = 8 * kXLoads;       // rows of a wave's X loads
constexpr int kBlockM = 8;

struct TiledF8 {
  GemmF8 g, sp;
  int rows;      // of g's result
  int sp_tiles;  // tiles of sp, 0: none
};

// The lane id, recomputed behind a volatile asm: what is derived from it is
// not hoisted out of the tile loop and holds no register across it.
__device__ __forceinline__ int opaque_lane() {
  int ln;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(ln));
  return ln & 63;  // (known to be small and not negative)
}

// n / d for 0 <= n, 0 < d, n / d < 2^22 (tiles of a launch): the quotient in
// fp32 is off by one at most.
__device__ __forceinline__ int quotient(int n, int d) {
  int q = static_cast<int>(static_cast<float>(n) * __builtin_amdgcn_rcpf(static_cast<float>(d)));
  const int r = n - q * d;
  q += r < 0 ? -1 : r >= d ? 1 : 0;
  return q;
}

// f(0), f(1), ...: a loop of more steps than the compiler unrolls.
template <class F, int... I>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

template <bool GATED, int PFX>
__global__ __launch_bounds__(kTiledThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void tiled_f8_kernel(TiledF8 ta) {
  constexpr int COLS = GATED ? kTileW / 2 : kTileW;  // output columns of a tile
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = lane_id();
  const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int lrow = lane & 15, lquad = lane >> 4;
  const GemmF8& a = ta.g;

  // ---- tiles ----
  // lane L holds the end of the row tiles of groups L + 64 i
  int mt_end[PFX];
  int total_mt = 0;
  if (a.offsets == nullptr) {
    total_mt = ceil_div(a.static_rows, kTileX);
#pragma unroll
    for (int i = 0; i < PFX; ++i) mt_end[i] = 0x7fffffff;
  } else {
#pragma unroll
    for (int i = 0; i < PFX; ++i) {
      const int g = i * kWave + lane;
      int cnt = 0;
      if (g < a.groups) cnt = ceil_div(max(row_at(a.offsets, g + 1, ta.rows) - row_at(a.offsets, g, ta.rows), 0), kTileX);
      int inc = cnt;
#pragma unroll
      for (int off = 1; off < kWave; off <<= 1) {
        const int o = __shfl_up(inc, off);
        if (lane >= off) inc += o;
      }
      mt_end[i] = g < a.groups ? total_mt + inc : 0x7fffffff;
      total_mt += __shfl(inc, kWave - 1);
    }
    total_mt = uniform(total_mt);
  }
  const int tiles_n = ceil_div(a.N, COLS);
  const int total = ta.sp_tiles + total_mt * tiles_n;
  const int n_wg = static_cast<int>(gridDim.x);  // a multiple of the XCDs
  const int xcd = static_cast<int>(blockIdx.x) % kXcds, in_xcd = static_cast<int>(blockIdx.x) / kXcds;
  const int rounds = total / n_wg, rest = total - rounds * n_wg;
  // the last round's tiles in `split` parts of 192 / split rows
  const int split = last_round_parts(rest, n_wg);
  const int rest_lo = static_cast<int>(static_cast<long long>(rest) * split * xcd / kXcds);
  const int rest_hi = static_cast<int>(static_cast<long long>(rest) * split * (xcd + 1) / kXcds);
  int mine = rounds + (in_xcd < rest_hi - rest_lo ? 1 : 0);  // tiles of this workgroup

  struct TileInfo {
    int sp, g, row_base, m0, rows, nt;  // rows of the tile: m0 .. m0 + rows - 1 of the group
  };
  auto tile_info = [&](int i) {
    const int part = rest_lo + in_xcd;  // (in the last round)
    const int id = i < rounds ? i * n_wg + xcd * (n_wg / kXcds) + in_xcd : rounds * n_wg + part / split;
    TileInfo ti;
    ti.sp = id < ta.sp_tiles ? 1 : 0;
    int local = id, mg, m, tn = tiles_n;
    ti.g = 0;
    ti.row_base = 0;
    if (ti.sp) {
      m = ta.sp.static_rows;
      mg = ceil_div(m, kTileX);
      tn = ceil_div(ta.sp.N, COLS);
    } else if (a.offsets == nullptr) {
      local -= ta.sp_tiles;
      m = a.static_rows;
      mg = total_mt;
    } else {
      local -= ta.sp_tiles;
      const int at = quotient(local, tiles_n);  // row tile, of all groups
      int cnt = 0, lo = 0;
#pragma unroll
      for (int k = 0; k < PFX; ++k) {
        const uint64_t before = __ballot(mt_end[k] <= at);  // the groups that end before it: the first ones
        const int n = __popcll(before);
        cnt += n;
        if (n > 0) lo = __builtin_amdgcn_readlane(mt_end[k], n - 1);
      }
      ti.g = cnt;
      ti.row_base = min(max(load_scalar(a.offsets, cnt), 0), ta.rows);
      m = min(max(load_scalar(a.offsets, cnt + 1), 0), ta.rows) - ti.row_base;
      mg = ceil_div(m, kTileX);
      local -= lo * tiles_n;
    }
    // blocks of kBlockM row tiles, the last block with the rest
    const int b = quotient(local, kBlockM * tn), r = local - b * (kBlockM * tn);
    const int bm = min(kBlockM, mg - b * kBlockM);
    ti.nt = quotient(r, bm);
    ti.m0 = (b * kBlockM + r - ti.nt * bm) * kTileX;
    ti.rows = min(kTileX, m - ti.m0);
    if (i == rounds && split > 1) {
      const int at = part % split * (kTileX / split);
      ti.m0 += at;
      ti.rows = min(kTileX / split, ti.rows - at);
    }
    ti.sp = uniform(ti.sp);
    ti.g = uniform(ti.g);
    ti.row_base = uniform(ti.row_base);
    ti.m0 = uniform(ti.m0);
    ti.rows = uniform(ti.rows);
    ti.nt = uniform(ti.nt);
    return ti;
  };
  auto prob = [&](const TileInfo& ti) -> const GemmF8& { return ti.sp ? ta.sp : ta.g; };
  auto stages = [&](const TileInfo& ti) { return ceil_div(prob(ti).K, kRow); };
  auto full_tile = [](const TileInfo& ti) { return ti.rows > kTileX / 2; };

  // (a part past the tile's rows is none)
  if (mine > rounds && split > 1 && tile_info(rounds).rows <= 0) --mine;
  if (mine == 0) return;

  // ---- loads ----
  // Wave w fills rows 48 w .. 48 w + 47 of an X part and 64 w .. 64 w + 63 of a W
  // part; load i writes rows 8 i + lane / 8 of them, slot lane % 8, with the chunk
  // that belongs there.  The scales of rows 64 w .. 64 w + 63 go along with X.
  auto chunk_of = [&](int i, int ln) { return (ln % 8) ^ ((4 * i + ln / 16) % 8); };
  const bool w_up = GATED && (wave & 1);  // the wave's 64 weight rows are all gate or all up rows
  __amdgpu_buffer_rsrc_t rs_x, rs_w, rs_s;
  uint32_t xoff[kXLoads], woff[kWLoads], soff;
  // Source rows of a tile: of the wave's rows of X and of its scales (read two
  // tiles ahead: loads still in flight at the K loop's start, if it used them, would
  // all be waited for there).
  int xr = 0, xr_next = 0, sr = 0, sr_next = 0;
  auto x_rows_of = [&](const TileInfo& ti, int row) {
    const GemmF8& p = prob(ti);
    int v = 0;
    if (p.x_rows) v = p.x_rows[ti.row_base + ti.m0 + min(row, ti.rows - 1)];
    return v;
  };
  auto read_rows = [&](const TileInfo& ti, int& xr_to, int& sr_to) {
    const int ln = opaque_lane();
    xr_to = x_rows_of(ti, kXRows * wave + ln);
    sr_to = x_rows_of(ti, kWave * wave + ln);
  };
  auto x_setup = [&](const TileInfo& ti, bool live) {
    const GemmF8& p = prob(ti);
    const int ln = opaque_lane();
    const int kb = ceil_div(p.K, kRow);
    const long long first = p.x_rows ? 0 : ti.row_base + ti.m0;
    rs_x = rsrc(p.x + first * p.ldx);
    rs_s = rsrc(p.x_scale + first * kb);
    auto source = [&](int row, int listed, int stride) {
      const int own = p.x_rows ? listed : row;
      const bool in = live && row < ti.rows && (!p.x_rows || static_cast<unsigned>(own) < static_cast<unsigned>(p.x_count));
      return in ? own * stride : static_cast<int>(kPastEnd);
    };
    const int at = ln < kXRows ? source(kXRows * wave + ln, xr, static_cast<int>(p.ldx)) : static_cast<int>(kPastEnd);
#pragma unroll
    for (int i = 0; i < kXLoads; ++i)
      xoff[i] = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(4 * (8 * i + ln / 8), at)) + chunk_of(i, ln) * 16;
    soff = static_cast<uint32_t>(source(kWave * wave + ln, sr, 4 * kb));
  };
  auto w_setup = [&](const TileInfo& ti, bool live) {
    const GemmF8& p = prob(ti);
    const int ln = opaque_lane();
    const int col0 = ti.nt * COLS;
    rs_w = rsrc((w_up ? p.w1 : p.w0) + (static_cast<long long>(ti.g) * p.N + col0) * p.ldw);
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
      const int r = 8 * i + ln / 8, col = GATED ? 64 * (wave >> 1) + r : 64 * wave + r;
      woff[i] = live && col0 + col < p.N ? static_cast<uint32_t>(col) * static_cast<uint32_t>(p.ldw) + chunk_of(i, ln) * 16 : kPastEnd;
    }
  };
  // (the range check looks at the lane's offset, not at the scalar one)
  auto load = [&](__amdgpu_buffer_rsrc_t rs, int at, uint32_t off, int kb) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(smem + at), 16, off, kb * kRow, 0, 0);
  };
  auto x_load = [&](int i, int kb, int slot) { load(rs_x, slot * kXPart + wave * (kXRows * kRow) + i * 1024, xoff[i], kb); };
  auto s_load = [&](int kb, int slot) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rs_s, (__attribute__((address_space(3))) void*)(smem + kScales + slot * kScaleSlot + wave * (kWave * 4)), 4, soff, kb * 4, 0, 0);
  };
  auto w_load = [&](int i, int kb, int slot) { load(rs_w, kXSlots * kXPart + slot * kWPart + wave * (64 * kRow) + i * 1024, woff[i], kb); };
  // A tile's last stage: chunks past K (the offsets are not used again)
  auto mask_tail = [&](auto& off, int kb, int bytes) {
    const int ln = opaque_lane();
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(off) / sizeof(off[0])); ++i)
      if (kb * kRow + chunk_of(i, ln) * 16 >= bytes) off[i] = kPastEnd;
  };

  TileInfo cur = tile_info(0), nxt = cur, nn = cur;

  // ---- products ----
  // A wave's block of a tile, in 16 x 16 results: eight tiles of weights by six of
  // rows, the waves two by two; in a tile of up to 96 (64) rows four by six (four),
  // all waves along the weights.
  f32x4 acc[8][6];
  i32x8 xf[6], wf[8];
  // Where the lane's 32 bytes, two chunks, lie in the stage that is read: of the
  // block's first row and first weight row.  (Which columns a lane quarter takes is
  // free, the same in both operands: with chunks q and q + 4 the 16 lanes of an LDS
  // access touch all banks once, with 2 q and 2 q + 1 half of them twice.)
  int x_at[2], w_at[2], s_at = 0;
  auto wave_row = [&](const TileInfo& ti) { return full_tile(ti) ? 96 * (wave & 1) : 0; };
  auto place = [&](const TileInfo& ti, int xs, int ws) {
    const bool full = full_tile(ti);
    const int row = wave_row(ti), w_row = full ? 128 * (wave >> 1) : GATED ? 128 * (wave >> 1) + 32 * (wave & 1) : 64 * wave;
    const int lds = static_cast<int>((uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem);
    s_at = kScales + 4 * (row + lrow);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int at = lds + lrow * kRow + (((lquad + 4 * c) ^ ((lrow / 2) % 8)) << 4);
      x_at[c] = at + row * kRow + xs * kXPart;
      w_at[c] = at + w_row * kRow + kXSlots * kXPart + ws * kWPart;
    }
  };
  auto read32 = [&](i32x8& to, const int (&at)[2], int off) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const i32x4 v = *(const __attribute__((address_space(3))) i32x4*)(static_cast<uintptr_t>(static_cast<uint32_t>(at[c] + off)));
#pragma unroll
      for (int i = 0; i < 4; ++i) to[4 * c + i] = v[i];
    }
  };
  auto read_x = [&](int tm) { read32(xf[tm], x_at, tm * 16 * kRow); };
  // (the second half of the weight tiles: gated the up rows)
  auto read_w = [&](auto tn_c, int t) {
    constexpr int TN = decltype(tn_c)::value;
    constexpr int kSecond = (TN == 8 || GATED ? 64 : 32) * kRow;
    read32(wf[t], w_at, t / (TN / 2) * kSecond + t % (TN / 2) * 16 * kRow);
  };

  // Scales of the matrix blocks: lane l holds those of stages l, l + 64, ... (gated:
  // gate's and up's)
  float cs[2] = {0.0f, 0.0f}, cs_next[2] = {0.0f, 0.0f};
  auto read_scales = [&](const TileInfo& ti, int kb0, float (&to)[2]) {
    const GemmF8& p = prob(ti);
    const int ln = opaque_lane(), kb = ceil_div(p.K, kRow), nb = ceil_div(p.N, kF8Block);
    const int block = GATED ? ti.nt : min(2 * ti.nt + (wave >> 1), nb - 1);
    const long long at = (static_cast<long long>(ti.g) * nb + block) * kb + min(kb0 + ln, kb - 1);
    to[0] = p.ws0[at];
    if constexpr (GATED) to[1] = p.ws1[at];
  };

  // Quantised results leave the registers without LDS (1 to 3 % of a launch; bf16 ones,
  // whose rows are twice as long, lose as much so).  A lane holds columns 4 q .. 4 q + 3 (q
  // its quarter of the wave) of row lane % 16 of each 16 x 16 tile; swaps of neighbouring
  // quarters and of halves between two tiles' registers gather 16 bytes of a row.
  auto swap16 = [](uint32_t& x, uint32_t& y) {  // even quarters x and the next one's, odd ones the last one's y and y
    const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = r[0], y = r[1];
  };
  auto swap32 = [](uint32_t& x, uint32_t& y) {  // the same of halves
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = r[0], y = r[1];
  };

  // A gated tile's hidden rows, quantised: its 128 columns share a scale, so the
  // largest of a row is found over the waves that hold parts of it.
  auto quantize = [&](auto tn_c, auto tm_c, const TileInfo& ti, int col_w) {
    constexpr int TN = decltype(tn_c)::value, TM = decltype(tm_c)::value;
    constexpr int TILES = TN / 2;                    // of 16 columns
    constexpr int PARTS = TN == 8 ? 2 : 4;           // waves that hold a row
    const GemmF8& p = prob(ti);
    const int row_w = wave_row(ti), rows = ti.rows - row_w;
    const int ln = opaque_lane(), erow = ln & 15, eq = ln >> 4;
    const int col_part = TN == 8 ? wave >> 1 : wave;
    uint32_t* tops = reinterpret_cast<uint32_t*>(smem + kTops);  // [row of the tile][part]
    uint32_t h[TM][TILES][2];                        // four columns of a row, as bf16
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
      u16x2 top = {0, 0};
#pragma unroll
      for (int tn = 0; tn < TILES; ++tn) {
        float o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = silu(acc[tn][tm][i]) * acc[tn + TILES][tm][i];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          h[tm][tn][i] = pack_bf16x2(o[2 * i], o[2 * i + 1]);
          top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, h[tm][tn][i] & 0x7fff7fffu));
        }
      }
      uint32_t t = max(static_cast<uint32_t>(top[0]), static_cast<uint32_t>(top[1])), u = t;
      swap16(t, u);
      u = t = max(t, u);
      swap32(t, u);
      if (eq == 0) tops[(row_w + 16 * tm + erow) * PARTS + col_part] = max(t, u);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    phase_barrier();
    const long long row0 = ti.row_base + ti.m0 + row_w;
    const int blocks = ceil_div(p.N, kF8Block), padded = ceil_div(p.N, 16) * 16;
    uint32_t top[TM];
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
      top[tm] = 0;
#pragma unroll
      for (int q = 0; q < PARTS; ++q) top[tm] = max(top[tm], tops[(row_w + 16 * tm + erow) * PARTS + q]);
    }
    const int col = col_w + (TILES == 4 ? 16 * eq : 16 * (eq & 1) + 8 * (eq >> 1));
    uint8_t* to = p.outq + (row0 + erow) * p.ldq + col;
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) {
      const F8Scale sc = f8_scale(top[tm] << 16);
      const bool in = 16 * tm + erow < rows;
      if (eq == 0 && col_part == 0 && in) p.outs[(row0 + 16 * tm + erow) * blocks + ti.nt] = sc.scale;
      uint32_t v[TILES];
#pragma unroll
      for (int tn = 0; tn < TILES; ++tn) v[tn] = quantize_f8_4(h[tm][tn][0], h[tm][tn][1], sc);
      if constexpr (TILES == 4) {
        swap32(v[0], v[2]);
        swap32(v[1], v[3]);
        swap16(v[0], v[1]);
        swap16(v[2], v[3]);
        if (in && col < padded) store16(to + 16 * tm * p.ldq, u32x4{v[0], v[1], v[2], v[3]});
      } else {
        swap16(v[0], v[1]);
        if (in && col < padded) *reinterpret_cast<u32x2*>(to + 16 * tm * p.ldq) = u32x2{v[0], v[1]};
      }
    }
  };
  auto epilogue = [&](auto tn_c, auto tm_c, const TileInfo& ti, int col_w, unsigned char* scr) {
    constexpr int TN = decltype(tn_c)::value, TM = decltype(tm_c)::value;
    constexpr int PASS = 4;                         // tiles of 16 columns stored at a time
    constexpr int CH = 2 * PASS;                    // 16-byte chunks of a row of them
    const GemmF8& p = prob(ti);
    const int row_w = wave_row(ti);
    uint16_t* out = p.out + static_cast<long long>(ti.row_base + ti.m0 + row_w) * p.ldo;
    const int rows = ti.rows - row_w;
    const int ln = opaque_lane();
    const int erow = ln & 15, eq = ln >> 4;
    // 32 rows of CH chunks in one of two buffers, chunk c of row r rotated by the row
    auto place = [&](int buf, int r, int c) { return scr + buf * 4096 + r * (16 * CH) + ((c ^ ((r / (8 / CH)) % CH)) << 4); };
    auto emit = [&](auto inside) {
      constexpr bool kInside = decltype(inside)::value;  // every row and column of the wave's block is a result
#pragma unroll
      for (int pass = 0; pass < TN / PASS; ++pass) {
        // 32 rows' results go out while the next ones' are computed
        const int rr = ln / CH, cc = ln % CH;
        const int col = col_w + 16 * PASS * pass + 8 * cc;
        uint16_t* at = out + rr * p.ldo + col;
        auto put = [&](int m) {
#pragma unroll
          for (int q = 0; q < CH / 2; ++q) {
            const int r = q * (kWave / CH) + rr;
            const u32x4 v = *reinterpret_cast<const u32x4*>(place(m & 1, r, cc));
            uint16_t* to = at + (32 * m + q * (kWave / CH)) * p.ldo;
            if constexpr (kInside) *reinterpret_cast<u32x4_a2*>(to) = v;
            else if (32 * m + r < rows && col < p.N) store_cols(to, v, col, p.N);
          }
        };
#pragma unroll
        for (int m = 0; m < TM / 2; ++m) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int h = 0; h < PASS; ++h) {
              const int tn = PASS * pass + h, tm = 2 * m + t;
              const f32x4 o = acc[tn][tm];
              *reinterpret_cast<u32x2*>(place(m & 1, 16 * t + erow, 2 * h + eq / 2) + 8 * (eq % 2)) =
                  u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
            }
          if (m > 0) put(m - 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        put(TM / 2 - 1);
      }
    };
    if constexpr (GATED) {
      quantize(tn_c, tm_c, ti, col_w);
    } else {
      if (rows >= 16 * TM && col_w + 16 * TN <= p.N) emit(std::true_type{});
      else emit(std::false_type{});
    }
  };

  // ---- the workgroup's tiles ----
  read_rows(cur, xr, sr);
  read_scales(cur, 0, cs_next);
  if (mine > 1) {
    nxt = tile_info(1);
    read_rows(nxt, xr_next, sr_next);
  }
  x_setup(cur, true);
  w_setup(cur, true);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) x_load(i, j, j);
    s_load(j, j);
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) w_load(i, j, j);
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(kXLoads + 1 + kWLoads));  // own stage-0 loads landed
  phase_barrier();
  int xs = 0, ws = 0;  // slots of the stage that is computed
  for (int i = 0; i < mine; ++i) {
    const int nkb = stages(cur), bytes = ceil_div(prob(cur).K, 16) * 16;
    const bool full = full_tile(cur), more = i + 1 < mine;
    const int col_w = cur.nt * COLS + (full ? 2 * (wave >> 1) : wave) * (COLS / 4);
    place(cur, xs, ws);
    xr = xr_next;
    sr = sr_next;
    cs[0] = cs_next[0];
    cs[1] = cs_next[1];
    asm volatile("" : "+v"(xr), "+v"(sr), "+v"(cs[0]), "+v"(cs[1]));  // (waited for here, long after their loads, not in the loop)
    if (more) read_scales(nxt, 0, cs_next);
    if (i + 2 < mine) {
      nn = tile_info(i + 2);
      read_rows(nn, xr_next, sr_next);
    }
#pragma unroll
    for (int tn = 0; tn < 8; ++tn)
#pragma unroll
      for (int tm = 0; tm < 6; ++tm) acc[tn][tm] = f32x4{};
    // Stage j: W of stage j + 2 goes out with its first results, X of stage j + 2
    // with its last ones, past the barrier.
    auto tile = [&](auto tn_c, auto tm_c) {
      constexpr int TN = decltype(tn_c)::value, TM = decltype(tm_c)::value;
      constexpr int TILES = TN * TM;
      // The results of a stage go row tile by row tile.  From kTurn on the next
      // stage's fragments take the place of those that are done with: the rows' first,
      // with the last row tile the weights'.
      constexpr int kTurn = TN * (TM - 2), kLastRows = TN * (TM - 1);
      constexpr int kLag = 3;  // a result is added so many after it was begun
#pragma unroll
      for (int t = 0; t < TN; ++t) read_w(tn_c, t);
#pragma unroll
      for (int t = 0; t < TM; ++t) read_x(t);
      f32x4 part[kLag + 1];
#pragma unroll
      for (int t = 0; t <= kLag; ++t) part[t] = f32x4{};
      float sx[TM], last[GATED ? 2 : 1] = {};  // (last: the scales of the stage's last results)
#pragma unroll
      for (int t = 0; t < TM; ++t) sx[t] = *reinterpret_cast<const float*>(smem + s_at + xs * kScaleSlot + 64 * t);
      auto scale_add = [&](int t, float f) {  // result t of a stage, in its order
        const int tm = t / TN, tn = t % TN;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[tn][tm][e] = fmaf(part[t % (kLag + 1)][e], f, acc[tn][tm][e]);
        asm volatile("" : "+v"(acc[tn][tm]));  // (else the additions are gathered at the end of the stage)
      };
      auto is_up = [](int t) { return GATED && t % TN >= TN / 2 ? 1 : 0; };
      int k2 = 2;  // the stage to load, of this tile or the next one
#pragma clang loop unroll(disable)
      for (int kb = 0; kb < nkb; ++kb) {
        if (kb == nkb - 2) {
          asm volatile("");  // (nothing of it is computed ahead)
          x_setup(nxt, more);
          w_setup(nxt, more);
          k2 = 0;
        } else if (kb == nkb - 3 && bytes % kRow != 0) {
          asm volatile("");
          mask_tail(xoff, k2, bytes);
          mask_tail(woff, k2, bytes);
        }
        const int to_w = ws == 0 ? kWSlots - 1 : ws - 1;
        const float s0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(cs[0]), kb & 63));
        const float s1 = GATED ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(cs[1]), kb & 63)) : s0;
        float s[2][TM];
        __builtin_amdgcn_sched_barrier(0);
        each([&](auto t_c) {
          constexpr int t = decltype(t_c)::value, tm = t / TN, tn = t % TN;
          if constexpr (t == kTurn) {
            // The next stage has landed, for all; this one's fragments are in
            // registers, for all: X of two stages on goes into its slot.
            __builtin_amdgcn_s_waitcnt(wait_vm(kWLoads));
            __builtin_amdgcn_s_waitcnt(kWaitLds);
            phase_barrier();
            const int dx = xs == 0 ? kXPart : -kXPart, dw = ws == kWSlots - 1 ? -(kWSlots - 1) * kWPart : kWPart;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              x_at[c] += dx;
              w_at[c] += dw;
            }
          }
          part[t % (kLag + 1)] = mfma_f8_16(wf[tn], xf[tm], f32x4{});
          __builtin_amdgcn_sched_barrier(0);
          if (tn == 0) s[0][tm] = sx[tm] * s0;
          if (GATED && tn == 0) s[1][tm] = sx[tm] * s1;
          if constexpr (t < kLag) scale_add(TILES - kLag + t, last[is_up(TILES - kLag + t)]);
          else scale_add(t - kLag, s[is_up(t - kLag)][(t - kLag) / TN]);
          if (t < kTurn) {
#pragma unroll
            for (int q = 0; q < kWLoads; ++q)
              if (q * kTurn / kWLoads == t) w_load(q, k2, to_w);
          } else if (t < kLastRows) {
            const int u = t - kTurn;
#pragma unroll
            for (int q = 0; q < kXLoads; ++q)
              if (q * TN / kXLoads == u) x_load(q, k2, xs);
            if (u == TN - 1) s_load(k2, xs);
#pragma unroll
            for (int q = 0; q < TM - 2; ++q)
              if (q * TN / (TM - 2) == u) read_x(q);
          } else {
            read_w(tn_c, tn);
            if (tn == 0) read_x(TM - 2);
          }
          __builtin_amdgcn_sched_barrier(0);
        }, std::make_integer_sequence<int, TILES>{});
        last[0] = s[0][TM - 1];
        if constexpr (GATED) last[1] = s[1][TM - 1];
        const int xs1 = xs ^ 1;
        read_x(TM - 1);
#pragma unroll
        for (int t = 0; t < TM; ++t) sx[t] = *reinterpret_cast<const float*>(smem + s_at + xs1 * kScaleSlot + 64 * t);
        xs = xs1;
        ws = ws == kWSlots - 1 ? 0 : ws + 1;
        ++k2;
        if (((kb + 1) & 63) == 0 && kb + 1 < nkb) {
          read_scales(cur, kb + 1, cs);
          asm volatile("" : "+v"(cs[0]), "+v"(cs[1]));  // (waited for here)
        }
      }
#pragma unroll
      for (int t = 0; t < kLag; ++t) scale_add(TILES - kLag + t, last[is_up(TILES - kLag + t)]);
      epilogue(tn_c, tm_c, cur, col_w, smem + kXSlots * kXPart + (ws == 0 ? kWSlots - 1 : ws - 1) * kWPart + wave * (64 * kRow));
    };
    using Four = std::integral_constant<int, 4>;
    using Six = std::integral_constant<int, 6>;
    using Eight = std::integral_constant<int, 8>;
    if (full) tile(Eight{}, Six{});
    else if (cur.rows > 64) tile(Four{}, Six{});
    else tile(Four{}, Four{});
    cur = nxt;
    nxt = nn;
  }
  __builtin_amdgcn_s_waitcnt(0);  // the dead loads past the last tile: nothing may still write the LDS
}

template <bool GATED, int PFX>
hipError_t launch_pfx(const TiledF8& ta, int grid, hipStream_t st) {
  static unsigned long long lds_set = 0;  // devices with the LDS limit raised
  const hipError_t e = set_max_dynamic_lds(reinterpret_cast<const void*>(&tiled_f8_kernel<GATED, PFX>), kTiledLds, &lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tiled_f8_kernel<GATED, PFX>), dim3(grid), dim3(kTiledThreads), kTiledLds, st, ta);
  return hipGetLastError();
}

}  // namespace

static int shared_tiles(const GemmF8* sh, bool gated) {
  return sh ? ceil_div(sh->static_rows, kTileX) * ceil_div(sh->N, gated ? kTileW / 2 : kTileW) : 0;
}

// One workgroup per CU (its LDS), a whole number per XCD; fewer where the tiles
// there may be, in their most parts, are fewer.
int tiled_f8_grid(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  const long long m_tiles = a.offsets ? seg.total_rows / kTileX + std::min(seg.groups, seg.total_rows) : ceil_div(a.static_rows, kTileX);
  const long long tiles = shared_tiles(sh, gated) + m_tiles * ceil_div(a.N, gated ? kTileW / 2 : kTileW);
  return static_cast<int>((std::min<long long>(kMaxParts * tiles, device_cu_count()) + kXcds - 1) / kXcds * kXcds);
}

hipError_t launch_tiled_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated, hipStream_t st) {
  const TiledF8 ta{a, sh ? *sh : GemmF8{}, seg.total_rows, shared_tiles(sh, gated)};
  const int grid = tiled_f8_grid(seg, a, sh, gated);
  if (grid == 0) return hipSuccess;
  if (seg.groups <= kWave) return gated ? launch_pfx<true, 1>(ta, grid, st) : launch_pfx<false, 1>(ta, grid, st);
  if (seg.groups <= 4 * kWave) return gated ? launch_pfx<true, 4>(ta, grid, st) : launch_pfx<false, 4>(ta, grid, st);
  return gated ? launch_pfx<true, 16>(ta, grid, st) : launch_pfx<false, 16>(ta, grid, st);
}

}  // namespace moe
