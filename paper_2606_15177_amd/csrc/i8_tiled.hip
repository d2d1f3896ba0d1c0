// 8-bit products for prefill-sized batches: persistent 256 x 256 tiles on
// v_mfma_i32_32x32x32_i8, operands straight into LDS, one wave per SIMD.
//
// Bound: the board's power.  An MFMA takes 32 cycles for 32 x 32 x 32 products,
// 16 bytes per lane of either operand; back to back from registers alone they
// run the chip at 1.9 GHz (3.9 POP/s), and what else moves costs clock: eight
// waves that only read LDS at 112 bytes a cycle pull it down to 1.3 GHz.  So the
// waves are few and their blocks as square as they come: four waves, 128 x 128
// each, read eight 1 KB fragments per 16 MFMAs (eight waves of 64 x 128 read
// twelve and issued four times the scalar instructions: dense 16384 x 4096 x
// 7168 in 510 us where these take 466, in one sustained run).  Measured beside
// the library's int8 product, in turn: 378 us there and 371 (2.59 POP/s), 425 and
// 418 for 8192 x 8192 x 8192, 241 and 220 for 16384 x 7168 x 2048.
//
// Tiles.  256 token rows x 256 weight rows of one group.  Gated products take
// 128 gate and the 128 up rows of the same columns, so that both sums of an
// output meet in one lane.  Tile ids go group by group; within a group by
// blocks of 8 row tiles, column tiles within a block, row tiles fastest: the 32
// tiles that run on one XCD at a time share weight tiles and token tiles in its
// L2.  Each round of the grid is dealt to the XCDs in contiguous shares, the
// last partly filled one too.  The shared experts (static rows) are one more
// group, first, with operands of its own.
//
// Last round.  Where the tiles past the last whole round of the grid are at most
// half (a quarter) of the workgroups, each is run in two (four) parts of its
// rows on as many CUs.  So is an only round: the grid is sized for the parts (90
// tiles of K 1700 31.2 us on 96 workgroups, 24.0 on 256; 96 of K 7168 70 and 51;
// 128 of K 14336 131 and 112; up to 3 % more where no tile has a second part).
//
// A group's last tile: rows past its end cost no traffic (their loads lie past
// the descriptor's range), and a tile of up to 128 or 64 rows takes half or a
// quarter of the MFMAs, the four waves side by side along the weights.
//
// Stages and pipeline.  K advances by 128 bytes.  A stage is an X and a W part
// [256 rows x 128 bytes]; rings of two X and three W parts take all 160 KB of
// LDS.  (Weights come from HBM, rows mostly from the L2: with three X and two W
// parts 1024 tokens of 16 experts of K 5120 took 217 us, 206 here, DSV3's 32 local
// experts with 512 tokens 434 and 417.  Telling the L2 that weights are read once,
// as the items do, gained up to 6 % where every group has one row tile and lost
// up to 5 % elsewhere.)  16-byte chunk c of row r sits at slot c ^ ((r / 2) % 8),
// which spreads a fragment's rows over the banks.  One barrier per stage, before
// its last K-step, once the wave's loads of the next stage have landed and its LDS
// reads are done; past it X of two stages on goes into the slot of this one, and
// W of three on during the next stage.  Stages run on across tiles.  Within a
// K-step the next one's fragment reads and the loads are spread over the MFMAs in
// the order of their use.  The 256 accumulators fill the accumulation registers.
#include <algorithm>
#include <type_traits>

#include "i8_impl.h"

namespace moe {
namespace {

constexpr int kTile = 256;
constexpr int kTiledThreads = 4 * kWave;
constexpr int kRow = 128;                 // bytes of an LDS row: K per stage
constexpr int kPart = kTile * kRow;       // one operand of a stage: 32 KB
constexpr int kXSlots = 2, kWSlots = 3;
constexpr int kTiledLds = (kXSlots + kWSlots) * kPart;
constexpr int kLoads = 8;                 // per part and wave: 8 rows each
constexpr int kSteps = kRow / 32;         // MFMA K-steps of a stage
constexpr int kBlockM = 8;

struct TiledI8 {
  GemmI8 g, sp;
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

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// An accumulator element, read where it is used: the 256 accumulators fill the
// accumulation registers, and left to itself the compiler copies all of them to
// the other half of the register file at the end of the K loop.
__device__ __forceinline__ float acc_value(int a) {
  int v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
  return static_cast<float>(v);
}

template <bool GATED, int PFX>
__global__ __launch_bounds__(kTiledThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void tiled_i8_kernel(TiledI8 ta) {
  constexpr int COLS = GATED ? kTile / 2 : kTile;  // output columns of a tile
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = lane_id();
  const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int lrow = lane & 31, lhalf = lane >> 5;
  const GemmI8& a = ta.g;

  // ---- tiles ----
  // lane L holds the end of the row tiles of groups L + 64 i
  int mt_end[PFX];
  int total_mt = 0;
  if (a.offsets == nullptr) {
    total_mt = ceil_div(a.static_rows, kTile);
#pragma unroll
    for (int i = 0; i < PFX; ++i) mt_end[i] = 0x7fffffff;
  } else {
#pragma unroll
    for (int i = 0; i < PFX; ++i) {
      const int g = i * kWave + lane;
      int cnt = 0;
      if (g < a.groups) cnt = ceil_div(max(row_at(a.offsets, g + 1, ta.rows) - row_at(a.offsets, g, ta.rows), 0), kTile);
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
  // the last round's tiles in `split` parts of 256 / split rows
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
      mg = ceil_div(m, kTile);
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
      mg = ceil_div(m, kTile);
      local -= lo * tiles_n;
    }
    // blocks of kBlockM row tiles, the last block with the rest
    const int b = quotient(local, kBlockM * tn), r = local - b * (kBlockM * tn);
    const int bm = min(kBlockM, mg - b * kBlockM);
    ti.nt = quotient(r, bm);
    ti.m0 = (b * kBlockM + r - ti.nt * bm) * kTile;
    ti.rows = min(kTile, m - ti.m0);
    if (i == rounds && split > 1) {
      const int at = part % split * (kTile / split);
      ti.m0 += at;
      ti.rows = min(kTile / split, ti.rows - at);
    }
    ti.sp = uniform(ti.sp);
    ti.g = uniform(ti.g);
    ti.row_base = uniform(ti.row_base);
    ti.m0 = uniform(ti.m0);
    ti.rows = uniform(ti.rows);
    ti.nt = uniform(ti.nt);
    return ti;
  };
  auto prob = [&](const TileInfo& ti) -> const GemmI8& { return ti.sp ? ta.sp : ta.g; };
  auto stages = [&](const TileInfo& ti) { return ceil_div(prob(ti).K, kRow); };

  // (a part past the tile's rows is none)
  if (mine > rounds && split > 1 && tile_info(rounds).rows <= 0) --mine;
  if (mine == 0) return;

  // ---- loads ----
  // Wave w fills rows 64 w .. 64 w + 63 of a part; load i writes rows 64 w + 8 i
  // + lane / 8, slot lane % 8, with the chunk that belongs there.
  auto chunk_of = [&](int i, int ln) { return (ln % 8) ^ ((4 * i + ln / 16) % 8); };
  const bool w_up = GATED && (wave & 1);  // the wave's 64 weight rows are all gate or all up rows
  __amdgpu_buffer_rsrc_t rs_x, rs_w;
  uint32_t xoff[kLoads], woff[kLoads];
  // the stages to load next, of their tiles, and their slots
  int x_kb = 0, w_kb = 0, x_nkb = 0, w_nkb = 0, x_bytes = 0, w_bytes = 0, x_slot = 0, w_slot = 0;
  // First row of the wave's block of a tile (see place).
  auto wave_row = [&](const TileInfo& ti) { return ti.rows > kTile / 2 ? 128 * (wave & 1) : 0; };
  // Source rows of a tile: of the wave's 64 rows of a part (read two tiles
  // ahead: loads still in flight at the K loop's start, if it used them, would
  // all be waited for there), and of rows l and 64 + l of its block of the
  // results (read a tile ahead).
  int xr = 0, xr_next = 0, src_row[2];
  auto x_rows_of = [&](const TileInfo& ti) {
    const GemmI8& p = prob(ti);
    int v = 0;
    if (p.x_rows) v = p.x_rows[ti.row_base + ti.m0 + min(64 * wave + opaque_lane(), ti.rows - 1)];
    return v;
  };
  auto result_rows_of = [&](const TileInfo& ti) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    if (p.x_rows) {
#pragma unroll
      for (int t = 0; t < 2; ++t) src_row[t] = p.x_rows[ti.row_base + ti.m0 + min(wave_row(ti) + 64 * t + ln, ti.rows - 1)];
    }
  };
  auto x_setup = [&](const TileInfo& ti, bool live) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    rs_x = rsrc(p.x_rows ? p.x : p.x + static_cast<long long>(ti.row_base + ti.m0) * p.ldx);
    const int own = p.x_rows ? xr : 64 * wave + ln;
    const bool in = live && 64 * wave + ln < ti.rows && (!p.x_rows || static_cast<unsigned>(own) < static_cast<unsigned>(p.x_count));
    const int at = in ? own * static_cast<int>(p.ldx) : static_cast<int>(kPastEnd);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      xoff[i] = static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(4 * (8 * i + ln / 8), at)) + chunk_of(i, ln) * 16;
    x_kb = 0;
    x_nkb = stages(ti);
    x_bytes = ceil_div(p.K, 16) * 16;
  };
  auto w_setup = [&](const TileInfo& ti, bool live) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    const int col0 = ti.nt * COLS;
    rs_w = rsrc((w_up ? p.w1 : p.w0) + (static_cast<long long>(ti.g) * p.N + col0) * p.ldw);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = 8 * i + ln / 8, col = GATED ? 64 * (wave >> 1) + r : 64 * wave + r;
      woff[i] = live && col0 + col < p.N ? static_cast<uint32_t>(col) * static_cast<uint32_t>(p.ldw) + chunk_of(i, ln) * 16 : kPastEnd;
    }
    w_kb = 0;
    w_nkb = stages(ti);
    w_bytes = ceil_div(p.K, 16) * 16;
  };
  // (the range check looks at the lane's offset, not at the scalar one)
  auto load = [&](__amdgpu_buffer_rsrc_t rs, int at, uint32_t off, int kb) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(smem + at), 16, off, kb * kRow, 0, 0);
  };
  auto x_load = [&](int i) { load(rs_x, x_slot + wave * (64 * kRow) + i * 1024, xoff[i], x_kb); };
  auto w_load = [&](int i) { load(rs_w, kXSlots * kPart + w_slot + wave * (64 * kRow) + i * 1024, woff[i], w_kb); };
  // The stream's last stage: chunks past K (the offsets are not used again)
  auto mask_tail = [&](uint32_t (&off)[kLoads], int kb, int bytes) {
    const int ln = opaque_lane();
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (kb * kRow + chunk_of(i, ln) * 16 >= bytes) off[i] = kPastEnd;
  };

  TileInfo cur = tile_info(0), nxt = cur, nn = cur;
  bool more = false;
  // (a product has at least four stages here, so the loads, up to three stages
  // ahead, are on the current tile or the next one)
  auto x_advance = [&]() {
    x_slot ^= kPart;
    if (++x_kb == x_nkb) x_setup(nxt, more);
    else if (x_kb == x_nkb - 1 && x_bytes % kRow != 0) mask_tail(xoff, x_kb, x_bytes);
  };
  auto w_advance = [&]() {
    w_slot = w_slot == (kWSlots - 1) * kPart ? 0 : w_slot + kPart;
    if (++w_kb == w_nkb) w_setup(nxt, more);
    else if (w_kb == w_nkb - 1 && w_bytes % kRow != 0) mask_tail(woff, w_kb, w_bytes);
  };

  // ---- products ----
  // A wave's block of a tile, in 32 x 32 results: four tiles of weights by four
  // of rows, the waves two by two; in a tile of up to 128 (64) rows two by four
  // (two), all waves along the weights.
  i32x4 xf[2][4], wf[2][4];
  i32x16 acc[4][4];
  int frag[kSteps];  // the lane's place in its row of a part, for K-step ks
#pragma unroll
  for (int ks = 0; ks < kSteps; ++ks) frag[ks] = lrow * kRow + (((2 * ks + lhalf) ^ ((lrow / 2) % 8)) << 4);
  // bytes from a part's start to the block's rows, to its weight tiles and to
  // the second half of them (gated: the up rows)
  int x_at = 0, w_at[2] = {0, 0};
  auto place = [&](const TileInfo& ti) {
    const bool full = ti.rows > kTile / 2;
    x_at = wave_row(ti) * kRow;
    w_at[0] = kXSlots * kPart + kRow * (full ? 128 * (wave >> 1) : GATED ? 128 * (wave >> 1) + 32 * (wave & 1) : 64 * wave);
    w_at[1] = w_at[0] + kRow * (full || GATED ? 64 : 32);
  };
  // Fragment q of a K-step, in the order of their first use.
  auto read_frag = [&](auto tn, auto tm, int q, int xs, int ws, int ks, int set) {
    constexpr int TN = decltype(tn)::value, TM = decltype(tm)::value;
    if (q == 1 || q > TN) {
      const int t = q == 1 ? 0 : q - TN;
      if (t < TM) xf[set][t] = *reinterpret_cast<const i32x4*>(smem + xs + x_at + t * 32 * kRow + frag[ks]);
    } else {
      const int t = q == 0 ? 0 : q - 1;
      wf[set][t] = *reinterpret_cast<const i32x4*>(smem + ws + w_at[t / (TN / 2)] + t % (TN / 2) * 32 * kRow + frag[ks]);
    }
  };

  // Scales: of the block's weight rows (lane l: gate l and up l, or rows l and
  // 64 + l), and of its rows l and 64 + l.
  float cs[2], rsc[2];
  int in_x = 0;  // bit t: row 64 t + l is a row of x (else zeros, whatever scale was read)
  auto epilogue = [&](auto tn_c, auto tm_c, const TileInfo& ti, int col_w, unsigned char* scr) {
    constexpr int TN = decltype(tn_c)::value, TM = decltype(tm_c)::value;
    constexpr int TILES = GATED ? TN / 2 : TN;      // of 32 output columns
    constexpr int PASS = TILES < 2 ? TILES : 2;     // ... stored at a time
    constexpr int CH = 4 * PASS;                    // 16-byte chunks of a row of them
    const GemmI8& p = prob(ti);
    const int row_w = wave_row(ti);
    uint16_t* out = p.out + static_cast<long long>(ti.row_base + ti.m0 + row_w) * p.ldo;
    const int rows = ti.rows - row_w;
    auto from_lane = [&](float v, int l) { return __int_as_float(__builtin_amdgcn_ds_bpermute(4 * l, __float_as_int(v))); };
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const int ln = opaque_lane();
    const int erow = ln & 31, eh = ln >> 5;
    float rs[TM];
#pragma unroll
    for (int tm = 0; tm < TM; ++tm) rs[tm] = from_lane((in_x >> (tm / 2)) & 1 ? rsc[tm / 2] : 0.0f, 32 * (tm % 2) + erow);
    // 32 rows of CH chunks in one of two buffers, chunk c of row r rotated by the row
    auto place = [&](int buf, int r, int c) { return scr + buf * 4096 + r * (16 * CH) + ((c ^ ((r / (8 / CH)) % CH)) << 4); };
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");  // the last MFMAs' results are readable (acc_value)
    auto emit = [&](auto inside) {
      constexpr bool kInside = decltype(inside)::value;  // every row and column of the wave's block is a result
#pragma unroll
      for (int pass = 0; pass < TILES / PASS; ++pass) {
        float s0[16 * PASS], s1[16 * PASS];
#pragma unroll
        for (int v = 0; v < 16 * PASS; ++v) {
          const int tn = PASS * pass + v / 16, l = 32 * (tn % 2) + 8 * (v % 16 / 4) + v % 4;
          s0[v] = from_lane(GATED ? cs[0] : cs[tn / 2], l + 4 * eh);
          if constexpr (GATED) s1[v] = from_lane(cs[1], l + 4 * eh);
        }
        // a row tile's results go out while the next one's are computed
        const int rr = ln / CH, cc = ln % CH;
        const int col = col_w + 32 * PASS * pass + 8 * cc;
        uint16_t* at = out + rr * p.ldo + col;
        auto put = [&](int tm) {
#pragma unroll
          for (int q = 0; q < CH / 2; ++q) {
            const int r = q * (kWave / CH) + rr;
            const u32x4 v = *reinterpret_cast<const u32x4*>(place(tm & 1, r, cc));
            uint16_t* to = at + (32 * tm + q * (kWave / CH)) * p.ldo;
            if constexpr (kInside) *reinterpret_cast<u32x4_a2*>(to) = v;
            else if (32 * tm + r < rows && col < p.N) store_cols(to, v, col, p.N);
          }
        };
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
#pragma unroll
          for (int h = 0; h < PASS; ++h)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int tn = PASS * pass + h;
              float o[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int e = 4 * v + i;
                o[i] = acc_value(acc[tn][tm][e]) * s0[16 * h + e] * rs[tm];
                if constexpr (GATED) o[i] = silu(o[i]) * (acc_value(acc[tn + TILES][tm][e]) * s1[16 * h + e] * rs[tm]);
              }
              *reinterpret_cast<u32x2*>(place(tm & 1, erow, 4 * h + v) + 8 * eh) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
            }
          if (tm > 0) put(tm - 1);
          __builtin_amdgcn_sched_barrier(0);  // (accumulators are read a tile at a time)
        }
        put(TM - 1);
      }
    };
    if (rows >= 32 * TM && col_w + 32 * TILES <= p.N) emit(std::true_type{});
    else emit(std::false_type{});
  };

  // ---- the workgroup's tiles ----
  xr = x_rows_of(cur);
  result_rows_of(cur);
  if (mine > 1) {
    nxt = tile_info(1);
    xr_next = x_rows_of(nxt);
  }
  x_setup(cur, true);
  w_setup(cur, true);
  auto load_part = [&](bool x) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (x) x_load(i);
      else w_load(i);
    }
  };
  load_part(true);
  x_advance();
  load_part(false);
  w_advance();
  load_part(true);
  x_advance();
  load_part(false);
  w_advance();
  __builtin_amdgcn_s_waitcnt(wait_vm(2 * kLoads));  // own stage-0 loads landed
  phase_barrier();
  int xs = 0, ws = 0;  // slots of the stage that is computed
  for (int i = 0; i < mine; ++i) {
    const GemmI8& p = prob(cur);
    const int nkb = stages(cur);
    const bool full = cur.rows > kTile / 2;
    const int col_w = cur.nt * COLS + (full ? 2 * (wave >> 1) : wave) * (COLS / 4);
    {
      const int ln = opaque_lane();
      const long long sc = static_cast<long long>(cur.g) * p.N;
      cs[0] = p.ws0[sc + min(col_w + ln, p.N - 1)];
      cs[1] = GATED ? p.ws1[sc + min(col_w + ln, p.N - 1)] : p.ws0[sc + min(col_w + 64 + ln, p.N - 1)];
      in_x = 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int src = p.x_rows ? src_row[t] : cur.row_base + cur.m0 + min(wave_row(cur) + 64 * t + ln, cur.rows - 1);
        const bool in = !p.x_rows || static_cast<unsigned>(src) < static_cast<unsigned>(p.x_count);
        rsc[t] = p.x_scale[in ? src : 0];
        in_x |= in ? 1 << t : 0;
      }
    }
    place(cur);
    more = i + 1 < mine;
    xr = xr_next;
    asm volatile("" : "+v"(xr));  // (waited for here, long after its load, not in the loop)
    if (more) result_rows_of(nxt);
    if (i + 2 < mine) {
      nn = tile_info(i + 2);
      xr_next = x_rows_of(nn);
    }
#pragma unroll
    for (int tn = 0; tn < 4; ++tn)
#pragma unroll
      for (int tm = 0; tm < 4; ++tm) acc[tn][tm] = i32x16{};
    // Stage j: W of stage j + 2 goes out with its first two K-steps, X of stage
    // j + 2 with its last one, past the barrier.
    auto tile = [&](auto tn_c, auto tm_c) {
      constexpr int TN = decltype(tn_c)::value, TM = decltype(tm_c)::value;
      constexpr int FRAGS = TN + TM, MFMAS = TN * TM;
#pragma unroll
      for (int q = 0; q < FRAGS; ++q) read_frag(tn_c, tm_c, q, xs, ws, 0, 0);
      for (int kb = 0; kb < nkb; ++kb) {
        const int xs1 = xs ^ kPart, ws1 = ws == (kWSlots - 1) * kPart ? 0 : ws + kPart;
#pragma unroll
        for (int ks = 0; ks < kSteps; ++ks) {
          const bool last = ks == kSteps - 1;
          if (last) {
            w_advance();
            __builtin_amdgcn_s_waitcnt(wait_vm(kLoads));  // own loads of stage j + 1 landed
            __builtin_amdgcn_s_waitcnt(kWaitLds);
            phase_barrier();
          }
          const int set = ks & 1, nx = last ? xs1 : xs, nw = last ? ws1 : ws, nk = last ? 0 : ks + 1;
          // (the reads past the tile's last stage are not used)
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if (q < FRAGS) read_frag(tn_c, tm_c, q, nx, nw, nk, set ^ 1);
            if (last) x_load(q);
            else if (ks < 2 && q % 2 == 0) w_load(4 * ks + q / 2);
#pragma unroll
            for (int m = q * MFMAS / 8; m < (q + 1) * MFMAS / 8; ++m) {
              const int tm = m / TN, tn = m % TN;
              acc[tn][tm] = mfma_i8(wf[set][tn], xf[set][tm], acc[tn][tm]);
            }
          }
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if (q < FRAGS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (last || (ks < 2 && q % 2 == 0)) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            if (MFMAS >= 8 || q % 2 == 1) __builtin_amdgcn_sched_group_barrier(0x008, MFMAS == 16 ? 2 : 1, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        x_advance();
        xs = xs1;
        ws = ws1;
      }
      // The W part of the tile's last stage is free until this wave's next loads
      // into its own 8 KB of it, with the next tile's first stage.
      epilogue(tn_c, tm_c, cur, col_w, smem + kXSlots * kPart + (ws == 0 ? (kWSlots - 1) * kPart : ws - kPart) + wave * (64 * kRow));
    };
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (full) tile(Four{}, Four{});
    else if (cur.rows > kTile / 4) tile(Two{}, Four{});
    else tile(Two{}, Two{});
    cur = nxt;
    nxt = nn;
  }
  __builtin_amdgcn_s_waitcnt(0);  // the dead loads past the last tile: nothing may still write the LDS
}

template <bool GATED, int PFX>
hipError_t launch_pfx(const TiledI8& ta, int grid, hipStream_t st) {
  static unsigned long long lds_set = 0;  // devices with the LDS limit raised
  const hipError_t e = set_max_dynamic_lds(reinterpret_cast<const void*>(&tiled_i8_kernel<GATED, PFX>), kTiledLds, &lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((tiled_i8_kernel<GATED, PFX>), dim3(grid), dim3(kTiledThreads), kTiledLds, st, ta);
  return hipGetLastError();
}

}  // namespace

static int shared_tiles(const GemmI8* sh, bool gated) {
  return sh ? ceil_div(sh->static_rows, kTile) * ceil_div(sh->N, gated ? kTile / 2 : kTile) : 0;
}

// One workgroup per CU (its LDS), a whole number per XCD; fewer where the tiles
// there may be, in their most parts, are fewer.
int tiled_grid(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  const long long m_tiles = a.offsets ? seg.total_rows / kTile + std::min(seg.groups, seg.total_rows) : ceil_div(a.static_rows, kTile);
  const long long tiles = shared_tiles(sh, gated) + m_tiles * ceil_div(a.N, gated ? kTile / 2 : kTile);
  return static_cast<int>((std::min<long long>(kMaxParts * tiles, device_cu_count()) + kXcds - 1) / kXcds * kXcds);
}

hipError_t launch_tiled_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  const TiledI8 ta{a, sh ? *sh : GemmI8{}, seg.total_rows, shared_tiles(sh, gated)};
  const int grid = tiled_grid(seg, a, sh, gated);
  if (grid == 0) return hipSuccess;
  if (seg.groups <= kWave) return gated ? launch_pfx<true, 1>(ta, grid, st) : launch_pfx<false, 1>(ta, grid, st);
  if (seg.groups <= 4 * kWave) return gated ? launch_pfx<true, 4>(ta, grid, st) : launch_pfx<false, 4>(ta, grid, st);
  return gated ? launch_pfx<true, 16>(ta, grid, st) : launch_pfx<false, 16>(ta, grid, st);
}

}  // namespace moe
