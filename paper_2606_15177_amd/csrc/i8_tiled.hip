// 8-bit products for prefill-sized batches: persistent 256 x 256 tiles on
// v_mfma_i32_32x32x32_i8, operands straight into LDS, two waves per SIMD.
//
// Bound.  An MFMA takes 32 cycles for 32 x 32 x 32 products, 16 bytes per lane
// of either operand: the same bytes per cycle as bf16 at twice the products.
// A wave's 64 x 128 block needs six 1 KB fragment reads per eight MFMAs; with
// the fills the LDS moves 64 KB per 512 cycles of MFMA time, near its 128
// bytes a cycle.
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
// Rows past a group's end cost neither traffic (their loads lie past the
// descriptor's range) nor MFMAs where they fill whole 64-row blocks: a wave
// without rows only loads and waits.  Wave w on SIMD w % 4 takes rows 64 wm and
// columns 128 wn with wm = (w % 4) / 2 + 2 (w / 4), wn = w % 2, so that the two
// waves of a SIMD lie 128 rows apart: a group's last tile of up to 128 rows
// keeps one wave busy on every SIMD and takes about half a tile's MFMA time.
//
// Stages and pipeline.  K advances by 128 bytes.  A stage is an X and a W part
// [256 rows x 128 bytes], each in a slot of a ring of five (all 160 KB of
// LDS): part P in slot P mod 5, X of stage s is P = 2 s, W 2 s + 1.  16-byte
// chunk c of row r sits at slot c ^ ((r / 2) % 8), which spreads a fragment's
// rows over the banks.  One barrier per stage, before its last K-step, once the
// wave's loads of the next stage have landed and its LDS reads are done; past
// it the two slots of the finished stage take W of stage + 2 and X of stage +
// 3, two loads per wave and K-step among the MFMAs.  Stages run on across tiles.
#include <algorithm>
#include <type_traits>

#include "i8_impl.h"

namespace moe {
namespace {

constexpr int kTile = 256;
constexpr int kTiledThreads = 8 * kWave;
constexpr int kRow = 128;                 // bytes of an LDS row: K per stage
constexpr int kPart = kTile * kRow;       // 32 KB
constexpr int kParts = 5;
constexpr int kTiledLds = kParts * kPart;
constexpr int kLoads = 4;                 // per part and wave: 8 rows each
constexpr int kSteps = kRow / 32;         // MFMA K-steps of a stage
constexpr int kBlockM = 8;
constexpr int kWaitLds = 15 | (3 << 14) | (7 << 4);  // lgkmcnt(0)

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

// A scalar load: its wait leaves the vector-memory counter, and so the tile
// loads in flight, alone.
typedef const int __attribute__((address_space(4)))* ConstIntPtr;
__device__ __forceinline__ int load_scalar(const int* p, int i) { return ((ConstIntPtr)(uintptr_t)p)[i]; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

template <bool GATED, int PFX>
__global__ __launch_bounds__(kTiledThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void tiled_i8_kernel(TiledI8 ta) {
  constexpr int COLS = GATED ? kTile / 2 : kTile;  // output columns of a tile
  constexpr int WCOLS = COLS / 2;                  // ... of a wave
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = lane_id();
  const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int wm = ((wave & 3) >> 1) + 2 * (wave >> 2), wn = wave & 1;
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
  const int rest_lo = static_cast<int>(static_cast<long long>(rest) * xcd / kXcds);
  const int rest_hi = static_cast<int>(static_cast<long long>(rest) * (xcd + 1) / kXcds);
  const int mine = rounds + (in_xcd < rest_hi - rest_lo ? 1 : 0);  // tiles of this workgroup
  if (mine == 0) return;

  struct TileInfo {
    int sp, g, row_base, m0, rows, nt;  // rows of the tile: m0 .. m0 + rows - 1 of the group
  };
  auto tile_info = [&](int i) {
    const int id = i < rounds ? i * n_wg + xcd * (n_wg / kXcds) + in_xcd : rounds * n_wg + rest_lo + in_xcd;
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
      const int at = local / tiles_n;  // row tile, of all groups
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
    const int b = local / (kBlockM * tn), r = local - b * (kBlockM * tn);
    const int bm = min(kBlockM, mg - b * kBlockM);
    ti.nt = r / bm;
    ti.m0 = (b * kBlockM + r - ti.nt * bm) * kTile;
    ti.rows = min(kTile, m - ti.m0);
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

  // ---- loads ----
  // Wave w fills rows 32 w .. 32 w + 31 of a part; load i writes rows 32 w + 8 i
  // + lane / 8, slot lane % 8, with the chunk that belongs there.
  auto load_row = [&](int i, int ln) { return 32 * wave + 8 * i + ln / 8; };
  auto chunk_of = [&](int i, int ln) { return (ln % 8) ^ ((load_row(i, ln) / 2) % 8); };
  auto part = [&](int P) { return smem + (P % kParts) * kPart; };
  const bool w_up = GATED && ((wave >> 1) & 1);  // the wave's 32 weight rows are all gate or all up rows
  __amdgpu_buffer_rsrc_t rs_x, rs_w;
  uint32_t xoff[kLoads], woff[kLoads], kx[2], kw[2];
  int x_kb = 0, w_kb = 0, x_nkb = 0, w_nkb = 0, x_bytes = 0, w_bytes = 0;
  int xr[kLoads];  // source rows of the next tile's loads, read a tile ahead
  auto x_rows_of = [&](const TileInfo& ti) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    if (p.x_rows) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) xr[i] = p.x_rows[ti.row_base + ti.m0 + min(load_row(i, ln), ti.rows - 1)];
    }
  };
  auto k_offsets = [&](uint32_t (&k)[2], int kb, int bytes) {
    const int ln = opaque_lane();
#pragma unroll
    for (int i = 0; i < 2; ++i) k[i] = static_cast<uint32_t>(kb * kRow) | (kb * kRow + chunk_of(i, ln) * 16 < bytes ? 0u : kPastEnd);
  };
  auto x_setup = [&](const TileInfo& ti, bool live) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    rs_x = rsrc(p.x_rows ? p.x : p.x + static_cast<long long>(ti.row_base + ti.m0) * p.ldx);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = load_row(i, ln);
      const int src = p.x_rows ? xr[i] : r;
      const bool ok = live && r < ti.rows && (!p.x_rows || static_cast<unsigned>(src) < static_cast<unsigned>(p.x_count));
      xoff[i] = ok ? static_cast<uint32_t>(src) * static_cast<uint32_t>(p.ldx) + chunk_of(i, ln) * 16 : kPastEnd;
    }
    x_kb = 0;
    x_nkb = stages(ti);
    x_bytes = ceil_div(p.K, 16) * 16;
    k_offsets(kx, 0, x_bytes);
  };
  auto w_setup = [&](const TileInfo& ti, bool live) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    const int col0 = ti.nt * COLS;
    rs_w = rsrc((w_up ? p.w1 : p.w0) + (static_cast<long long>(ti.g) * p.N + col0) * p.ldw);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = load_row(i, ln);
      const int col = GATED ? (r >> 7) * 64 + (r & 63) : r;
      woff[i] = live && col0 + col < p.N ? static_cast<uint32_t>(col) * static_cast<uint32_t>(p.ldw) + chunk_of(i, ln) * 16 : kPastEnd;
    }
    w_kb = 0;
    w_nkb = stages(ti);
    w_bytes = ceil_div(p.K, 16) * 16;
    k_offsets(kw, 0, w_bytes);
  };
  auto load = [&](__amdgpu_buffer_rsrc_t rs, unsigned char* dst, const uint32_t (&off)[kLoads], const uint32_t (&k)[2], int i) {
    load_lds16(rs, dst + wave * (32 * kRow) + i * 1024, (off[i] + k[i & 1]) | ((off[i] | k[i & 1]) & kPastEnd));
  };
  auto x_load = [&](int s, int i) { load(rs_x, part(2 * s), xoff, kx, i); };
  auto w_load = [&](int s, int i) { load(rs_w, part(2 * s + 1), woff, kw, i); };

  TileInfo cur = tile_info(0), nxt = cur;
  bool more = false;
  // (a product has at least four stages here, so the loads, up to two stages
  // ahead, are on the current tile or the next one)
  auto x_advance = [&]() {
    if (++x_kb == x_nkb) x_setup(nxt, more);
    else k_offsets(kx, x_kb, x_bytes);
  };
  auto w_advance = [&]() {
    if (++w_kb == w_nkb) w_setup(nxt, more);
    else k_offsets(kw, w_kb, w_bytes);
  };

  // ---- products ----
  i32x4 xf[2][2], wf[2][4];
  i32x16 acc[4][2];
  auto read_frags = [&](int s, int ks, int set) {
    const unsigned char* xp = part(2 * s) + (64 * wm + lrow) * kRow;
    const unsigned char* wp = part(2 * s + 1) + (128 * wn + lrow) * kRow;
    const int slot = ((2 * ks + lhalf) ^ ((lrow / 2) % 8)) << 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) wf[set][t] = *reinterpret_cast<const i32x4*>(wp + t * 32 * kRow + slot);
#pragma unroll
    for (int t = 0; t < 2; ++t) xf[set][t] = *reinterpret_cast<const i32x4*>(xp + t * 32 * kRow + slot);
  };
  auto mfma_set = [&](int set) {
#pragma unroll
    for (int tn = 0; tn < 4; ++tn)
#pragma unroll
      for (int tm = 0; tm < 2; ++tm) acc[tn][tm] = mfma_i8(wf[set][tn], xf[set][tm], acc[tn][tm]);
  };

  // Scales of the wave's columns (lane l: column l, and column 64 + l or, gated,
  // column l of up) and of the lane's two rows.
  float cs[2], rsc[2];
  int src_row[2];
  auto epilogue = [&](const TileInfo& ti, unsigned char* scr) {
    const GemmI8& p = prob(ti);
    const int ln = opaque_lane();
    const int erow = ln & 31, eh = ln >> 5;
    const int col_w = ti.nt * COLS + wn * WCOLS;
    uint16_t* out = p.out + static_cast<long long>(ti.row_base + ti.m0 + 64 * wm) * p.ldo;
    const int rows = ti.rows - 64 * wm;
    // column scale of element 4 v + i of accumulator tile t of 32 columns
    auto col_scale = [&](float c, int t, int v, int i) {
      return __int_as_float(__builtin_amdgcn_ds_bpermute(16 * eh + 4 * (32 * t + 8 * v + i), __float_as_int(c)));
    };
#pragma unroll
    for (int tn = 0; tn < (GATED ? 2 : 4); ++tn) {
      float s0[16], s1[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s0[v] = col_scale(GATED ? cs[0] : cs[tn / 2], tn % 2, v / 4, v % 4);
        if constexpr (GATED) s1[v] = col_scale(cs[1], tn, v / 4, v % 4);
      }
#pragma unroll
      for (int tm = 0; tm < 2; ++tm) {
        uint32_t pk[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          float o[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            o[i] = static_cast<float>(acc[tn][tm][2 * v + i]) * s0[2 * v + i] * rsc[tm];
            if constexpr (GATED) o[i] = silu(o[i]) * (static_cast<float>(acc[tn + 2][tm][2 * v + i]) * s1[2 * v + i] * rsc[tm]);
          }
          pk[v] = pack_bf16x2(o[0], o[1]);
        }
        if constexpr (GATED) {
          const int r = 32 * tm + erow;
#pragma unroll
          for (int q = 0; q < 2; ++q) {  // columns 16 q ..: the lane halves swap to 8 consecutive ones each
            const auto a0 = __builtin_amdgcn_permlane32_swap(pk[4 * q], pk[4 * q + 2], false, false);
            const auto a1 = __builtin_amdgcn_permlane32_swap(pk[4 * q + 1], pk[4 * q + 3], false, false);
            const int col = col_w + 32 * tn + 16 * q + 8 * eh;
            if (r < rows && col < p.N) store_cols(out + r * p.ldo + col, u32x4{a0[0], a1[0], a0[1], a1[1]}, col, p.N);
          }
        } else {
          // 32 rows x 64 bytes of this wave's LDS, chunk c of row r at c ^ ((r / 2) % 4)
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
          for (int v = 0; v < 4; ++v)
            *reinterpret_cast<u32x2*>(scr + erow * 64 + ((v ^ ((erow / 2) % 4)) << 4) + 8 * eh) = u32x2{pk[2 * v], pk[2 * v + 1]};
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int rr = 16 * q + (ln >> 2), c = ln & 3;
            const u32x4 v = *reinterpret_cast<const u32x4*>(scr + rr * 64 + ((c ^ ((rr / 2) % 4)) << 4));
            const int r = 32 * tm + rr, col = col_w + 32 * tn + 8 * c;
            if (r < rows && col < p.N) store_cols(out + r * p.ldo + col, v, col, p.N);
          }
        }
      }
    }
  };

  // ---- the workgroup's tiles ----
  x_rows_of(cur);
  x_setup(cur, true);
  w_setup(cur, true);
  for (int s = 0; s < 2; ++s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x_load(s, i);
    x_advance();
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (s == 0 || i < kLoads / 2) w_load(s, i);
    if (s == 0) w_advance();
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(kLoads + kLoads / 2));  // own stage-0 loads landed
  phase_barrier();
  read_frags(0, 0, 0);
  int j = 0;
  for (int i = 0; i < mine; ++i) {
    more = i + 1 < mine;
    if (more) {
      nxt = tile_info(i + 1);
      x_rows_of(nxt);
    }
    const GemmI8& p = prob(cur);
    const int nkb = stages(cur);
    {
      const int ln = opaque_lane();
      const long long sc = static_cast<long long>(cur.g) * p.N;
      const int col = cur.nt * COLS + wn * WCOLS + ln;
      cs[0] = p.ws0[sc + min(col, p.N - 1)];
      cs[1] = GATED ? p.ws1[sc + min(col, p.N - 1)] : p.ws0[sc + min(col + 64, p.N - 1)];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = cur.row_base + cur.m0 + min(64 * wm + 32 * t + (ln & 31), cur.rows - 1);
        src_row[t] = p.x_rows ? p.x_rows[r] : r;
      }
    }
#pragma unroll
    for (int tn = 0; tn < 4; ++tn)
#pragma unroll
      for (int tm = 0; tm < 2; ++tm) acc[tn][tm] = i32x16{};
    // (compiled twice: a wave without rows has neither reads nor MFMAs)
    auto k_loop = [&](auto with_rows) {
      constexpr bool kRows = decltype(with_rows)::value;
      for (int kb = 0; kb < nkb; ++kb, ++j) {
#pragma unroll
        for (int ks = 0; ks < kSteps - 1; ++ks) {
          if constexpr (kRows) read_frags(j, ks + 1, (ks + 1) & 1);
#pragma unroll
          for (int l = 0; l < kLoads / 2; ++l) {
            if (ks == 0) w_load(j + 1, kLoads / 2 + l);
            else x_load(j + 2, (ks - 1) * (kLoads / 2) + l);
          }
          if (ks == 0) w_advance();
          if constexpr (kRows) mfma_set(ks & 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        x_advance();
        __builtin_amdgcn_s_waitcnt(wait_vm(kLoads));  // own stage j + 1 landed
        __builtin_amdgcn_s_waitcnt(kWaitLds);
        phase_barrier();
        if (kRows && kb == 0) {
          // the rows' scales, through the rows just read (a row outside x is zeros)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const bool in = !p.x_rows || static_cast<unsigned>(src_row[t]) < static_cast<unsigned>(p.x_count);
            rsc[t] = p.x_scale[in ? src_row[t] : 0];
            if (!in) rsc[t] = 0.0f;
          }
        }
        if (kRows || kb == nkb - 1) read_frags(j + 1, 0, 0);  // (past the last stage: a harmless stale read)
#pragma unroll
        for (int l = 0; l < kLoads / 2; ++l) w_load(j + 2, l);
        if constexpr (kRows) mfma_set((kSteps - 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const bool active = 64 * wm < cur.rows;
    if (active) k_loop(std::true_type{});
    else k_loop(std::false_type{});
    // The W part of the tile's last stage is free until this wave loads X of the
    // stage three ahead into its own 4 KB of it.
    if (active) epilogue(cur, part(2 * (j - 1) + 1) + wave * (32 * kRow));
    cur = nxt;
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

hipError_t launch_tiled_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  const int cols = gated ? kTile / 2 : kTile;
  long long m_tiles = a.offsets ? seg.total_rows / kTile + std::min(seg.groups, seg.total_rows) : ceil_div(a.static_rows, kTile);
  TiledI8 ta{a, sh ? *sh : GemmI8{}, seg.total_rows, 0};
  if (sh) ta.sp_tiles = ceil_div(sh->static_rows, kTile) * ceil_div(sh->N, cols);
  const long long tiles = ta.sp_tiles + m_tiles * ceil_div(a.N, cols);
  if (tiles == 0) return hipSuccess;
  // one workgroup per CU (its LDS), a whole number per XCD
  const int grid = static_cast<int>((std::min<long long>(tiles, device_cu_count()) + kXcds - 1) / kXcds * kXcds);
  if (seg.groups <= kWave) return gated ? launch_pfx<true, 1>(ta, grid, st) : launch_pfx<false, 1>(ta, grid, st);
  if (seg.groups <= 4 * kWave) return gated ? launch_pfx<true, 4>(ta, grid, st) : launch_pfx<false, 4>(ta, grid, st);
  return gated ? launch_pfx<true, 16>(ta, grid, st) : launch_pfx<false, 16>(ta, grid, st);
}

}  // namespace moe
