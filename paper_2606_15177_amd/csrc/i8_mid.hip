// 8-bit products for decode and mid-sized batches: from one token to far fewer
// rows per group than fill 256-row tiles.  Bound by reading the weights of the
// groups that have rows once; groups of many rows add MFMA work.
//
// Items.  A workgroup of four waves takes a chunk of the token rows of one group
// times a block of weight rows.  K undivided: up to 128 token rows, 128 weight
// rows for groups of up to 64 rows (narrow items), 256 or 128 for larger ones
// (wide).  A wave owns blocks of 32 weight rows (gated: 16 gate rows and the 16
// up rows of the same columns, which meet in one lane of the MFMA's result) and
// all rows of the chunk.  Where a launch has few items, KP = 2 or 4 groups of
// waves split K, over a half, a quarter or (KP 4, HALF) an eighth of 128 weight
// rows each and chunks of 64, 32 or 8 token rows, and add their sums through LDS
// (integers: the order changes nothing).  At 256 tokens the gate product of Qwen3
// reads 201 MB in 43 us (4.7 TB/s); 1 x 2048 x 7168 takes 7.1 us with its weights
// in the cache behind the L2, of which a launch of nothing is 2.
//
// Pipeline.  buffer_load_dwordx4 ... lds into a ring of K stages, D - 1 stages
// ahead (its size: item_lds).  One barrier per stage, none where a wave reads its
// own loads alone (KP 4).  With K divided the next stage's fragments are read among
// the MFMAs of one, since then a SIMD has no other wave to run.  Chunks of up to 8
// rows hold no more in the ring.  16-byte chunk c of a row sits at a slot rotated
// by the row, which spreads a fragment's rows over the banks.  Each workgroup
// starts its walk along K elsewhere, so that rows that lie a power of two apart
// spread over the memory channels.
//
// Order.  Items are numbered per kind (shared, wide, narrow) by group, column
// block, chunk; an XCD owns a contiguous run of each kind, so that a group's
// token rows and the weight block that its chunks share stay in one L2.  Within
// an XCD heavy (shared and wide) and narrow items take turns of eight, a
// multiple of its shader engines.
//
// Caches.  Weights that one workgroup alone reads, in whole 128-byte lines, leave
// the L2 first: layers of 16 to 256 tokens are 5 to 11 % faster (us, without the
// hint and with it: Qwen3 of 256 150 and 138, DSV2-Lite of 128 149 and 132, DSV3's
// 32 local experts of 32 290 and 261).  Not where chunks share weights or a stage
// takes half a line (DSV2-Lite of 1021, gate/up: 119 and 160) or parts of two (16
// experts of 4104 x 3600, 16 tokens: 155 and 176), and not in the small launches
// that divide K, whose weights a program may find in the cache behind the L2 again:
// 1 x 2048 x 7168 from HBM 9.9 and 9.5, from that cache 8.2 and 8.8, 32 x 4096 x
// 14336 24.1 and 23.8, 15.2 and 23.0.
#include <algorithm>
#include <type_traits>

#include "i8_impl.h"

namespace moe {
namespace {

constexpr int kChunk = 128;         // token rows of a chunk of a wide item
constexpr int kSplitChunk = 64;     // ... of any item where K is split (32 where there are very few)
constexpr int kFewHalf = 32;        // items (of 32 token rows) up to which they are halved once more, K in 4 parts
constexpr int kBriefChunk = 8;      // ... where no group has more rows
constexpr int kWideRows = 64;       // groups of more rows take wide items
constexpr int kItemRows = 128;      // weight rows of a narrow item
constexpr int kFewWide = 128;       // fewer wide items than this take 128 weight rows: half the CUs' worth
constexpr int kOneWide = 256;       // ... or fewer than this, one per CU, in a launch of fewer items than
constexpr int kSlots = 512;         // workgroups fit the chip
constexpr int kTurn = 8;
constexpr int kItemThreads = 4 * kWave;

// LDS of a workgroup, and so workgroups per CU: two, or one where K is divided
// over chunks of more than 8 rows (the launch has hardly more than one per CU).
// More than the ring is worth keeps the next launch waiting: 80 KB and rings of
// four stages against 160 KB and seven, 1 x 2048 x 7168 8.2 and 9.5 us; 96 against
// 160, 256 x 1024 x 1024 5.1 and 5.4; 128 against 160, 777 x 1003 x 528 6.2 and 6.5.
constexpr int item_lds(int parts, int chunk) {
  return 1024 * (parts == 1 || chunk == kBriefChunk ? 80 : chunk == 32 ? 96 : parts == 2 ? 128 : 160);
}

struct ItemsI8 {
  GemmI8 g;   // groups with device offsets (groups 0: none)
  GemmI8 sp;  // static rows (static_rows 0: none)
  int rows;   // of g's result
};

__device__ __forceinline__ int run_start(int n, int x) { return static_cast<int>(static_cast<long long>(n) * x / kXcds); }

// The wave's loads of stage j have landed.  After them were issued (with AHEAD
// stages in flight behind it) the token loads of the first FIRST stages, whose
// weights went out before, and whole stages.
template <int FIRST, int AHEAD, int XL, int LOADS, int J = 0>
__device__ __forceinline__ void wait_stage(int j) {
  if constexpr (J == FIRST) {
    __builtin_amdgcn_s_waitcnt(wait_vm(AHEAD * LOADS));
  } else {
    if (j == J)
      __builtin_amdgcn_s_waitcnt(wait_vm((FIRST - 1 - J) * XL + (AHEAD - (FIRST - 1 - J)) * LOADS));
    else
      wait_stage<FIRST, AHEAD, XL, LOADS, J + 1>(j);
  }
}

template <bool GATED, int KP, int CHUNK, bool HALF>
__global__ __launch_bounds__(kItemThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void items_i8_kernel(ItemsI8 ma) {
  constexpr int FULL_COLS = GATED ? kItemRows / 2 : kItemRows;  // output columns of 128 weight rows
  constexpr int OUT_COLS = FULL_COLS / KP / (HALF ? 2 : 1);     // ... of a narrow item
  constexpr int WIDE_ROWS = KP > 1 ? 0x7fffffff : kWideRows;    // groups of more rows take wide items
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);

  // ---- which item ----
  const int sp_m = ma.sp.static_rows;
  const int sp_chunks = ceil_div(sp_m, CHUNK);
  // first row and rows of groups g0 + 64 i + lane
  constexpr int kPasses = 4;
  int first_row[kPasses], n_rows[kPasses];
  auto load_groups = [&](int g0) {
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      first_row[i] = n_rows[i] = 0;
      if (g0 + i * kWave < ma.g.groups) {
        const int gg = min(g0 + i * kWave + lane, ma.g.groups);  // past the last group: no rows
        first_row[i] = ma.g.offsets[gg];
        n_rows[i] = ma.g.offsets[min(gg + 1, ma.g.groups)];
      }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      first_row[i] = min(max(first_row[i], 0), ma.rows);
      n_rows[i] = max(min(n_rows[i], ma.rows) - first_row[i], 0);
    }
  };
  // Chunks of the groups, wide and narrow.  Where no group has more than one,
  // they are counted by votes of the lanes.
  int c_wide = 0, c_narrow = 0;
  bool several = false;
  for (int g0 = 0; g0 < ma.g.groups; g0 += kPasses * kWave) {
    load_groups(g0);
    int wide_here = 0, narrow_here = 0, ones = 0;
    bool more = false;
#pragma unroll
    for (int q = 0; q < kPasses; ++q) {
      const int n = ceil_div(n_rows[q], CHUNK);
      const bool w = n_rows[q] > WIDE_ROWS;
      more |= n > 1 || w;
      ones += __popcll(__ballot(n > 0));
      wide_here += w ? n : 0;
      narrow_here += w ? 0 : n;
    }
    if (__ballot(more) != 0) {
      several = true;
#pragma unroll
      for (int off = 1; off < kWave; off <<= 1) {
        wide_here += __shfl_xor(wide_here, off);
        narrow_here += __shfl_xor(narrow_here, off);
      }
      c_wide += __builtin_amdgcn_readfirstlane(wide_here);
      c_narrow += __builtin_amdgcn_readfirstlane(narrow_here);
    } else {
      c_narrow += ones;
    }
  }
  const int narrow_blocks = ma.g.groups > 0 ? ceil_div(ma.g.N, OUT_COLS) : 0;
  const int n_narrow = c_narrow * narrow_blocks;
  auto shared_items = [&](int cols) { return sp_m > 0 ? sp_chunks * ceil_div(ma.sp.N, sp_m > WIDE_ROWS ? cols : OUT_COLS) : 0; };
  int wide_cols = 2 * FULL_COLS;
  const int heavy = shared_items(wide_cols) + c_wide * ceil_div(ma.g.N, wide_cols);
  if (heavy < kFewWide || (heavy < kOneWide && heavy + n_narrow < kSlots)) wide_cols = FULL_COLS;
  const int n_shared = shared_items(wide_cols);
  const int wide_blocks = ceil_div(ma.g.N, wide_cols);
  const int n_wide = c_wide * wide_blocks;
  const int xcd = static_cast<int>(blockIdx.x) % kXcds, i = static_cast<int>(blockIdx.x) / kXcds;
  const int s_lo = run_start(n_shared, xcd), w_lo = run_start(n_wide, xcd), n_lo = run_start(n_narrow, xcd);
  const int my_shared = run_start(n_shared, xcd + 1) - s_lo;
  const int my_heavy = my_shared + run_start(n_wide, xcd + 1) - w_lo;
  const int my_narrow = run_start(n_narrow, xcd + 1) - n_lo;
  if (i >= my_heavy + my_narrow) return;
  const int turns = min(my_heavy, my_narrow) / kTurn;
  bool narrow;
  int idx;
  if (i < 2 * turns * kTurn) {
    narrow = (i / kTurn) & 1;
    idx = i / (2 * kTurn) * kTurn + i % kTurn;
  } else {
    idx = i - turns * kTurn;
    narrow = idx >= my_heavy;
    idx = narrow ? i - my_heavy : idx;
  }
  const bool shared = !narrow && idx < my_shared;
  const bool wide = shared ? sp_m > WIDE_ROWS : !narrow;
  idx = narrow ? n_lo + idx : shared ? s_lo + idx : w_lo + idx - my_shared;
  int g = 0, row_base = 0, m = sp_m, item = idx;
  if (!shared) {
    // the group of the kind's chunk `at`
    const int blocks = wide ? wide_blocks : narrow_blocks;
    const int at = idx / blocks;
    bool found = false;
    for (int g0 = 0, before = 0; !found && g0 < ma.g.groups; g0 += kPasses * kWave) {
      if (ma.g.groups > kPasses * kWave) load_groups(g0);
#pragma unroll
      for (int q = 0; q < kPasses; ++q) {
        if (found || g0 + q * kWave >= ma.g.groups) continue;
        // chunks of the kind in the lane's group, and up to and with it
        const int own = (n_rows[q] > WIDE_ROWS) == wide ? ceil_div(n_rows[q], CHUNK) : 0;
        int inc = own;
        if (several) {
#pragma unroll
          for (int off = 1; off < kWave; off <<= 1) {
            const int o = __shfl_up(inc, off);
            if (lane >= off) inc += o;
          }
        } else {
          const uint64_t has = __ballot(own > 0);
          inc += static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(has >> 32),
                                                            __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(has), 0u)));
        }
        const uint64_t past = __ballot(before + inc > at);
        if (past) {
          const int l = __ffsll(static_cast<long long>(past)) - 1;
          g = g0 + q * kWave + l;
          row_base = __builtin_amdgcn_readlane(first_row[q], l);
          m = __builtin_amdgcn_readlane(n_rows[q], l);
          item = idx - (before + __builtin_amdgcn_readlane(inc - own, l)) * blocks;
          found = true;
        } else {
          before += __builtin_amdgcn_readlane(inc, kWave - 1);
        }
      }
    }
    if (!found) return;  // not reached: idx lies within the groups' items
  }
  const int n_chunks = ceil_div(m, CHUNK);
  int nblk = item / n_chunks;
  int chunk = item - nblk * n_chunks;
  g = __builtin_amdgcn_readfirstlane(g);
  row_base = __builtin_amdgcn_readfirstlane(row_base);
  m = __builtin_amdgcn_readfirstlane(m);
  chunk = __builtin_amdgcn_readfirstlane(chunk);
  nblk = __builtin_amdgcn_readfirstlane(nblk);

  const GemmI8& p = shared ? ma.sp : ma.g;
  const int N = p.N, bytes = ceil_div(p.K, 16) * 16;
  const uint32_t ldx = static_cast<uint32_t>(p.ldx), ldw = static_cast<uint32_t>(p.ldw);
  const int32_t* x_rows = p.x_rows;
  // the group's rows in equal chunks of whole 32-row MFMA tiles
  constexpr int UNIT = CHUNK < 32 ? CHUNK : 32;
  const int chunk_rows = ceil_div(ceil_div(m, n_chunks), UNIT) * UNIT;
  const int m0 = chunk * chunk_rows;
  const int rows = min(chunk_rows, m - m0);
  const int n0 = nblk * (wide ? wide_cols : OUT_COLS);

  const long long scales = static_cast<long long>(g) * N;
  const int8_t* w0 = p.w0 + (scales + n0) * p.ldw;
  const __amdgpu_buffer_rsrc_t rs_w0 = rsrc(w0);
  const __amdgpu_buffer_rsrc_t rs_w1 = rsrc(GATED ? p.w1 + (scales + n0) * p.ldw : w0);
  const __amdgpu_buffer_rsrc_t rs_x = rsrc(x_rows ? p.x : p.x + static_cast<long long>(row_base + m0) * p.ldx);
  const int lrow = lane & 31, lhalf = lane >> 5;
  const bool once = n_chunks == 1 && whole_lines(p.w0, p.ldw);  // this workgroup alone reads its weights

  auto body = [&](auto nsub_c, auto wb_c, auto kp_c, auto bk_c, auto depth_c, auto few_c) {
    constexpr int NSUB = decltype(nsub_c)::value;  // 32-row tiles of tokens
    constexpr int WB = decltype(wb_c)::value;      // 32-row blocks of weights per wave
    constexpr int NK = decltype(kp_c)::value;      // K parts; waves WN apart take the same columns
    constexpr int WN = 4 / NK;                     // waves along the weight rows
    constexpr int BK = decltype(bk_c)::value;      // bytes of K per stage
    constexpr int D = decltype(depth_c)::value;
    constexpr int CPR = BK / 16;                   // 16-byte chunks per LDS row
    constexpr int RPI = kWave / CPR;               // rows per load
    constexpr int SWZ = 16 / CPR;                  // rows that share a rotation
    constexpr bool FEW = decltype(few_c)::value;   // up to 8 rows: the ring holds no more
    constexpr int XR = FEW ? 8 : NSUB * 32;        // token rows of a stage
    constexpr int XPART = XR * BK;                 // ... of one K part
    constexpr int WR = HALF ? 16 : 32;             // weight rows of a block
    constexpr int STAGE = NK * XPART + 4 * WB * WR * BK;
    constexpr int XL = FEW ? 1 : XR / RPI / WN;    // token loads per wave and stage
    constexpr int WL = WB * WR / RPI;              // weight loads per wave and stage
    constexpr int LOADS = XL + WL;
    constexpr int KS = BK / 32;                    // MFMA K-steps per stage
    static_assert(D * STAGE <= item_lds(KP, CHUNK), "the ring fits");
    static_assert(FEW ? RPI == 8 : XL * RPI * WN == XR, "whole loads fill the token rows");
    const int lr = lane / CPR;                     // row of a load
    const int wn = wave % WN, wk = wave / WN;
    // What waits for nothing goes out first: the source rows of the token loads
    // and of the results, then the weights of the first stages; the rest follows.
    auto x_row = [&](int q) { return FEW ? lr : RPI * (WN * q + wn) + lr; };  // (few rows: every wave of a K part loads them)
    int xsrc[XL], src[NSUB];
#pragma unroll
    for (int q = 0; q < XL; ++q) xsrc[q] = x_rows ? x_rows[row_base + m0 + min(x_row(q), rows - 1)] : x_row(q);
#pragma unroll
    for (int s = 0; s < NSUB; ++s) {
      const int r = row_base + m0 + min(32 * s + lrow, rows - 1);
      src[s] = x_rows ? x_rows[r] : r;
    }
    const int nst = ceil_div(ceil_div(bytes, BK), NK);  // stages of a K part (the last part's may lie past K)
    const int rot = static_cast<int>((static_cast<unsigned>(nblk) * 7u + static_cast<unsigned>(g) * 3u) % static_cast<unsigned>(nst));
    // first byte of stage s of the wave's K part
    auto k_at = [&](int s) { return (wk * nst + (rot + s < nst ? rot + s : rot + s - nst)) * BK; };
    uint32_t woff[WL], xoff[XL];
    int wpiece[WL], xpiece[XL];
#pragma unroll
    for (int i = 0; i < WL; ++i) {
      const int r = RPI * i + lr;
      const int b = WB * wn + r / WR;  // block of weights
      const int col = GATED ? 16 * b + (r & 15) : WR * b + r % WR;
      woff[i] = n0 + col < N ? static_cast<uint32_t>(col) * ldw : kPastEnd;
      wpiece[i] = (lane % CPR) ^ ((r / SWZ) % CPR);
    }
    // offset `off` of rows of K at byte k, or past the end
    auto at_k = [&](uint32_t off, int k, bool live) {
      const uint32_t kill = (live && k < bytes ? 0u : kPastEnd) | (off & kPastEnd);
      return (off + static_cast<uint32_t>(k)) | kill;
    };
    auto issue_w = [&](int s, int slot) {
      unsigned char* wl = smem + slot * STAGE + NK * XPART + wave * (WB * WR * BK);
      const int k0 = k_at(s);
      if (KP == 1 && BK == kLine && once) {  // (see Caches above)
#pragma unroll
        for (int i = 0; i < WL; ++i)
          load_lds16_once(GATED && ((RPI * i) & 16) ? rs_w1 : rs_w0, wl + i * 1024, at_k(woff[i], k0 + wpiece[i] * 16, s < nst));
      } else {
#pragma unroll
        for (int i = 0; i < WL; ++i)
          load_lds16(GATED && ((RPI * i) & 16) ? rs_w1 : rs_w0, wl + i * 1024, at_k(woff[i], k0 + wpiece[i] * 16, s < nst));
      }
    };
    auto issue_x = [&](int s, int slot) {
      unsigned char* xl = smem + slot * STAGE + wk * XPART;
      const int k0 = k_at(s);
#pragma unroll
      for (int q = 0; q < XL; ++q)
        load_lds16(rs_x, xl + (FEW ? 0 : RPI * (WN * q + wn) * BK), at_k(xoff[q], k0 + xpiece[q] * 16, s < nst));
    };
#pragma unroll 1
    for (int s = 0; s < D - 1; ++s) issue_w(s, s);
#pragma unroll
    for (int q = 0; q < XL; ++q) {
      const int r = x_row(q);
      const bool ok = r < rows && (!x_rows || static_cast<unsigned>(xsrc[q]) < static_cast<unsigned>(p.x_count));
      xoff[q] = ok ? static_cast<uint32_t>(xsrc[q]) * ldx : kPastEnd;
      xpiece[q] = (lane % CPR) ^ ((r / SWZ) % CPR);
    }
#pragma unroll 1
    for (int s = 0; s < D - 1; ++s) issue_x(s, s);
    // Scales: lane l holds that of weight row l of the wave's WB * 32, and
    // those of the token rows of its results.
    const int wr = lane % (WB * 32);
    const int wcol = n0 + (GATED ? 16 * (WB * wn + wr / 32) + (wr & 15) : WR * WB * wn + wr);
    const float cs = (GATED && (wr & 16) ? p.ws1 : p.ws0)[scales + min(wcol, N - 1)];
    float rsc[NSUB];
    bool in_x[NSUB];  // (else a row of zeros, whatever scale was read)
#pragma unroll
    for (int s = 0; s < NSUB; ++s) {
      in_x[s] = !x_rows || static_cast<unsigned>(src[s]) < static_cast<unsigned>(p.x_count);
      rsc[s] = p.x_scale[in_x[s] ? src[s] : 0];
    }
    i32x16 acc[WB][NSUB];
#pragma unroll
    for (int b = 0; b < WB; ++b)
#pragma unroll
      for (int s = 0; s < NSUB; ++s) acc[b][s] = i32x16{};
    constexpr bool OWN = NK == 4;                    // every wave reads only what it loads itself
    constexpr bool PIPE = NK > 1;                    // a stage's fragments are read among the MFMAs of the one before
    constexpr int SETS = PIPE ? 2 : 1;
    i32x4 wf[SETS][KS][WB], xf[SETS][KS][NSUB];
    auto read_frags = [&](int slot, auto set_c) {
      constexpr int SET = decltype(set_c)::value;
      const unsigned char* xp = smem + slot * STAGE + wk * XPART;
      const unsigned char* wp = smem + slot * STAGE + NK * XPART + wave * (WB * WR * BK);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int at = ((2 * ks + lhalf) ^ ((lrow % WR / SWZ) % CPR)) << 4;
        const int xrow = FEW ? lrow % 8 : lrow;  // (few rows: columns past them are not results)
        const int xat = ((2 * ks + lhalf) ^ ((xrow / SWZ) % CPR)) << 4;
#pragma unroll
        for (int b = 0; b < WB; ++b) wf[SET][ks][b] = *reinterpret_cast<const i32x4*>(wp + (WR * b + lrow % WR) * BK + at);
#pragma unroll
        for (int s = 0; s < NSUB; ++s) xf[SET][ks][s] = *reinterpret_cast<const i32x4*>(xp + (32 * s + xrow) * BK + xat);
      }
    };
    auto multiply = [&](auto set_c) {
      constexpr int SET = decltype(set_c)::value;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int s = 0; s < NSUB; ++s) acc[b][s] = mfma_i8(wf[SET][ks][b], xf[SET][ks][s], acc[b][s]);
    };
    // Stage j has landed, for this wave and (unless it reads its own loads
    // alone) for all; its LDS reads of the stage before are done.
    auto arrive = [&](int j) {
      wait_stage<D - 1, D - 2, XL, LOADS>(j);
      if constexpr (PIPE) __builtin_amdgcn_s_waitcnt(kWaitLds);
      if constexpr (OWN) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      } else {
        phase_barrier();
      }
    };
    auto next_slot = [](int slot) { return slot == D - 1 ? 0 : slot + 1; };
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, SETS - 1>;
    int slot = 0;
    if constexpr (PIPE) {
      // stage j + D goes into the slot of stage j, whose fragments are in registers
      issue_x(D - 1, D - 1);
      issue_w(D - 1, D - 1);
      arrive(0);
      read_frags(0, S0{});
      auto step = [&](int j, auto cur, auto nxt) {
        const int next = next_slot(slot);
        arrive(j + 1);
        issue_x(j + D, slot);
        issue_w(j + D, slot);
        read_frags(next, nxt);  // (past the last stage: not used)
        multiply(cur);
        slot = next;
      };
      for (int j = 0; j < nst; j += 2) {
        step(j, S0{}, S1{});
        if (j + 1 < nst) step(j + 1, S1{}, S0{});
      }
    } else {
      for (int j = 0; j < nst; ++j) {
        arrive(j);
        // stage j + D - 1 into the slot of stage j - 1
        const int into = slot == 0 ? D - 1 : slot - 1;
        issue_x(j + D - 1, into);
        issue_w(j + D - 1, into);
        read_frags(slot, S0{});
        multiply(S0{});
        slot = next_slot(slot);
      }
    }
    __builtin_amdgcn_s_waitcnt(wait_vm(0));  // the loads past the last stage: nothing may still write the LDS
    if constexpr (NK > 1) {
      static_assert((NK - 1) * WN * WB * NSUB * 16 * kWave * 4 <= item_lds(KP, CHUNK), "the partial sums fit the LDS");
      int* red = reinterpret_cast<int*>(smem);
      __syncthreads();  // every wave is past its last stage
      if (wk > 0) {
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int s = 0; s < NSUB; ++s)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              red[((((wk - 1) * WN + wn) * WB + b) * NSUB + s) * (16 * kWave) + v * kWave + lane] = acc[b][s][v];
      }
      __syncthreads();
      if (wk > 0) return;
#pragma unroll
      for (int q = 0; q < NK - 1; ++q)
#pragma unroll
        for (int b = 0; b < WB; ++b)
#pragma unroll
          for (int s = 0; s < NSUB; ++s)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              acc[b][s][v] += red[(((q * WN + wn) * WB + b) * NSUB + s) * (16 * kWave) + v * kWave + lane];
    }
#pragma unroll
    for (int s = 0; s < NSUB; ++s) rsc[s] = in_x[s] ? rsc[s] : 0.0f;
    // ---- results: lane holds C[n = 8 v4 + 4 lhalf + i][t = lrow] of each block ----
    uint16_t* out = p.out + static_cast<long long>(row_base + m0) * p.ldo;
#pragma unroll
    for (int b = 0; b < WB; ++b) {
      float sc[16];
#pragma unroll
      for (int v = 0; v < 16; ++v)
        sc[v] = __int_as_float(__builtin_amdgcn_ds_bpermute(16 * lhalf + 4 * (32 * b + 8 * (v / 4) + v % 4), __float_as_int(cs)));
#pragma unroll
      for (int s = 0; s < NSUB; ++s) {
        const int r = 32 * s + lrow;
#pragma unroll
        for (int h = 0; h < (GATED || HALF ? 1 : 2); ++h) {  // 16 columns each
          uint32_t pk[2][2];
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            float o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = 8 * h + 4 * v + i;
              o[i] = static_cast<float>(acc[b][s][e]) * sc[e] * rsc[s];
              if constexpr (GATED) o[i] = silu(o[i]) * (static_cast<float>(acc[b][s][8 + e]) * sc[8 + e] * rsc[s]);
            }
            pk[v][0] = pack_bf16x2(o[0], o[1]);
            pk[v][1] = pack_bf16x2(o[2], o[3]);
          }
          // lower lanes take columns 0..7, upper lanes 8..15
          const auto a0 = __builtin_amdgcn_permlane32_swap(pk[0][0], pk[1][0], false, false);
          const auto a1 = __builtin_amdgcn_permlane32_swap(pk[0][1], pk[1][1], false, false);
          const int col = n0 + (GATED ? 16 * (WB * wn + b) : WR * (WB * wn + b) + 16 * h) + 8 * lhalf;
          if (r < rows && col < N) store_cols(out + r * p.ldo + col, u32x4{a0[0], a1[0], a0[1], a1[1]}, col, N);
        }
      }
    }
  };
  using std::integral_constant;
  using C1 = integral_constant<int, 1>;
  using C2 = integral_constant<int, 2>;
  using C3 = integral_constant<int, 3>;
  using C4 = integral_constant<int, 4>;
  using C5 = integral_constant<int, 5>;
  using K64 = integral_constant<int, 64>;
  using K128 = integral_constant<int, 128>;
  constexpr std::false_type whole{};
  constexpr std::true_type few{};
  if constexpr (KP == 1) {
    if (wide && wide_cols > FULL_COLS) body(C4{}, C2{}, C1{}, K64{}, C3{}, whole);
    else if (wide) body(C4{}, C1{}, C1{}, K64{}, C5{}, whole);
    else if (rows > 32) body(C2{}, C1{}, C1{}, K128{}, C3{}, whole);
    else body(C1{}, C1{}, C1{}, K128{}, C4{}, whole);
  } else if constexpr (CHUNK == kBriefChunk) {
    body(C1{}, C1{}, integral_constant<int, KP>{}, K128{}, integral_constant<int, HALF ? 6 : 4>{}, few);
  } else if constexpr (KP == 2) {
    if (rows > 32) body(C2{}, C1{}, C2{}, K128{}, C4{}, whole);
    else if (rows > 8) body(C1{}, C1{}, C2{}, K128{}, C5{}, whole);
    else body(C1{}, C1{}, C2{}, K128{}, C4{}, few);
  } else {
    if constexpr (CHUNK > 32) {
      if (rows > 32) return body(C2{}, C1{}, C4{}, K128{}, C3{}, whole);
    }
    if (rows > 8) body(C1{}, C1{}, C4{}, K128{}, integral_constant<int, HALF ? 4 : CHUNK == 32 ? 3 : 5>{}, whole);
    else body(C1{}, C1{}, C4{}, K128{}, integral_constant<int, HALF ? 6 : 4>{}, few);
  }
}

template <bool GATED, int KP, int CHUNK, bool HALF = false>
hipError_t launch_kp(long long blocks, const ItemsI8& ma, hipStream_t st) {
  constexpr int lds = item_lds(KP, CHUNK);
  static unsigned long long lds_set = 0;  // devices with the LDS limit raised
  const hipError_t e = set_max_dynamic_lds(reinterpret_cast<const void*>(&items_i8_kernel<GATED, KP, CHUNK, HALF>), lds, &lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((items_i8_kernel<GATED, KP, CHUNK, HALF>), dim3(static_cast<unsigned>(blocks)), dim3(kItemThreads), lds, st, ma);
  return hipGetLastError();
}

}  // namespace

// With the sums of few items (64 rows x 128 weight rows each, of an evenly
// routed batch) most CUs would idle, and an item runs through its whole K
// alone.  Time with K undivided, in 2 and in 4 parts, us (products of static
// rows): 64 items, 64 x 8192 x 4096 19.9, 14.8, 12.7; 112, 64 x 14336 x 4096
// 22.8, 17.2, 23.8; 189, 396 x 3391 x 12416 78, 55, 67; 256 of short K, 1000 x
// 2048 x 768 10.6, 12.8, 22.4; 392, 849 x 3534 x 4367 35, 52, 71.
//
// In 4 parts and still at most half a chip of workgroups, a wave takes 16 weight
// rows instead of 32: half of an MFMA's rows go unused, twice as many CUs read.
// Weights from HBM, us, 32 rows and 16: 1 x 2048 x 7168 9.9 and 8.2, 16 x 4096 x
// 14336 22.4 and 17.0, 128 x 1024 x 4096 8.8 and 7.4; with more workgroups than CUs
// (1 x 5120 x 4096) 8.7 and 9.1.
Cut items_cut(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  const int cols = gated ? kItemRows / 2 : kItemRows;
  // items of 128 weight rows and so many token rows
  auto count = [&](int rows) {
    auto chunks = [&](int n) { return std::max(1, ceil_div(n, rows)); };
    return (a.offsets ? static_cast<long long>(seg.hit_groups) * chunks(seg.mean_rows) : chunks(a.static_rows)) * ceil_div(a.N, cols) +
           (sh ? static_cast<long long>(chunks(sh->static_rows)) * ceil_div(sh->N, cols) : 0);
  };
  const long long items = count(kSplitChunk);
  Cut c{1, kChunk, false};
  if (items <= 64) c.parts = 4;
  else if (items <= 128 || (items <= 256 && a.K >= 4096)) c.parts = 2;
  if (c.parts > 1) c.rows = seg.max_rows <= kBriefChunk ? kBriefChunk : items <= 32 && seg.max_rows > 32 ? 32 : kSplitChunk;
  c.half = !gated && c.parts == 4 && count(32) <= kFewHalf;
  if (c.half && c.rows > 32) c.rows = 32;
  return c;
}

long long items_blocks(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  const Cut c = items_cut(seg, a, sh, gated);
  const int cols = (gated ? kItemRows / 2 : kItemRows) / c.parts / (c.half ? 2 : 1);
  // at most one partly filled chunk per group; wide items need fewer column blocks
  const long long chunks = a.offsets ? seg.total_rows / c.rows + std::min(seg.groups, seg.total_rows) : ceil_div(a.static_rows, c.rows);
  long long items = chunks * ceil_div(a.N, cols);
  if (sh) items += static_cast<long long>(ceil_div(sh->static_rows, c.rows)) * ceil_div(sh->N, cols);
  return items == 0 ? 0 : (items / kXcds + 3) * kXcds;  // each kind's run on an XCD rounds up by one
}

template <bool GATED>
static hipError_t launch_cut(const Cut& c, long long blocks, const ItemsI8& ma, hipStream_t st) {
  if (c.parts == 1) return launch_kp<GATED, 1, kChunk>(blocks, ma, st);
  if (c.parts == 2)
    return c.rows == kBriefChunk ? launch_kp<GATED, 2, kBriefChunk>(blocks, ma, st) : launch_kp<GATED, 2, kSplitChunk>(blocks, ma, st);
  if constexpr (!GATED)
    if (c.half) {
      return c.rows == kBriefChunk ? launch_kp<false, 4, kBriefChunk, true>(blocks, ma, st) : launch_kp<false, 4, 32, true>(blocks, ma, st);
    }
  if (c.rows == kBriefChunk) return launch_kp<GATED, 4, kBriefChunk>(blocks, ma, st);
  return c.rows == 32 ? launch_kp<GATED, 4, 32>(blocks, ma, st) : launch_kp<GATED, 4, kSplitChunk>(blocks, ma, st);
}

hipError_t launch_items_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  const long long blocks = items_blocks(seg, a, sh, gated);
  if (blocks == 0) return hipSuccess;
  ItemsI8 ma{a, sh ? *sh : GemmI8{}, seg.total_rows};
  if (!a.offsets) ma = ItemsI8{GemmI8{}, a, 0};  // a product of static rows alone
  const Cut c = items_cut(seg, a, sh, gated);
  return gated ? launch_cut<true>(c, blocks, ma, st) : launch_cut<false>(c, blocks, ma, st);
}

}  // namespace moe
