// e4m3 products of a few rows per group whose rows are still bf16: each workgroup
// quantises the rows that it multiplies.  A decode step of up to 8 tokens is bound by
// the latency of its launches and by reading the weights of the experts that it hits;
// this leaves out the launches that quantise x and the hidden rows.
//
// A workgroup of four waves takes up to 8 rows of one group times 128 / KP weight
// rows, K in KP parts of whole blocks of 128 columns.  A wave streams its own 32 weight
// rows (gated: 16 gate rows and the 16 up rows of the same columns) of its K part
// through a ring of three 128-byte stages of its own, so that no barrier is needed
// among the stages.  The first weights are on their way before the rows are read;
// those are quantised as moe_quantize_rows_f8 does, 16 threads for each 128 columns,
// and stay in LDS over the whole K with their scales, rows 32 bytes past a multiple of
// 256 apart, which spreads what a fragment reads over the banks.  The MFMA's columns
// past the rows repeat the last one; no result is taken of them.
//
// Weights are read once, but where a group has more rows than expected, and leave
// the L2 first where a stage takes whole lines.
//
// Two workgroups share a CU.  Rows that leave room for one only are quantised by a
// launch.
//
// One token of a layer of 128 experts, H 2048, I 768, 8 of them hit: 29 us, where the
// quantisers' launches and the items took 32.
#include <algorithm>
#include <type_traits>

#include "f8_impl.h"

namespace moe {
namespace {

constexpr int kThreads = 4 * kWave;
constexpr int kStage = 32 * 128;              // a wave's stage: 32 weight rows x 128 bytes
constexpr int kDepth = 3;
constexpr int kRing = 4 * kDepth * kStage;    // 48 KB
constexpr int kMaxLds = 80 * 1024;           // two workgroups per CU
constexpr int kVecs = 4;                      // vectors of a row per thread held in registers
constexpr int kLoads = 4;                     // per wave and stage, 8 rows each

struct FewF8 {
  GemmF8 g;   // groups with device offsets
  GemmF8 sp;  // static rows (static_rows 0: none)
  int rows;   // of g's result
  int chunk;  // rows of an item, up to kFewRows
};

__host__ __device__ constexpr int row_bytes(int K) { return (K + 255) / 256 * 256 + 32; }
// the rows' scales, and the rows, behind the ring
__host__ __device__ constexpr int scale_bytes(int K) { return (K + kF8Block - 1) / kF8Block * 4; }

__device__ __forceinline__ int run_start(int n, int x) { return static_cast<int>(static_cast<long long>(n) * x / kXcds); }

template <bool GATED, int KP, bool ONCE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void few_f8_kernel(FewF8 ma) {
  constexpr int OUT_COLS = (GATED ? 64 : 128) / KP;  // output columns of an item
  constexpr int WN = 4 / KP;                         // waves along the weight rows
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);

  // ---- which item: chunks of 8 rows by column blocks, the shared rows first ----
  const int sp_chunks = ceil_div(ma.sp.static_rows, ma.chunk);
  const int n_shared = sp_chunks > 0 ? sp_chunks * ceil_div(ma.sp.N, OUT_COLS) : 0;
  const int blocks = ceil_div(ma.g.N, OUT_COLS);
  auto group_rows = [&](int g, int& first) {  // lane: rows of group g
    first = row_at(ma.g.offsets, min(g, ma.g.groups), ma.rows);
    return max(row_at(ma.g.offsets, min(g + 1, ma.g.groups), ma.rows) - first, 0);
  };
  // chunks of the lane's group and of those before it in its batch of 64
  auto scan = [&](int n, int& own) {
    own = ceil_div(n, ma.chunk);
    int inc = own;
    if (__ballot(own > 1) != 0) {
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
    return inc;
  };
  int chunks = 0;
  for (int g0 = 0; g0 < ma.g.groups; g0 += kWave) {
    int first, own;
    const int inc = scan(group_rows(g0 + lane, first), own);
    chunks += __builtin_amdgcn_readlane(inc, kWave - 1);
  }
  const int total = n_shared + chunks * blocks;
  const int xcd = static_cast<int>(blockIdx.x) % kXcds, in_xcd = static_cast<int>(blockIdx.x) / kXcds;
  const int id = run_start(total, xcd) + in_xcd;
  if (id >= run_start(total, xcd + 1)) return;
  const bool shared = id < n_shared;
  int g = 0, row_base = 0, m = ma.sp.static_rows, item = id;
  if (!shared) {
    const int at = (id - n_shared) / blocks;  // chunk, of all groups
    int before = 0;
    bool found = false;
    for (int g0 = 0; !found && g0 < ma.g.groups; g0 += kWave) {
      int first, own;
      const int n = group_rows(g0 + lane, first);
      const int inc = scan(n, own);
      const uint64_t past = __ballot(before + inc > at);
      if (past) {
        const int l = __ffsll(static_cast<long long>(past)) - 1;
        g = g0 + l;
        row_base = __builtin_amdgcn_readlane(first, l);
        m = __builtin_amdgcn_readlane(n, l);
        item = id - n_shared - (before + __builtin_amdgcn_readlane(inc - own, l)) * blocks;
        found = true;
      }
      before += __builtin_amdgcn_readlane(inc, kWave - 1);
    }
    if (!found) return;  // not reached: the chunk lies within the groups' chunks
  }
  g = __builtin_amdgcn_readfirstlane(g);
  row_base = __builtin_amdgcn_readfirstlane(row_base);
  m = __builtin_amdgcn_readfirstlane(m);
  const GemmF8& p = shared ? ma.sp : ma.g;
  const int n_chunks = ceil_div(m, ma.chunk);
  const int nblk = __builtin_amdgcn_readfirstlane(item / n_chunks);
  const int m0 = __builtin_amdgcn_readfirstlane((item - nblk * n_chunks) * ma.chunk);
  const int rows = min(ma.chunk, m - m0);
  const int N = p.N, n0 = nblk * OUT_COLS, bytes = ceil_div(p.K, 16) * 16;
  const int kb_all = ceil_div(p.K, kF8Block);  // blocks of 128 columns
  const long long wrow = static_cast<long long>(g) * N;

  // ---- weights ----
  const int wn = wave % WN, wk = wave / WN;
  const uint32_t ldw = static_cast<uint32_t>(p.ldw);
  const __amdgpu_buffer_rsrc_t rs_w0 = rsrc(p.w0 + (wrow + n0) * p.ldw);
  const __amdgpu_buffer_rsrc_t rs_w1 = rsrc((GATED ? p.w1 : p.w0) + (wrow + n0) * p.ldw);
  const int nst = ceil_div(kb_all, KP);  // stages of a K part (the last part's may lie past K)
  const int rot = static_cast<int>((static_cast<unsigned>(nblk) * 7u + static_cast<unsigned>(g) * 3u) % static_cast<unsigned>(nst));
  uint32_t woff[kLoads];
  int piece[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = 8 * i + lane / 8;
    const int col = GATED ? 16 * wn + (r & 15) : 32 * wn + r;
    woff[i] = n0 + col < N ? static_cast<uint32_t>(col) * ldw : kPastEnd;
    piece[i] = (lane % 8) ^ ((r / 2) % 8);
  }
  auto k_at = [&](int s) { return (wk * nst + (rot + s < nst ? rot + s : rot + s - nst)) * 128; };
  unsigned char* ring = smem + wave * (kDepth * kStage);
  auto issue = [&](int s, int slot) {
    const int k0 = k_at(s);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int k = k0 + piece[i] * 16;
      const uint32_t kill = (s < nst && k < bytes ? 0u : kPastEnd) | (woff[i] & kPastEnd);
      const uint32_t at = (woff[i] + static_cast<uint32_t>(k)) | kill;
      if constexpr (ONCE) load_lds16_once(GATED && i >= kLoads / 2 ? rs_w1 : rs_w0, ring + slot * kStage + i * 1024, at);
      else load_lds16(GATED && i >= kLoads / 2 ? rs_w1 : rs_w0, ring + slot * kStage + i * 1024, at);
    }
  };
  // Scales of the matrix blocks: lane l holds those of stages l, l + 64, ... (of a
  // stage past K none).
  const int block0 = min(n0 + (GATED ? 16 * wn : 32 * wn), N - 1) / kF8Block;
  float ws0, ws1;
  auto read_scales = [&](int s0) {
    const int kb = k_at(min(s0 + lane, nst - 1)) / kF8Block;
    const long long at = (static_cast<long long>(g) * ceil_div(N, kF8Block) + block0) * kb_all + min(kb, kb_all - 1);
    ws0 = kb < kb_all ? p.ws0[at] : 0.0f;
    ws1 = GATED && kb < kb_all ? p.ws1[at] : 0.0f;
  };
  read_scales(0);
#pragma unroll 1
  for (int s = 0; s < kDepth; ++s) issue(s, s);

  // ---- rows ----
  const int stride = row_bytes(p.K);
  float* scales = reinterpret_cast<float*>(smem + kRing);  // [row][block]
  unsigned char* xl = smem + kRing + kFewRows * scale_bytes(p.K);
  const int nvec = bytes / kVec, tid = static_cast<int>(threadIdx.x);
  const uint16_t* src[kFewRows];
  u32x4 v[kFewRows][kVecs];
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    src[r] = nullptr;
    if (r >= rows) continue;
    int at = row_base + m0 + r;
    if (p.x_rows) at = load_scalar(p.x_rows, at);
    const bool in = !p.x_rows || static_cast<unsigned>(at) < static_cast<unsigned>(p.x_count);
    if (in) src[r] = p.xb + static_cast<long long>(at) * p.ldxb;
  }
  auto vec = [&](int r, int i) { return src[r] && i < nvec ? load_vec(src[r], i, p.K) : u32x4{0u, 0u, 0u, 0u}; };
#pragma unroll
  for (int r = 0; r < kFewRows; ++r)
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (r < rows && i * kThreads < nvec) v[r][i] = vec(r, tid + i * kThreads);
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    if (r >= rows) break;
    auto put = [&](int i, u32x4 x) {
      const F8Scale s = f8_scale(group_max(max_bits_f32(x)));
      if (i >= nvec) return;
      if (i % kF8Lanes == 0) scales[r * kb_all + i / kF8Lanes] = s.scale;
      *reinterpret_cast<u32x2*>(xl + r * stride + i * kVec) = quantize_f8_vec(x, s);
    };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (i * kThreads < nvec) put(tid + i * kThreads, v[r][i]);
    for (int i0 = kVecs * kThreads; i0 < nvec; i0 += kThreads) put(tid + i0, vec(r, tid + i0));
  }
  const int lrow = lane & 31, lhalf = lane >> 5;
  asm volatile("" : "+v"(ws0), "+v"(ws1));  // (waited for here, not in the loop)
  __syncthreads();

  // ---- products ----
  // A stage past K (the last part's) reads zeros as weights, and no scale; its row
  // chunks and scales are clamped to the row.
  f32x16 acc = {};
  const unsigned char* xrow = xl + min(lrow, rows - 1) * stride;
  const float* xscale = scales + min(lrow, rows - 1) * kb_all;
  int slot = 0;
  for (int j = 0; j < nst; ++j) {
    // own loads of stage j landed; the first ones went out before the rows' own
    __builtin_amdgcn_s_waitcnt(wait_vm((kDepth - 1) * kLoads));
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    const unsigned char* wp = ring + slot * kStage;
    const int k0 = k_at(j);
    i32x8 wf[2], xf[2];
    auto read16 = [](i32x8& to, int c, const unsigned char* from) {
      const i32x4 q = *reinterpret_cast<const i32x4*>(from);
#pragma unroll
      for (int i = 0; i < 4; ++i) to[4 * c + i] = q[i];
    };
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int chunk = 4 * ks + 2 * lhalf + c;
        read16(wf[ks], c, wp + lrow * 128 + ((chunk ^ ((lrow / 2) % 8)) << 4));
        read16(xf[ks], c, xrow + min(k0 + 16 * chunk, bytes - 16));
      }
    const float xs = xscale[min(k0 / kF8Block, kb_all - 1)];
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    issue(j + kDepth, slot);
    if ((j & 63) == 0 && j > 0) {
      read_scales(j);
      asm volatile("" : "+v"(ws0), "+v"(ws1));  // (waited for here)
    }
    const float f0 = xs * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ws0), j & 63));
    const float f1 = GATED ? xs * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ws1), j & 63)) : f0;
    f32x16 part = {};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) part = mfma_f8(wf[ks], xf[ks], part);
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = fmaf(part[i], i < 8 ? f0 : f1, acc[i]);
    slot = slot == kDepth - 1 ? 0 : slot + 1;
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(0));  // the loads past the last stage: nothing may still write the LDS
  if constexpr (KP > 1) {
    float* red = reinterpret_cast<float*>(smem);
    __syncthreads();  // every wave is past its last stage
    if (wk > 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) red[((wk - 1) * WN + wn) * (16 * kWave) + i * kWave + lane] = acc[i];
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int q = 0; q < KP - 1; ++q)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] += red[(q * WN + wn) * (16 * kWave) + i * kWave + lane];
  }
  // ---- results: lane holds C[n = 8 v4 + 4 lhalf + i][t = lrow] ----
  uint16_t* out = p.out + static_cast<long long>(row_base + m0 + lrow) * p.ldo;
#pragma unroll
  for (int h = 0; h < (GATED ? 1 : 2); ++h) {  // 16 columns each
    uint32_t pk[2][2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 8 * h + 4 * w + i;
        o[i] = acc[e];
        if constexpr (GATED) o[i] = silu(o[i]) * acc[8 + e];
      }
      pk[w][0] = pack_bf16x2(o[0], o[1]);
      pk[w][1] = pack_bf16x2(o[2], o[3]);
    }
    // lower lanes take columns 0..7, upper lanes 8..15
    const auto a0 = __builtin_amdgcn_permlane32_swap(pk[0][0], pk[1][0], false, false);
    const auto a1 = __builtin_amdgcn_permlane32_swap(pk[0][1], pk[1][1], false, false);
    const int col = n0 + (GATED ? 16 * wn : 32 * wn + 16 * h) + 8 * lhalf;
    if (lrow < rows && col < N) store_cols(out + col, u32x4{a0[0], a1[0], a0[1], a1[1]}, col, N);
  }
}

template <bool GATED, int KP, bool ONCE>
hipError_t launch_few_kp(int blocks, int lds, const FewF8& ma, hipStream_t st) {
  static unsigned long long lds_set = 0;  // devices with the LDS limit raised
  const hipError_t e = set_max_dynamic_lds(reinterpret_cast<const void*>(&few_f8_kernel<GATED, KP, ONCE>), kMaxLds, &lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((few_f8_kernel<GATED, KP, ONCE>), dim3(blocks), dim3(kThreads), lds, st, ma);
  return hipGetLastError();
}

template <bool ONCE>
hipError_t launch_few_once(bool gated, int parts, int blocks, int lds, const FewF8& ma, hipStream_t st) {
  if (parts == 4) return gated ? launch_few_kp<true, 4, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 4, ONCE>(blocks, lds, ma, st);
  if (parts == 2) return gated ? launch_few_kp<true, 2, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 2, ONCE>(blocks, lds, ma, st);
  return gated ? launch_few_kp<true, 1, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 1, ONCE>(blocks, lds, ma, st);
}

// Rows of an item: no more than any group is expected to have.
int chunk_rows(const Segments& seg, const GemmF8* sh) {
  return std::min(std::max(seg.max_rows, sh ? sh->static_rows : 0), kFewRows);
}

int few_lds(const Segments& seg, const GemmF8& a, const GemmF8* sh) {
  const int K = std::max(a.K, sh ? sh->K : 0);
  return kRing + kFewRows * scale_bytes(K) + chunk_rows(seg, sh) * row_bytes(K);
}

// Items of 128 weight rows, however the rows are spread over the groups.
long long few_items(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  const int cols = gated ? 64 : 128, rows = chunk_rows(seg, sh);
  const long long chunks = seg.total_rows / rows + std::min(seg.groups, seg.total_rows);
  return chunks * ceil_div(a.N, cols) + (sh ? static_cast<long long>(ceil_div(sh->static_rows, rows)) * ceil_div(sh->N, cols) : 0);
}

}  // namespace

// The rows fit the LDS behind the ring, and the items the grid.
bool few_f8_supported(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  return few_lds(seg, a, sh) <= kMaxLds && few_items(seg, a, sh, gated) < (1 << 20);
}

// K in parts where the items (128 weight rows of a group that has rows) are few.
// Weights from HBM, K undivided, in 2 and in 4 parts, us:
//   32 items: gated K 7168 24.7, 15.9, 11.9; K 1024 8.1, 7.0, 6.5; 64: K 14336 45, 29, 24;
//   96: gated K 2048 11.2, 9.0, 9.2; K 1408 9.2, 7.9, 8.7; 112: K 2048 11.0, 9.3, 9.2;
//   128: K 768 8.1, 7.5, 8.2; K 5000 29, 20, 19; gated K 7168 26.1, 20.5, 20.4;
//   168: K 2048 11.6, 12.2, 15.2; 192: gated K 4096 20.9, 20.8, 24.0; 256: K 768 8.8, 9.8,
//     14.5; 448: gated K 4096 36.5, 38.6, 43.9.
Cut few_f8_cut(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated) {
  const int cols = gated ? 64 : 128;
  const long long hit = static_cast<long long>(seg.hit_groups) * ceil_div(a.N, cols) + (sh ? ceil_div(sh->N, cols) : 0);
  return {hit <= 64 ? 4 : hit <= 128 ? 2 : 1, chunk_rows(seg, sh), false};
}

hipError_t launch_few_f8(const Segments& seg, const GemmF8& a, const GemmF8* sh, bool gated, hipStream_t st) {
  const Cut c = few_f8_cut(seg, a, sh, gated);
  const int parts = c.parts;
  const int blocks = static_cast<int>((parts * few_items(seg, a, sh, gated) / kXcds + 1) * kXcds);
  const int lds = few_lds(seg, a, sh);
  const FewF8 ma{a, sh ? *sh : GemmF8{}, seg.total_rows, c.rows};
  auto lines = [](const uint8_t* w) { return reinterpret_cast<const int8_t*>(w); };
  const bool once = whole_lines(lines(a.w0), a.ldw) && whole_lines(lines(a.w1), 0) && (!sh || (whole_lines(lines(sh->w0), sh->ldw) && whole_lines(lines(sh->w1), 0)));
  return once ? launch_few_once<true>(gated, parts, blocks, lds, ma, st) : launch_few_once<false>(gated, parts, blocks, lds, ma, st);
}

}  // namespace moe
