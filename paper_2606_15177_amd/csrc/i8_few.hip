// 8-bit products of a few rows per group whose rows are still bf16: each
// workgroup quantises the rows that it multiplies.  A decode step of up to 8
// tokens is bound by the latency of its launches and by reading the weights of
// the experts that it hits; this leaves out two of six launches (us, with the
// rows quantised by launches of their own and by the products: Qwen3 layer of 1
// token 32.7 and 26.0, of 4 55.9 and 45.0, of 8 82 and 65; DSV2-Lite of 1 37.0
// and 30.0; DSV3's 32 local experts of 1 106 and 82, of 4 200 and 169).
//
// A workgroup of four waves takes up to 8 rows of one group times 128 / KP
// weight rows, K in KP parts.  A wave streams its own 32 weight rows (gated: 16
// gate rows and the 16 up rows of the same columns) of its K part through a ring
// of three 128-byte stages of its own, so that no barrier is needed among the
// stages.  The first weights are on their way before the rows are read; those
// are quantised as moe_quantize_rows does, 256 threads along each row, and stay
// in LDS over the whole K, rows 32 bytes past a multiple of 256 apart, which
// spreads the 16 chunks that a fragment reads over the banks.  The MFMA's
// columns past the rows repeat the last one; no result is taken of them.
//
// Weights are read once, but where a group has more rows than expected, and leave
// the L2 first where a stage takes whole lines (Qwen3 of 8 tokens 71.8 us without
// the hint, 65.1 with it; 16 experts of 4104 x 3600, 1 token: 32 and 40).
//
// Two workgroups share a CU.  Rows that leave room for one only lose what the
// launches cost (8 rows of 7168: 250 us before, 257 here), as does a ring of
// four stages for the same reason (DSV2-Lite, 8 tokens: 89 us with three stages,
// 104 with four, 93 before): those are quantised by a launch.
#include <algorithm>
#include <type_traits>

#include "i8_impl.h"

namespace moe {
namespace {

constexpr int kThreads = 4 * kWave;
constexpr int kStage = 32 * 128;              // a wave's stage: 32 weight rows x 128 bytes
constexpr int kDepth = 3;
constexpr int kRing = 4 * kDepth * kStage;    // 48 KB
constexpr int kMaxLds = 80 * 1024;           // two workgroups per CU
constexpr int kVecs = 4;                      // vectors of a row per thread held in registers
constexpr int kLoads = 4;                     // per wave and stage, 8 rows each

struct FewI8 {
  GemmI8 g;   // groups with device offsets
  GemmI8 sp;  // static rows (static_rows 0: none)
  int rows;   // of g's result
  int chunk;  // rows of an item, up to kFewRows
};

__host__ __device__ constexpr int row_bytes(int K) { return (K + 255) / 256 * 256 + 32; }
// the waves' maxima, the rows' scales, and the rows behind the ring
constexpr int kHead = 4 * kFewRows * 4 + kFewRows * 4;

__device__ __forceinline__ int run_start(int n, int x) { return static_cast<int>(static_cast<long long>(n) * x / kXcds); }

template <bool GATED, int KP, bool ONCE>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void few_i8_kernel(FewI8 ma) {
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
  const GemmI8& p = shared ? ma.sp : ma.g;
  const int n_chunks = ceil_div(m, ma.chunk);
  const int nblk = __builtin_amdgcn_readfirstlane(item / n_chunks);
  const int m0 = __builtin_amdgcn_readfirstlane((item - nblk * n_chunks) * ma.chunk);
  const int rows = min(ma.chunk, m - m0);
  const int N = p.N, n0 = nblk * OUT_COLS, bytes = ceil_div(p.K, 16) * 16;
  const long long wrow = static_cast<long long>(g) * N;

  // ---- weights ----
  const int wn = wave % WN, wk = wave / WN;
  const uint32_t ldw = static_cast<uint32_t>(p.ldw);
  const __amdgpu_buffer_rsrc_t rs_w0 = rsrc(p.w0 + (wrow + n0) * p.ldw);
  const __amdgpu_buffer_rsrc_t rs_w1 = rsrc((GATED ? p.w1 : p.w0) + (wrow + n0) * p.ldw);
  const int nst = ceil_div(ceil_div(bytes, 128), KP);  // stages of a K part (the last part's may lie past K)
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
#pragma unroll 1
  for (int s = 0; s < kDepth; ++s) issue(s, s);

  // ---- rows ----
  const int stride = row_bytes(p.K);
  uint32_t* tops = reinterpret_cast<uint32_t*>(smem + kRing);
  float* scales = reinterpret_cast<float*>(tops + 4 * kFewRows);
  unsigned char* xl = smem + kRing + kHead;
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
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (i * kThreads < nvec) top = max_bits(top, v[r][i]);
    for (int i = tid + kVecs * kThreads; i < nvec; i += kThreads) top = max_bits(top, vec(r, i));
    const uint32_t t = wave_max(max(static_cast<uint32_t>(top[0]), static_cast<uint32_t>(top[1])));
    if (lane == 0) tops[r * 4 + wave] = t;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kFewRows; ++r) {
    if (r >= rows) break;
    const RowScale s = row_scale(max(max(tops[4 * r], tops[4 * r + 1]), max(tops[4 * r + 2], tops[4 * r + 3])));
    if (tid == 0) scales[r] = s.scale;
    auto put = [&](int i, u32x4 x) { *reinterpret_cast<u32x2*>(xl + r * stride + i * kVec) = quantize_vec(x, s); };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (tid + i * kThreads < nvec) put(tid + i * kThreads, v[r][i]);
    for (int i = tid + kVecs * kThreads; i < nvec; i += kThreads) put(i, vec(r, i));
  }
  const int lrow = lane & 31, lhalf = lane >> 5;
  // Scales of the wave's weight rows: lane l, weight row l % 32.
  const int wr = lane % 32;
  const int wcol = n0 + (GATED ? 16 * wn + (wr & 15) : 32 * wn + wr);
  const float cs = (GATED && (wr & 16) ? p.ws1 : p.ws0)[wrow + min(wcol, N - 1)];
  __syncthreads();
  const float rs = scales[min(lrow, rows - 1)];

  // ---- products ----
  // A stage past K (the last part's) reads zeros as weights; its row chunks are
  // clamped to the row.
  i32x16 acc = {};
  const unsigned char* xrow = xl + min(lrow, rows - 1) * stride;
  int slot = 0;
  for (int j = 0; j < nst; ++j) {
    // own loads of stage j landed; the first ones went out before the rows' own
    __builtin_amdgcn_s_waitcnt(wait_vm((kDepth - 1) * kLoads));
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    const unsigned char* wp = ring + slot * kStage;
    const int k0 = k_at(j);
    i32x4 wf[4], xf[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      wf[ks] = *reinterpret_cast<const i32x4*>(wp + lrow * 128 + (((2 * ks + lhalf) ^ ((lrow / 2) % 8)) << 4));
      xf[ks] = *reinterpret_cast<const i32x4*>(xrow + min(k0 + 32 * ks + 16 * lhalf, bytes - 16));
    }
    __builtin_amdgcn_s_waitcnt(kWaitLds);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    issue(j + kDepth, slot);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) acc = mfma_i8(wf[ks], xf[ks], acc);
    slot = slot == kDepth - 1 ? 0 : slot + 1;
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(0));  // the loads past the last stage: nothing may still write the LDS
  if constexpr (KP > 1) {
    int* red = reinterpret_cast<int*>(smem);
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
  float sc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i)
    sc[i] = __int_as_float(__builtin_amdgcn_ds_bpermute(16 * lhalf + 4 * (8 * (i / 4) + i % 4), __float_as_int(cs)));
  uint16_t* out = p.out + (row_base + m0 + lrow) * p.ldo;
#pragma unroll
  for (int h = 0; h < (GATED ? 1 : 2); ++h) {  // 16 columns each
    uint32_t pk[2][2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 8 * h + 4 * w + i;
        o[i] = static_cast<float>(acc[e]) * sc[e] * rs;
        if constexpr (GATED) o[i] = silu(o[i]) * (static_cast<float>(acc[8 + e]) * sc[8 + e] * rs);
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
hipError_t launch_few_kp(int blocks, int lds, const FewI8& ma, hipStream_t st) {
  static unsigned long long lds_set = 0;  // devices with the LDS limit raised
  const hipError_t e = set_max_dynamic_lds(reinterpret_cast<const void*>(&few_i8_kernel<GATED, KP, ONCE>), kMaxLds, &lds_set);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((few_i8_kernel<GATED, KP, ONCE>), dim3(blocks), dim3(kThreads), lds, st, ma);
  return hipGetLastError();
}

template <bool ONCE>
hipError_t launch_few_once(bool gated, int parts, int blocks, int lds, const FewI8& ma, hipStream_t st) {
  if (parts == 4) return gated ? launch_few_kp<true, 4, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 4, ONCE>(blocks, lds, ma, st);
  if (parts == 2) return gated ? launch_few_kp<true, 2, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 2, ONCE>(blocks, lds, ma, st);
  return gated ? launch_few_kp<true, 1, ONCE>(blocks, lds, ma, st) : launch_few_kp<false, 1, ONCE>(blocks, lds, ma, st);
}

// Rows of an item: no more than any group is expected to have.
int chunk_rows(const Segments& seg, const GemmI8* sh) {
  return std::min(std::max(seg.max_rows, sh ? sh->static_rows : 0), kFewRows);
}

int few_lds(const Segments& seg, const GemmI8& a, const GemmI8* sh) {
  return kRing + kHead + chunk_rows(seg, sh) * row_bytes(std::max(a.K, sh ? sh->K : 0));
}

// Items of 128 weight rows, however the rows are spread over the groups.
long long few_items(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  const int cols = gated ? 64 : 128, rows = chunk_rows(seg, sh);
  const long long chunks = seg.total_rows / rows + std::min(seg.groups, seg.total_rows);
  return chunks * ceil_div(a.N, cols) + (sh ? static_cast<long long>(ceil_div(sh->static_rows, rows)) * ceil_div(sh->N, cols) : 0);
}

}  // namespace

// The rows fit the LDS behind the ring, and the items the grid.
bool few_supported(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  return few_lds(seg, a, sh) <= kMaxLds && few_items(seg, a, sh, gated) < (1 << 20);
}

// K in parts where the items are few, and further on long K, whose items last
// (us of a layer with one part and two, gate/up: 288 items of K 7168 86.4 and
// 79.4, 344 of K 4096 75.6 and 73.6, 96 of K 2048 29.7 and 27.6, 384 of K 2048
// 43.2 and 46.5; with two and four, down: 64 of K 11008 65.5 and 60.8).
Cut few_cut(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated) {
  const int cols = gated ? 64 : 128;
  const long long hit = static_cast<long long>(seg.hit_groups) * ceil_div(a.N, cols) + (sh ? ceil_div(sh->N, cols) : 0);
  return {hit <= 64 ? 4 : hit <= 128 || (hit <= 512 && a.K >= 4096) ? 2 : 1, chunk_rows(seg, sh), false};
}

hipError_t launch_few_i8(const Segments& seg, const GemmI8& a, const GemmI8* sh, bool gated, hipStream_t st) {
  const Cut c = few_cut(seg, a, sh, gated);
  const int parts = c.parts;
  const int blocks = static_cast<int>((parts * few_items(seg, a, sh, gated) / kXcds + 1) * kXcds);
  const int lds = few_lds(seg, a, sh);
  const FewI8 ma{a, sh ? *sh : GemmI8{}, seg.total_rows, c.rows};
  const bool once = whole_lines(a.w0, a.ldw) && whole_lines(a.w1, 0) && (!sh || (whole_lines(sh->w0, sh->ldw) && whole_lines(sh->w1, 0)));
  return once ? launch_few_once<true>(gated, parts, blocks, lds, ma, st) : launch_few_once<false>(gated, parts, blocks, lds, ma, st);
}

}  // namespace moe
