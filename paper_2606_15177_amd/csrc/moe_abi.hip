// The C ABI (include/moe.h): host-side validation, workspace carving and the
// launch sequence of each entry point.  No allocation, no synchronisation,
// no device-to-host traffic: every data-dependent size stays on the device.
#include "moe.h"

#include <algorithm>
#include <cmath>

#include "kernels.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kIntMax = 2147483647;

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_dims(const moe_dims* d) {
  if (d == nullptr) return MOE_ERR_NULL;
  if (d->T < 0 || d->H < 1 || d->E < 1 || d->k < 1 || d->k > d->E || d->I < 1 || d->S < 1 ||
      d->E_local < 1 || d->E_local > d->E || d->n_shared < 0 ||
      (d->n_shared > 0 && d->I_shared < 1))
    return MOE_ERR_DIMS;
  if (d->flags < MOE_GATE_SOFTMAX_TOPK || d->flags > MOE_GATE_SIGMOID) return MOE_ERR_UNSUPPORTED;
  if (d->E > moe::kMaxExperts || d->k > 32) return MOE_ERR_UNSUPPORTED;
  if (d->H % 8 != 0 || d->I % 8 != 0 || (d->n_shared > 0 && d->I_shared % 8 != 0))
    return MOE_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->T) * d->k > kIntMax || static_cast<int64_t>(d->S) * d->E > kIntMax ||
      static_cast<int64_t>(d->n_shared) * std::max(d->I_shared, 0) > kIntMax)
    return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

// The router's gating variant: dims->flags picks the gate function, g (may be
// null) carries its parameters.
int gating_ok(const moe_dims* d, const moe_gating* g, moe::RouteGating* out) {
  *out = moe::RouteGating{d->flags, nullptr, 1.0f, 0, 0};
  if (g == nullptr) return MOE_OK;
  if (g->bias && d->flags != MOE_GATE_SIGMOID) return MOE_ERR_DIMS;
  if (g->bias && (reinterpret_cast<uintptr_t>(g->bias) & 3u) != 0) return MOE_ERR_ALIGN;
  if (g->n_group > 1) {
    if (g->n_group > 64) return MOE_ERR_UNSUPPORTED;
    if (d->E % g->n_group != 0 || g->topk_group < 1 || g->topk_group > g->n_group ||
        d->k > g->topk_group * (d->E / g->n_group))
      return MOE_ERR_DIMS;
  } else if (g->n_group < 0) {
    return MOE_ERR_DIMS;
  }
  *out = moe::RouteGating{d->flags, g->bias, g->routed_scale, g->n_group, g->topk_group};
  return MOE_OK;
}

int64_t sh_width(const moe_dims* d) {
  return d->n_shared > 0 ? static_cast<int64_t>(d->n_shared) * d->I_shared : 0;
}

// Rows that the workspace holds for h.  Decode-sized batches reserve every
// expert's rows in whole chunks of 32: more than they fill now, but the size
// decides what moe_forward_noalloc accepts, which stays as it was.
size_t h_rows(const moe_dims* d) {
  const size_t rows = static_cast<size_t>(d->T) * d->k;
  const moe::Segments routed{nullptr, d->E_local, 0, d->T, d->T * d->k, 0, 0};
  if (d->T == 0 || !moe::ffn_streams_weights(routed) || d->H % 16 != 0 || d->I % 16 != 0) return rows;
  return (rows / 32 + std::min<size_t>(d->E_local, rows)) * 32;
}

// Workspace of the expert FFN: h, then h_shared.
struct FfnWs {
  uint16_t* h;
  uint16_t* h_sh;
  size_t bytes;
};
FfnWs carve_ffn(const moe_dims* d, void* base) {
  FfnWs w{};
  unsigned char* p = static_cast<unsigned char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* r = p ? p + off : nullptr;
    off += align_up(bytes);
    return r;
  };
  w.h = reinterpret_cast<uint16_t*>(take(h_rows(d) * d->I * sizeof(uint16_t)));
  w.h_sh = reinterpret_cast<uint16_t*>(take(static_cast<size_t>(d->T) * sh_width(d) * sizeof(uint16_t)));
  w.bytes = off;
  return w;
}
size_t ffn_ws(const moe_dims* d) { return carve_ffn(d, nullptr).bytes; }

// The forward workspace, carved in this order.  The experts' outputs wait for the
// weighted sum in bf16, as moe_expert_ffn and moe_expert_ffn_i8 return them, so
// that the layer's bits are its steps'.  On int8 experts the layer is 0.20 to
// 0.23 % off the exact sum (norms) where one rounding at the end leaves 0.17 %;
// in fp32 they would cost 4 more bytes per value, 0.2 to 0.3 ms by bytes of the
// 1.6 to 2.3 ms that 16384 tokens of DSV3's 32 local experts take.
struct ForwardWs {
  int32_t* topk_idx;
  float* topk_w;
  int32_t* offsets;
  int32_t* perm_token;
  int32_t* inv_pos;
  uint16_t* y_perm;
  uint16_t* y_shared;
  void* permute_ws;
  void* ffn_ws;
  size_t bytes;
};

ForwardWs carve_forward(const moe_dims* d, size_t ffn_bytes, void* base) {
  ForwardWs w{};
  unsigned char* p = static_cast<unsigned char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* r = p ? p + off : nullptr;
    off += align_up(bytes);
    return r;
  };
  const size_t rows = static_cast<size_t>(d->T) * d->k;
  w.topk_idx = reinterpret_cast<int32_t*>(take(rows * sizeof(int32_t)));
  w.topk_w = reinterpret_cast<float*>(take(rows * sizeof(float)));
  w.offsets = reinterpret_cast<int32_t*>(take((d->E_local + 1) * sizeof(int32_t)));
  w.perm_token = reinterpret_cast<int32_t*>(take(rows * sizeof(int32_t)));
  w.inv_pos = reinterpret_cast<int32_t*>(take(rows * sizeof(int32_t)));
  w.y_perm = reinterpret_cast<uint16_t*>(take(rows * d->H * sizeof(uint16_t)));
  w.y_shared = reinterpret_cast<uint16_t*>(
      take(d->n_shared > 0 ? static_cast<size_t>(d->T) * d->H * sizeof(uint16_t) : 0));
  w.permute_ws = take(moe::permute_ws_bytes(d->T, d->k, d->E_local, d->S, d->E));
  w.ffn_ws = take(ffn_bytes);
  w.bytes = off;
  return w;
}

size_t ffn_i8_ws(const moe_dims* d, bool one_x);
size_t ffn_f8_ws(const moe_dims* d, bool one_x);

size_t entry_ws(const moe_dims* d, int entry) {
  switch (entry) {
    case MOE_ENTRY_PERMUTE:
      return align_up(moe::permute_ws_bytes(d->T, d->k, d->E_local));
    case MOE_ENTRY_EXPERT_FFN:
      return ffn_ws(d);
    case MOE_ENTRY_FORWARD:
      return carve_forward(d, ffn_ws(d), nullptr).bytes;
    case MOE_ENTRY_EXPERT_FFN_I8:
      return ffn_i8_ws(d, false);
    case MOE_ENTRY_FORWARD_I8:
      return carve_forward(d, ffn_i8_ws(d, true), nullptr).bytes;
    case MOE_ENTRY_EXPERT_FFN_F8:
      return ffn_f8_ws(d, false);
    case MOE_ENTRY_FORWARD_F8:
      return carve_forward(d, ffn_f8_ws(d, true), nullptr).bytes;
    default:
      return 0;
  }
}

int check_ws(const moe_dims* d, int entry, const void* ws, size_t ws_bytes) {
  const size_t need = entry_ws(d, entry);
  if (ws_bytes < need) return MOE_ERR_WORKSPACE;
  if (need > 0 && ws == nullptr) return MOE_ERR_WORKSPACE;
  if (ws != nullptr && (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0) return MOE_ERR_ALIGN;
  return MOE_OK;
}

int status(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_ERR_DEVICE; }

void record(const moe_taps* taps, int slot, hipStream_t st) {
  if (taps && taps->events[slot]) (void)hipEventRecord(static_cast<hipEvent_t>(taps->events[slot]), st);
}

int weights_ok(const moe_dims* d, const moe_weights* w) {
  if (w == nullptr || w->w_gate == nullptr || w->w_up == nullptr || w->w_down == nullptr)
    return MOE_ERR_NULL;
  if (d->n_shared > 0 && (w->sh_gate == nullptr || w->sh_up == nullptr || w->sh_down == nullptr))
    return MOE_ERR_NULL;
  if (!aligned16(w->w_gate) || !aligned16(w->w_up) || !aligned16(w->w_down)) return MOE_ERR_ALIGN;
  if (d->n_shared > 0 && (!aligned16(w->sh_gate) || !aligned16(w->sh_up) || !aligned16(w->sh_down)))
    return MOE_ERR_ALIGN;
  return MOE_OK;
}

// The routed rows; rows per expert and experts hit as if routing were even.
moe::Segments routed_segments(const moe_dims* d, const int32_t* offsets) {
  const int mean = static_cast<int>(static_cast<int64_t>(d->T) * d->k / d->E);
  const int hit = static_cast<int>(std::ceil(d->E_local * (1.0 - std::pow(1.0 - static_cast<double>(d->k) / d->E, d->T))));
  return moe::Segments{offsets, d->E_local, 0, d->T, d->T * d->k, mean, hit};
}

// The two grouped GEMMs of the experts (routed, then shared): their row
// segments and arguments, built the same way for the host-side limit check
// (null pointers; rows_indexed says whether the gate/up GEMM reads its rows
// through a row list of T entries) and for the launches.
struct FfnPlan {
  moe::Segments routed, shared;
  moe::UpArgs up, sh_up;
  moe::DownArgs dn, sh_dn;
};
FfnPlan plan_ffn(const moe_dims* d, const uint16_t* x_perm, const int32_t* x_rows, bool rows_indexed,
                 const int32_t* offsets, const moe_weights* w, const uint16_t* x, uint16_t* y_perm,
                 uint16_t* y_shared, void* ws) {
  const FfnWs fw = carve_ffn(d, ws);
  const int shw = static_cast<int>(sh_width(d));
  FfnPlan p{};
  p.routed = routed_segments(d, offsets);
  p.shared = moe::Segments{nullptr, 1, d->T, d->T, d->T, d->T, 1};
  p.up = moe::UpArgs{x_perm, w ? w->w_gate : nullptr, w ? w->w_up : nullptr, fw.h, d->H, d->I, x_rows,
                     rows_indexed ? d->T : 0};
  p.sh_up = moe::UpArgs{x, w ? w->sh_gate : nullptr, w ? w->sh_up : nullptr, fw.h_sh, d->H, shw, nullptr, 0};
  p.dn = moe::DownArgs{fw.h, w ? w->w_down : nullptr, y_perm, d->I, d->H, d->I, d->I, 0,
                       static_cast<size_t>(d->H) * d->I};
  p.sh_dn = moe::DownArgs{fw.h_sh, w ? w->sh_down : nullptr, y_shared, shw, d->H, d->I_shared, d->I_shared,
                          static_cast<size_t>(d->H) * d->I_shared, 0};
  return p;
}

// Kernel limits of the expert GEMMs for these sizes (MOE_ERR_UNSUPPORTED
// beyond them), decided before anything is enqueued: the same predicates the
// launchers apply, on the same arguments.
int check_ffn_limits(const moe_dims* d, bool rows_indexed) {
  if (d->T == 0) return MOE_OK;
  const FfnPlan p = plan_ffn(d, nullptr, nullptr, rows_indexed, nullptr, nullptr, nullptr, nullptr, nullptr,
                             nullptr);
  if (!moe::ffn_up_supported(p.routed, p.up) || !moe::ffn_down_supported(p.routed, p.dn))
    return MOE_ERR_UNSUPPORTED;
  if (d->n_shared > 0 &&
      (!moe::ffn_up_supported(p.shared, p.sh_up) || !moe::ffn_down_supported(p.shared, p.sh_dn)))
    return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

int check_ffn_i8_limits(const moe_dims* d, bool one_x);
int check_ffn_f8_limits(const moe_dims* d, bool one_x);

// The limits of one entry point (0: of every bf16 entry point).
int check_entry(const moe_dims* d, int entry) {
  int s = MOE_OK;
  if (entry == 0 || entry == MOE_ENTRY_EXPERT_FFN) s = check_ffn_limits(d, false);
  if (s == MOE_OK && (entry == 0 || entry == MOE_ENTRY_FORWARD)) s = check_ffn_limits(d, true);
  if (entry == MOE_ENTRY_EXPERT_FFN_I8 || entry == MOE_ENTRY_FORWARD_I8)
    s = check_ffn_i8_limits(d, entry == MOE_ENTRY_FORWARD_I8);
  if (entry == MOE_ENTRY_EXPERT_FFN_F8 || entry == MOE_ENTRY_FORWARD_F8)
    s = check_ffn_f8_limits(d, entry == MOE_ENTRY_FORWARD_F8);
  return s;
}

int run_ffn(const moe_dims* d, const uint16_t* x_perm, const int32_t* x_rows, const int32_t* offsets,
            const moe_weights* w, const uint16_t* x, uint16_t* y_perm, uint16_t* y_shared,
            void* ws, const moe_taps* taps, hipStream_t st) {
  const FfnPlan p = plan_ffn(d, x_perm, x_rows, x_rows != nullptr, offsets, w, x, y_perm, y_shared, ws);
  hipError_t e;

  // routed and shared experts: in one launch per GEMM or one each (plan_gemm2)
  record(taps, 2 * MOE_STAGE_FFN_UP, st);
  if (d->n_shared > 0)
    e = moe::launch_ffn_up2(p.routed, p.up, p.shared, p.sh_up, st);
  else
    e = moe::launch_ffn_up(p.routed, p.up, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_UP + 1, st);

  record(taps, 2 * MOE_STAGE_FFN_DOWN, st);
  if (d->n_shared > 0)
    e = moe::launch_ffn_down2(p.routed, p.dn, p.shared, p.sh_dn, st);
  else
    e = moe::launch_ffn_down(p.routed, p.dn, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_DOWN + 1, st);
  return MOE_OK;
}

// ---- the same on int8 experts ----

int64_t pad16(int64_t n) { return (n + 15) / 16 * 16; }
constexpr int64_t kMaxI8K = (1 << 17) - 1;  // inner dimension: sums of int8 products stay within int32
constexpr int64_t kMaxI8Stride = 1 << 21;   // 512 rows of a tile stay within 32-bit offsets
constexpr int64_t kSpan = kIntMax;          // gathered rows: 32-bit offsets
constexpr int64_t kMaxI8Rows = kIntMax - 255;  // a last tile or chunk, up to 256 rows, ends within int32

// Workspace of the int8 expert FFN: quantised inputs (x_rows_cap rows for the
// routed experts, T for the shared ones unless they read the same rows),
// hidden rows in bf16, and those quantised.
struct FfnI8Ws {
  int8_t *xq, *xq_sh, *hq, *hq_sh;
  float *xs, *xs_sh, *hs, *hs_sh;
  uint16_t *h, *h_sh;
  size_t bytes;
};
FfnI8Ws carve_ffn_i8(const moe_dims* d, bool one_x, void* base) {
  FfnI8Ws w{};
  unsigned char* p = static_cast<unsigned char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* r = p ? p + off : nullptr;
    off += align_up(bytes);
    return r;
  };
  const size_t T = d->T, rows = T * d->k, hp = pad16(d->H), ip = pad16(d->I), shw = sh_width(d), wp = pad16(shw);
  const size_t x_rows = one_x ? T : rows, sh_x = one_x || shw == 0 ? 0 : T, sh_h = shw == 0 ? 0 : T;
  w.xq = reinterpret_cast<int8_t*>(take(x_rows * hp));
  w.xs = reinterpret_cast<float*>(take(x_rows * sizeof(float)));
  w.xq_sh = reinterpret_cast<int8_t*>(take(sh_x * hp));
  w.xs_sh = reinterpret_cast<float*>(take(sh_x * sizeof(float)));
  w.h = reinterpret_cast<uint16_t*>(take(rows * d->I * sizeof(uint16_t)));
  w.hq = reinterpret_cast<int8_t*>(take(rows * ip));
  w.hs = reinterpret_cast<float*>(take(rows * sizeof(float)));
  w.h_sh = reinterpret_cast<uint16_t*>(take(sh_h * shw * sizeof(uint16_t)));
  w.hq_sh = reinterpret_cast<int8_t*>(take(sh_h * wp));
  w.hs_sh = reinterpret_cast<float*>(take(sh_h * sizeof(float)));
  if (one_x) {
    w.xq_sh = w.xq;
    w.xs_sh = w.xs;
  }
  w.bytes = off;
  return w;
}

size_t ffn_i8_ws(const moe_dims* d, bool one_x) { return carve_ffn_i8(d, one_x, nullptr).bytes; }

// The experts' products, built the same way for the limit check (null
// pointers) and for the launches.
struct FfnI8Plan {
  moe::Segments routed;
  moe::GemmI8 up, sh_up, dn, sh_dn;
  bool sh;
};
FfnI8Plan plan_ffn_i8(const moe_dims* d, const FfnI8Ws& fw, const int32_t* x_rows, const int32_t* offsets,
                      const moe_weights_i8& w, uint16_t* y_perm, uint16_t* y_shared) {
  const int shw = static_cast<int>(sh_width(d));
  const long long hp = pad16(d->H), ip = pad16(d->I), wp = pad16(shw);
  FfnI8Plan p{};
  p.routed = routed_segments(d, offsets);
  p.up = moe::GemmI8{fw.xq, fw.xs, x_rows, x_rows ? d->T : 0, offsets, 0, d->E_local, w.w_gate, w.w_up, w.s_gate, w.s_up,
                     fw.h, d->H, d->I, hp, hp, d->I};
  p.sh_up = moe::GemmI8{fw.xq_sh, fw.xs_sh, nullptr, 0, nullptr, d->T, 1, w.sh_gate, w.sh_up, w.sh_s_gate, w.sh_s_up,
                        fw.h_sh, d->H, shw, hp, hp, shw};
  p.dn = moe::GemmI8{fw.hq, fw.hs, nullptr, 0, offsets, 0, d->E_local, w.w_down, nullptr, w.s_down, nullptr,
                     y_perm, d->I, d->H, ip, ip, d->H};
  p.sh_dn = moe::GemmI8{fw.hq_sh, fw.hs_sh, nullptr, 0, nullptr, d->T, 1, w.sh_down, nullptr, w.sh_s_down, nullptr,
                        y_shared, shw, d->H, wp, wp, d->H};
  p.sh = d->n_shared > 0;
  return p;
}

int check_ffn_i8_limits(const moe_dims* d, bool one_x) {
  if (d->H > kMaxI8K || d->I > kMaxI8K || sh_width(d) > kMaxI8K) return MOE_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->T) * d->k > kMaxI8Rows) return MOE_ERR_UNSUPPORTED;
  if (one_x && static_cast<int64_t>(d->T) * pad16(d->H) > kSpan) return MOE_ERR_UNSUPPORTED;
  static const int32_t some = 0;  // stands for device offsets
  const FfnI8Plan p = plan_ffn_i8(d, FfnI8Ws{}, nullptr, &some, moe_weights_i8{}, nullptr, nullptr);
  if (!moe::gemm_i8_supported(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true) ||
      !moe::gemm_i8_supported(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false))
    return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

// Weights of 8 bits with their scales (either kind).
template <class Weights>
int weights_8bit_ok(const moe_dims* d, const Weights* w) {
  if (w == nullptr) return MOE_ERR_NULL;
  const void* routed[] = {w->w_gate, w->w_up, w->w_down, w->s_gate, w->s_up, w->s_down};
  const void* shared[] = {w->sh_gate, w->sh_up, w->sh_down, w->sh_s_gate, w->sh_s_up, w->sh_s_down};
  for (const void* p : routed)
    if (p == nullptr) return MOE_ERR_NULL;
  for (const void* p : shared)
    if (d->n_shared > 0 && p == nullptr) return MOE_ERR_NULL;
  for (int i = 0; i < 6; ++i) {
    const uintptr_t mask = i < 3 ? 15 : 3;
    if ((reinterpret_cast<uintptr_t>(routed[i]) & mask) != 0) return MOE_ERR_ALIGN;
    if (d->n_shared > 0 && (reinterpret_cast<uintptr_t>(shared[i]) & mask) != 0) return MOE_ERR_ALIGN;
  }
  return MOE_OK;
}

// Where there are few rows the products quantise them.
void quantize_in_products(const moe_dims* d, const FfnI8Ws& fw, const uint16_t* x, const uint16_t* x_sh, FfnI8Plan* p) {
  if (moe::gemm_i8_quantizes(p->routed, p->up, p->sh ? &p->sh_up : nullptr, true)) {
    p->up.xb = x, p->sh_up.xb = x_sh;
    p->up.ldxb = p->sh_up.ldxb = d->H;
  }
  if (moe::gemm_i8_quantizes(p->routed, p->dn, p->sh ? &p->sh_dn : nullptr, false)) {
    p->dn.xb = fw.h, p->sh_dn.xb = fw.h_sh;
    p->dn.ldxb = d->I, p->sh_dn.ldxb = p->sh_dn.K;
  }
}

// The experts' networks on int8: x quantised (rows rows, or *n_rows), gate/up
// on it (through x_rows where x holds tokens), the hidden rows quantised, down.
// x == x_sh: the shared experts read the rows quantised for the routed ones.
int run_ffn_i8(const moe_dims* d, const uint16_t* x, const int32_t* x_rows, const int32_t* offsets,
               const moe_weights_i8* w, const uint16_t* x_sh, uint16_t* y_perm, uint16_t* y_shared, void* ws,
               const moe_taps* taps, hipStream_t st) {
  const bool one_x = x_rows != nullptr;
  const FfnI8Ws fw = carve_ffn_i8(d, one_x, ws);
  FfnI8Plan p = plan_ffn_i8(d, fw, x_rows, offsets, *w, y_perm, y_shared);
  quantize_in_products(d, fw, x, x_sh, &p);
  const int shw = static_cast<int>(sh_width(d)), rows = d->T * d->k;
  const int32_t* n_rows = offsets + d->E_local;
  hipError_t e;

  record(taps, 2 * MOE_STAGE_FFN_UP, st);
  const moe::QuantArgs qx{x, fw.xq, fw.xs, one_x ? nullptr : n_rows, d->H, p.up.ldx, one_x ? d->T : rows, d->H};
  const moe::QuantArgs qx_sh{x_sh, fw.xq_sh, fw.xs_sh, nullptr, d->H, p.up.ldx, d->T, d->H};
  e = p.up.xb ? hipSuccess : moe::launch_quantize_rows(qx, p.sh && !one_x ? &qx_sh : nullptr, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  e = moe::launch_gemm_i8(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_UP + 1, st);

  record(taps, 2 * MOE_STAGE_FFN_DOWN, st);
  const moe::QuantArgs qh{fw.h, fw.hq, fw.hs, n_rows, d->I, p.dn.ldx, rows, d->I};
  const moe::QuantArgs qh_sh{fw.h_sh, fw.hq_sh, fw.hs_sh, nullptr, shw, p.sh_dn.ldx, d->T, shw};
  e = p.dn.xb ? hipSuccess : moe::launch_quantize_rows(qh, p.sh ? &qh_sh : nullptr, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  e = moe::launch_gemm_i8(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_DOWN + 1, st);
  return MOE_OK;
}

// ---- the same on e4m3 experts ----

int64_t blocks128(int64_t n) { return (n + 127) / 128; }

// Workspace of the e4m3 expert FFN, as the int8 one's with a scale per 128 columns.
struct FfnF8Ws {
  uint8_t *xq, *xq_sh, *hq, *hq_sh;
  float *xs, *xs_sh, *hs, *hs_sh;
  uint16_t *h, *h_sh;
  size_t bytes;
};
FfnF8Ws carve_ffn_f8(const moe_dims* d, bool one_x, void* base) {
  FfnF8Ws w{};
  unsigned char* p = static_cast<unsigned char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* r = p ? p + off : nullptr;
    off += align_up(bytes);
    return r;
  };
  const size_t T = d->T, rows = T * d->k, shw = sh_width(d);
  const size_t x_rows = one_x ? T : rows, sh_x = one_x || shw == 0 ? 0 : T, sh_h = shw == 0 ? 0 : T;
  auto q = [&](size_t r, size_t cols) { return take(r * pad16(cols)); };
  auto scales = [&](size_t r, size_t cols) { return reinterpret_cast<float*>(take(r * blocks128(cols) * sizeof(float))); };
  w.xq = q(x_rows, d->H);
  w.xs = scales(x_rows, d->H);
  w.xq_sh = q(sh_x, d->H);
  w.xs_sh = scales(sh_x, d->H);
  w.h = reinterpret_cast<uint16_t*>(take(rows * d->I * sizeof(uint16_t)));
  w.hq = q(rows, d->I);
  w.hs = scales(rows, d->I);
  w.h_sh = reinterpret_cast<uint16_t*>(take(sh_h * shw * sizeof(uint16_t)));
  w.hq_sh = q(sh_h, shw);
  w.hs_sh = scales(sh_h, shw);
  if (one_x) {
    w.xq_sh = w.xq;
    w.xs_sh = w.xs;
  }
  w.bytes = off;
  return w;
}

size_t ffn_f8_ws(const moe_dims* d, bool one_x) { return carve_ffn_f8(d, one_x, nullptr).bytes; }

// The experts' products, built the same way for the limit check (null
// pointers) and for the launches.
struct FfnF8Plan {
  moe::Segments routed;
  moe::GemmF8 up, sh_up, dn, sh_dn;
  bool sh;
};
FfnF8Plan plan_ffn_f8(const moe_dims* d, const FfnF8Ws& fw, const int32_t* x_rows, const int32_t* offsets,
                      const moe_weights_f8& w, uint16_t* y_perm, uint16_t* y_shared) {
  const int shw = static_cast<int>(sh_width(d));
  const long long hp = pad16(d->H), ip = pad16(d->I), wp = pad16(shw);
  FfnF8Plan p{};
  p.routed = routed_segments(d, offsets);
  p.up = moe::GemmF8{fw.xq, fw.xs, x_rows, x_rows ? d->T : 0, offsets, 0, d->E_local, w.w_gate, w.w_up, w.s_gate, w.s_up,
                     fw.h, d->H, d->I, hp, hp, d->I, fw.hq, fw.hs, ip};
  p.sh_up = moe::GemmF8{fw.xq_sh, fw.xs_sh, nullptr, 0, nullptr, d->T, 1, w.sh_gate, w.sh_up, w.sh_s_gate, w.sh_s_up,
                        fw.h_sh, d->H, shw, hp, hp, shw, fw.hq_sh, fw.hs_sh, wp};
  p.dn = moe::GemmF8{fw.hq, fw.hs, nullptr, 0, offsets, 0, d->E_local, w.w_down, nullptr, w.s_down, nullptr,
                     y_perm, d->I, d->H, ip, ip, d->H};
  p.sh_dn = moe::GemmF8{fw.hq_sh, fw.hs_sh, nullptr, 0, nullptr, d->T, 1, w.sh_down, nullptr, w.sh_s_down, nullptr,
                        y_shared, shw, d->H, wp, wp, d->H};
  p.sh = d->n_shared > 0;
  return p;
}

int check_ffn_f8_limits(const moe_dims* d, bool one_x) {
  if (d->H > kMaxI8K || d->I > kMaxI8K || sh_width(d) > kMaxI8K) return MOE_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->T) * d->k > kMaxI8Rows) return MOE_ERR_UNSUPPORTED;
  if (one_x && static_cast<int64_t>(d->T) * pad16(d->H) > kSpan) return MOE_ERR_UNSUPPORTED;
  if (d->T == 0) return MOE_OK;
  static const int32_t some = 0;  // stands for device offsets
  const FfnF8Plan p = plan_ffn_f8(d, FfnF8Ws{}, nullptr, &some, moe_weights_f8{}, nullptr, nullptr);
  if (!moe::gemm_f8_supported(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true) ||
      !moe::gemm_f8_supported(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false))
    return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

// Where there are few rows the products quantise them (x and x_sh: null where the
// rows came quantised).
void quantize_in_f8_products(const moe_dims* d, const FfnF8Ws& fw, const uint16_t* x, const uint16_t* x_sh, FfnF8Plan* p) {
  if (x && moe::gemm_f8_takes_bf16(p->routed, p->up, p->sh ? &p->sh_up : nullptr, true)) {
    p->up.xb = x, p->sh_up.xb = x_sh;
    p->up.ldxb = p->sh_up.ldxb = d->H;
  }
  const bool up_quantises = !p->up.xb && moe::gemm_f8_quantizes(p->routed, p->up, p->sh ? &p->sh_up : nullptr);
  if (!up_quantises && moe::gemm_f8_takes_bf16(p->routed, p->dn, p->sh ? &p->sh_dn : nullptr, false)) {
    p->dn.xb = fw.h, p->sh_dn.xb = fw.h_sh;
    p->dn.ldxb = d->I, p->sh_dn.ldxb = p->sh_dn.K;
  }
}

// The experts' networks on e4m3: x quantised (unless it came so: x NULL), gate/up on
// it (through x_rows where x holds tokens), the hidden rows quantised, down.
int run_ffn_f8(const moe_dims* d, const uint16_t* x, const uint8_t* xq, const float* xs, const int32_t* x_rows,
               const int32_t* offsets, const moe_weights_f8* w, const uint16_t* x_sh, uint16_t* y_perm, uint16_t* y_shared,
               void* ws, const moe_taps* taps, hipStream_t st) {
  const bool one_x = x_rows != nullptr;
  const FfnF8Ws fw = carve_ffn_f8(d, one_x, ws);
  FfnF8Plan p = plan_ffn_f8(d, fw, x_rows, offsets, *w, y_perm, y_shared);
  if (!x) {
    p.up.x = p.sh_up.x = xq;
    p.up.x_scale = p.sh_up.x_scale = xs;
  }
  quantize_in_f8_products(d, fw, x, x_sh, &p);
  const int shw = static_cast<int>(sh_width(d)), rows = d->T * d->k;
  const int32_t* n_rows = offsets + d->E_local;
  hipError_t e;

  record(taps, 2 * MOE_STAGE_FFN_UP, st);
  const moe::QuantF8Args qx{x, fw.xq, fw.xs, one_x ? nullptr : n_rows, d->H, p.up.ldx, one_x ? d->T : rows, d->H};
  const moe::QuantF8Args qx_sh{x_sh, fw.xq_sh, fw.xs_sh, nullptr, d->H, p.up.ldx, d->T, d->H};
  e = !x || p.up.xb ? hipSuccess : moe::launch_quantize_rows_f8(qx, p.sh && !one_x ? &qx_sh : nullptr, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  e = moe::launch_gemm_f8(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_UP + 1, st);

  record(taps, 2 * MOE_STAGE_FFN_DOWN, st);
  const moe::QuantF8Args qh{fw.h, fw.hq, fw.hs, n_rows, d->I, p.dn.ldx, rows, d->I};
  const moe::QuantF8Args qh_sh{fw.h_sh, fw.hq_sh, fw.hs_sh, nullptr, shw, p.sh_dn.ldx, d->T, shw};
  // (unless gate/up's tiles have quantised the hidden rows, or down does)
  const bool quantised = p.dn.xb || (!p.up.xb && moe::gemm_f8_quantizes(p.routed, p.up, p.sh ? &p.sh_up : nullptr));
  e = quantised ? hipSuccess : moe::launch_quantize_rows_f8(qh, p.sh ? &qh_sh : nullptr, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  e = moe::launch_gemm_f8(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_FFN_DOWN + 1, st);
  return MOE_OK;
}

// ---- the norms ----

bool aligned2(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 1u) == 0; }
constexpr int64_t kMaxNormStride = int64_t{1} << 40;

// The checks of a norm and its rows; T of them.
int norm_ok(const moe_norm* n, const moe_norm_io* r, int32_t T) {
  if (n == nullptr || r == nullptr) return MOE_ERR_NULL;
  if (n->H < 1 || T < 0 || r->ldh < n->H || (r->h_out && r->ldh_out < n->H) || (r->x && r->ldx < n->H) ||
      (r->q && r->ldq < n->H))
    return MOE_ERR_DIMS;
  if (r->gate && (r->gate_row < 0 || r->gate_col < 0 || r->gate_col > 1)) return MOE_ERR_DIMS;
  if (r->gate && r->gate_row > 0 && r->gate_col == 1 && r->gate_row < n->H) return MOE_ERR_DIMS;
  if (n->H > moe::kNormMaxH || r->ldh > kMaxNormStride || r->ldh_out > kMaxNormStride || r->ldx > kMaxNormStride ||
      r->ldq > kMaxNormStride || r->gate_row > kMaxNormStride)
    return MOE_ERR_UNSUPPORTED;
  if (T > 1 && r->h && r->h_out == r->h && r->ldh_out != r->ldh) return MOE_ERR_DIMS;  // rows over other rows
  if (r->q && r->ldq % 16 != 0) return MOE_ERR_ALIGN;
  if ((r->q == nullptr) != (r->scale == nullptr)) return MOE_ERR_NULL;
  if (T == 0) return MOE_OK;
  if (!r->h || (!r->h_out && !r->x && !r->q)) return MOE_ERR_NULL;
  if (!aligned2(r->h) || !aligned2(r->h_out) || !aligned2(r->x) || !aligned2(r->gate) || !aligned2(n->weight) ||
      !aligned2(n->post_weight) || !aligned16(r->q) || (reinterpret_cast<uintptr_t>(r->scale) & 3u) != 0)
    return MOE_ERR_ALIGN;
  return MOE_OK;
}

moe::NormArgs norm_args(const moe_norm* n, const moe_norm_io* r, int32_t T, const uint16_t* y, int64_t ldy) {
  moe::NormArgs a{};
  a.T = T, a.H = n->H;
  a.y = y, a.ldy = ldy;
  a.weight = n->weight, a.post_weight = n->post_weight;
  a.rho = n->residual_scale, a.eps = n->eps, a.add = n->weight_add;
  a.h = r->h, a.h_out = r->h_out, a.x = r->x, a.q = r->q, a.scale = r->scale, a.gate = r->gate;
  a.ldh = r->ldh, a.ldho = r->ldh_out, a.ldx = r->ldx, a.ldq = r->ldq;
  a.gate_row = r->gate_row, a.gate_col = r->gate_col;
  return a;
}

// Up to M rows in all groups, R of them expected (where it is a number of rows),
// evenly spread.  Room for four times the rows, with M and with R as the expected
// number, us: 64 groups of 20, N 2048, K 4096 130 (tiles) and 84 (items); 32 of 20,
// N 2048, K 7168 85 and 72; 8 of 20, N 14336, K 4096 116 and 75.
moe::Segments linear_segments(const moe_linear_dims* d, const int32_t* offsets, bool grouped) {
  if (!grouped) return moe::Segments{nullptr, 1, d->M, d->M, d->M, d->M, 1};
  const int rows = d->R >= 1 && d->R <= d->M ? d->R : d->M;
  return moe::Segments{offsets, d->G, 0, d->M, d->M, rows / d->G, std::min(d->G, rows)};
}

// The checks that the two 8-bit products share.
int linear_ok(const moe_linear_dims* d, bool grouped, bool gathered, const void* xq, const void* x_scale,
              const void* wq, const void* w_scale, const void* y) {
  if (d == nullptr) return MOE_ERR_NULL;
  if (d->M < 0 || d->N < 1 || d->K < 1 || (grouped && d->G < 1) || (gathered && d->X < (d->M > 0 ? 1 : 0)))
    return MOE_ERR_DIMS;
  if (d->ldx < pad16(d->K) || d->ldw < pad16(d->K) || d->ldy < d->N) return MOE_ERR_DIMS;
  if (d->M > kMaxI8Rows || d->K > kMaxI8K || d->ldx > kMaxI8Stride || d->ldw > kMaxI8Stride || d->ldy > kMaxI8Stride)
    return MOE_ERR_UNSUPPORTED;
  if (grouped && d->G > moe::kMaxExperts) return MOE_ERR_UNSUPPORTED;
  if (gathered && d->X * d->ldx > kSpan) return MOE_ERR_UNSUPPORTED;
  if (d->ldx % 16 != 0 || d->ldw % 16 != 0) return MOE_ERR_ALIGN;
  if (d->M == 0) return MOE_OK;
  if (!xq || !x_scale || !wq || !w_scale || !y) return MOE_ERR_NULL;
  if (!aligned16(xq) || !aligned16(wq)) return MOE_ERR_ALIGN;
  if (((reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(w_scale)) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(y) & 1u) != 0)
    return MOE_ERR_ALIGN;
  return MOE_OK;
}

int forward_io_ok(const moe_dims* d, const float* logits, const int32_t* src, const void* x,
                  const int64_t* counts, const moe_bf16* out) {
  if (d->T > 0 && (!logits || !x || !out)) return MOE_ERR_NULL;
  if (counts && d->T > 0 && !src) return MOE_ERR_NULL;
  if (d->T > 0 && (!aligned16(x) || !aligned16(out))) return MOE_ERR_ALIGN;
  return MOE_OK;
}

// The layer's launches, ffn(x_rows, offsets) being the experts' networks and
// end(inv_pos, topk_w) what makes the layer's output of theirs.
template <class Ffn, class End>
int run_forward(const moe_dims* d, const moe::RouteGating& rg, const float* logits, const int32_t* src,
                const int32_t* local_experts, int64_t* counts, const moe_taps* taps,
                const ForwardWs& fw, hipStream_t st, Ffn ffn, End end) {
  int32_t* topk_idx = (taps && taps->topk_idx) ? taps->topk_idx : fw.topk_idx;
  float* topk_w = (taps && taps->topk_w) ? taps->topk_w : fw.topk_w;
  int32_t* offsets = (taps && taps->offsets) ? taps->offsets : fw.offsets;
  int32_t* perm_token = (taps && taps->perm_token) ? taps->perm_token : fw.perm_token;
  int32_t* inv_pos = (taps && taps->inv_pos) ? taps->inv_pos : fw.inv_pos;
  int32_t* expert_load = taps ? taps->expert_load : nullptr;
  hipError_t e;

  record(taps, 2 * MOE_STAGE_ROUTE, st);
  if (counts && expert_load) {
    e = moe::launch_fill_i32(expert_load, d->E, 0, st);
    if (e != hipSuccess) return MOE_ERR_DEVICE;
  }
  // decode-sized batches: the routing launch also writes the dispatch.
  // Larger ones are dispatched by the permute passes, whose count pass then
  // also takes the statistics: its blocks hold many more pairs than the
  // router's, and their histograms are summed in two levels (see
  // permute.hip) rather than by global atomics per bin and block.
  const moe::DispatchArgs disp{local_experts, d->E_local, offsets, perm_token, inv_pos};
  const bool stats_in_permute = counts != nullptr && static_cast<int64_t>(d->T) * d->k > moe::kDispatchPairs;
  int64_t* route_counts = stats_in_permute ? nullptr : counts;
  bool dispatched = false;
  e = moe::launch_route(d->T, d->E, d->k, logits, topk_idx, topk_w, route_counts ? src : nullptr, d->S,
                        route_counts, route_counts ? expert_load : nullptr, &rg, st, &disp, &dispatched);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_ROUTE + 1, st);

  record(taps, 2 * MOE_STAGE_PERMUTE, st);
  if (!dispatched) {
    e = moe::launch_permute(d->T, d->k, d->E, d->E_local, local_experts, topk_idx, offsets, perm_token,
                            inv_pos, fw.permute_ws, st, src, d->S, stats_in_permute ? counts : nullptr,
                            stats_in_permute ? expert_load : nullptr);
    if (e != hipSuccess) return MOE_ERR_DEVICE;
  }
  // no gathered copy of x: the gate/up GEMM reads its rows through perm_token
  record(taps, 2 * MOE_STAGE_PERMUTE + 1, st);

  if (d->T > 0) {
    const int s = ffn(perm_token, offsets);
    if (s != MOE_OK) return s;
  } else {
    record(taps, 2 * MOE_STAGE_FFN_UP, st);
    record(taps, 2 * MOE_STAGE_FFN_UP + 1, st);
    record(taps, 2 * MOE_STAGE_FFN_DOWN, st);
    record(taps, 2 * MOE_STAGE_FFN_DOWN + 1, st);
  }

  record(taps, 2 * MOE_STAGE_COMBINE, st);
  e = end(inv_pos, topk_w);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  record(taps, 2 * MOE_STAGE_COMBINE + 1, st);
  return MOE_OK;
}

template <class Ffn>
int run_forward(const moe_dims* d, const moe::RouteGating& rg, const float* logits, const int32_t* src,
                const int32_t* local_experts, int64_t* counts, moe_bf16* out, const moe_taps* taps,
                const ForwardWs& fw, hipStream_t st, Ffn ffn) {
  return run_forward(d, rg, logits, src, local_experts, counts, taps, fw, st, ffn,
                     [&](const int32_t* inv_pos, const float* topk_w) {
                       return moe::launch_combine(d->T, d->k, d->H, fw.y_perm, inv_pos, topk_w,
                                                  d->n_shared > 0 ? fw.y_shared : nullptr, out, st);
                     });
}

// The workspace of moe_forward_noalloc: a library-owned device array, one
// copy per device (every device the library runs on holds it until the
// process ends).  Host code never uses its name as an address: the address
// of a device's copy comes from hipGetSymbolAddress on that device.
static __device__ __align__(256) unsigned char scratch[MOE_NOALLOC_SCRATCH_BYTES];

// The device address of the current device's copy of `scratch`, looked up
// once per device (the pointers are cached with atomic operations, so
// concurrent first calls are safe); nullptr when the lookup fails.
void* scratch_address() {
  constexpr int kMaxDevices = 64;
  static void* addr[kMaxDevices] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  void* p = __atomic_load_n(&addr[dev], __ATOMIC_ACQUIRE);
  if (p != nullptr) return p;
  if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr) {
    (void)hipGetLastError();
    return nullptr;
  }
  __atomic_store_n(&addr[dev], p, __ATOMIC_RELEASE);
  return p;
}

}  // namespace

extern "C" {

int moe_abi_version(void) { return MOE_ABI_VERSION; }

const char* moe_strerror(int s) {
  switch (s) {
    case MOE_OK: return "ok";
    case MOE_ERR_NULL: return "a required pointer is NULL";
    case MOE_ERR_DIMS: return "inconsistent or negative dimensions";
    case MOE_ERR_UNSUPPORTED: return "dimensions beyond the kernels' limits";
    case MOE_ERR_WORKSPACE: return "workspace missing or too small";
    case MOE_ERR_DEVICE: return "kernel launch failed";
    case MOE_ERR_ALIGN: return "pointer not aligned as required";
    default: return "unknown status";
  }
}

size_t moe_workspace_bytes(const moe_dims* d, int entry) {
  if (check_dims(d) != MOE_OK || check_entry(d, entry) != MOE_OK) return 0;
  return entry_ws(d, entry);
}

int moe_validate(const moe_dims* d, int entry, size_t ws_bytes) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  s = check_entry(d, entry);
  if (s != MOE_OK) return s;
  if (entry != 0 && ws_bytes < entry_ws(d, entry)) return MOE_ERR_WORKSPACE;
  return MOE_OK;
}

int moe_route(const moe_dims* d, const moe_gating* gating, const float* logits, int32_t* topk_idx,
              float* topk_w, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  moe::RouteGating rg;
  s = gating_ok(d, gating, &rg);
  if (s != MOE_OK) return s;
  if (d->T > 0 && (!logits || !topk_idx || !topk_w)) return MOE_ERR_NULL;
  return status(moe::launch_route(d->T, d->E, d->k, logits, topk_idx, topk_w, nullptr, d->S,
                                  nullptr, nullptr, &rg, static_cast<hipStream_t>(stream)));
}

int moe_route_stats(const moe_dims* d, const int32_t* src, const int32_t* topk_idx,
                    int64_t* counts, int32_t* expert_load, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (!counts || (d->T > 0 && (!src || !topk_idx))) return MOE_ERR_NULL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (expert_load && moe::launch_fill_i32(expert_load, d->E, 0, st) != hipSuccess)
    return MOE_ERR_DEVICE;
  return status(moe::launch_route_stats(d->T, d->k, d->S, d->E, src, topk_idx, counts,
                                        expert_load, st));
}

int moe_permute(const moe_dims* d, const int32_t* topk_idx, const int32_t* local_experts,
                const moe_bf16* x, int32_t* offsets, int32_t* perm_token, int32_t* inv_pos,
                moe_bf16* x_perm, void* ws, size_t ws_bytes, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (!local_experts && d->E_local != d->E) return MOE_ERR_DIMS;
  if (!offsets || (d->T > 0 && (!topk_idx || !perm_token || !inv_pos))) return MOE_ERR_NULL;
  if ((x == nullptr) != (x_perm == nullptr)) return MOE_ERR_NULL;
  if (x && (!aligned16(x) || !aligned16(x_perm))) return MOE_ERR_ALIGN;
  s = check_ws(d, MOE_ENTRY_PERMUTE, ws, ws_bytes);
  if (s != MOE_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e = moe::launch_permute(d->T, d->k, d->E, d->E_local, local_experts, topk_idx,
                                     offsets, perm_token, inv_pos, ws, st);
  if (e != hipSuccess) return MOE_ERR_DEVICE;
  if (x) {
    e = moe::launch_gather_rows(d->T * d->k, d->H, perm_token, offsets + d->E_local, x, x_perm, st);
    if (e != hipSuccess) return MOE_ERR_DEVICE;
  }
  return MOE_OK;
}

int moe_expert_ffn(const moe_dims* d, const moe_bf16* x_perm, const int32_t* offsets,
                   const moe_weights* w, const moe_bf16* x, moe_bf16* y_perm, moe_bf16* y_shared,
                   void* ws, size_t ws_bytes, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  s = weights_ok(d, w);
  if (s != MOE_OK) return s;
  if (!x_perm || !offsets || !y_perm) return MOE_ERR_NULL;
  if (d->n_shared > 0 && (!x || !y_shared)) return MOE_ERR_NULL;
  if (!aligned16(x_perm) || !aligned16(y_perm)) return MOE_ERR_ALIGN;
  if (d->n_shared > 0 && (!aligned16(x) || !aligned16(y_shared))) return MOE_ERR_ALIGN;
  s = check_entry(d, MOE_ENTRY_EXPERT_FFN);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_EXPERT_FFN, ws, ws_bytes);
  if (s != MOE_OK) return s;
  if (d->T == 0) return MOE_OK;
  return run_ffn(d, x_perm, nullptr, offsets, w, x, y_perm, y_shared, ws, nullptr,
                 static_cast<hipStream_t>(stream));
}

int moe_combine(const moe_dims* d, const moe_bf16* y_perm, const int32_t* inv_pos,
                const float* topk_w, const moe_bf16* y_shared, moe_bf16* out, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (d->T > 0 && (!y_perm || !inv_pos || !topk_w || !out)) return MOE_ERR_NULL;
  if (d->T > 0 && (!aligned16(y_perm) || !aligned16(out) || (y_shared && !aligned16(y_shared))))
    return MOE_ERR_ALIGN;
  return status(moe::launch_combine(d->T, d->k, d->H, y_perm, inv_pos, topk_w, y_shared, out,
                                    static_cast<hipStream_t>(stream)));
}

int moe_forward(const moe_dims* d, const moe_gating* gating, const float* logits, const int32_t* src,
                const moe_bf16* x, const int32_t* local_experts, const moe_weights* w, int64_t* counts,
                moe_bf16* out, const moe_taps* taps, void* ws, size_t ws_bytes, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  moe::RouteGating rg;
  s = gating_ok(d, gating, &rg);
  if (s != MOE_OK) return s;
  if (!local_experts && d->E_local != d->E) return MOE_ERR_DIMS;
  s = weights_ok(d, w);
  if (s != MOE_OK) return s;
  s = forward_io_ok(d, logits, src, x, counts, out);
  if (s != MOE_OK) return s;
  s = check_entry(d, MOE_ENTRY_FORWARD);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_FORWARD, ws, ws_bytes);
  if (s != MOE_OK) return s;

  hipStream_t st = static_cast<hipStream_t>(stream);
  const ForwardWs fw = carve_forward(d, ffn_ws(d), ws);
  return run_forward(d, rg, logits, src, local_experts, counts, out, taps, fw, st,
                     [&](const int32_t* x_rows, const int32_t* offsets) {
                       return run_ffn(d, x, x_rows, offsets, w, x, fw.y_perm, fw.y_shared, fw.ffn_ws, taps, st);
                     });
}

int moe_forward_noalloc(const moe_dims* d, const moe_gating* gating, const float* logits, const int32_t* src,
                        const moe_bf16* x, const int32_t* local_experts, const moe_weights* w, int64_t* counts,
                        moe_bf16* out, const moe_taps* taps, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  s = check_entry(d, MOE_ENTRY_FORWARD);
  if (s != MOE_OK) return s;
  if (entry_ws(d, MOE_ENTRY_FORWARD) > MOE_NOALLOC_SCRATCH_BYTES) return MOE_ERR_WORKSPACE;
  // the scratch copy used is the current device's: the stream must be one of its streams
  int cur = 0, sdev = 0;
  if (hipGetDevice(&cur) != hipSuccess || hipStreamGetDevice(static_cast<hipStream_t>(stream), &sdev) != hipSuccess ||
      cur != sdev)
    return MOE_ERR_DEVICE;
  void* ws = scratch_address();
  if (ws == nullptr) return MOE_ERR_DEVICE;
  // the forward workspace needs no initialisation: every region is written
  // before it is read within the call
  return moe_forward(d, gating, logits, src, x, local_experts, w, counts, out, taps, ws,
                     MOE_NOALLOC_SCRATCH_BYTES, stream);
}

int moe_quantize_rows(int32_t rows, int32_t cols, const moe_bf16* x, int64_t ldx, int8_t* q, int64_t ldq,
                      float* scale, void* stream) {
  if (rows < 0 || cols < 1 || ldx < cols || ldq < cols) return MOE_ERR_DIMS;
  if (ldx > (int64_t{1} << 40) || ldq > (int64_t{1} << 40) || cols > kIntMax - 64) return MOE_ERR_UNSUPPORTED;
  if (ldq % 16 != 0) return MOE_ERR_ALIGN;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return MOE_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(x) & 1u) != 0 || !aligned16(q) || (reinterpret_cast<uintptr_t>(scale) & 3u) != 0)
    return MOE_ERR_ALIGN;
  const moe::QuantArgs a{x, q, scale, nullptr, ldx, ldq, rows, cols};
  return status(moe::launch_quantize_rows(a, nullptr, static_cast<hipStream_t>(stream)));
}

int moe_linear_i8(const moe_linear_dims* d, const int8_t* xq, const float* x_scale, const int8_t* wq,
                  const float* w_scale, moe_bf16* y, void* stream) {
  const int s = linear_ok(d, false, false, xq, x_scale, wq, w_scale, y);
  if (s != MOE_OK || d->M == 0) return s;
  const moe::Segments seg = linear_segments(d, nullptr, false);
  const moe::GemmI8 a{xq, x_scale, nullptr, 0, nullptr, d->M, 1, wq, nullptr, w_scale, nullptr, y,
                      d->K, d->N, d->ldx, d->ldw, d->ldy};
  if (!moe::gemm_i8_supported(seg, a, nullptr, false)) return MOE_ERR_UNSUPPORTED;
  return status(moe::launch_gemm_i8(seg, a, nullptr, false, static_cast<hipStream_t>(stream)));
}

int moe_grouped_linear_i8(const moe_linear_dims* d, const int8_t* xq, const float* x_scale, const int32_t* x_rows,
                          const int32_t* offsets, const int8_t* wq, const float* w_scale, moe_bf16* y, void* stream) {
  const int s = linear_ok(d, true, x_rows != nullptr, xq, x_scale, wq, w_scale, y);
  if (s != MOE_OK || d->M == 0) return s;
  if (!offsets) return MOE_ERR_NULL;
  if (((reinterpret_cast<uintptr_t>(offsets) | reinterpret_cast<uintptr_t>(x_rows)) & 3u) != 0) return MOE_ERR_ALIGN;
  const moe::Segments seg = linear_segments(d, offsets, true);
  const moe::GemmI8 a{xq, x_scale, x_rows, x_rows ? d->X : 0, offsets, 0, d->G, wq, nullptr, w_scale, nullptr, y,
                      d->K, d->N, d->ldx, d->ldw, d->ldy};
  if (!moe::gemm_i8_supported(seg, a, nullptr, false)) return MOE_ERR_UNSUPPORTED;
  return status(moe::launch_gemm_i8(seg, a, nullptr, false, static_cast<hipStream_t>(stream)));
}

int moe_expert_ffn_i8(const moe_dims* d, const moe_bf16* x_perm, const int32_t* offsets, const moe_weights_i8* w,
                      const moe_bf16* x, moe_bf16* y_perm, moe_bf16* y_shared, void* ws, size_t ws_bytes,
                      void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  s = weights_8bit_ok(d, w);
  if (s != MOE_OK) return s;
  if (!x_perm || !offsets || !y_perm) return MOE_ERR_NULL;
  if (d->n_shared > 0 && (!x || !y_shared)) return MOE_ERR_NULL;
  if (!aligned16(x_perm) || !aligned16(y_perm)) return MOE_ERR_ALIGN;
  if (d->n_shared > 0 && (!aligned16(x) || !aligned16(y_shared))) return MOE_ERR_ALIGN;
  s = check_entry(d, MOE_ENTRY_EXPERT_FFN_I8);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_EXPERT_FFN_I8, ws, ws_bytes);
  if (s != MOE_OK) return s;
  if (d->T == 0) return MOE_OK;
  return run_ffn_i8(d, x_perm, nullptr, offsets, w, x, y_perm, y_shared, ws, nullptr, static_cast<hipStream_t>(stream));
}

int moe_forward_i8(const moe_dims* d, const moe_gating* gating, const float* logits, const int32_t* src,
                   const moe_bf16* x, const int32_t* local_experts, const moe_weights_i8* w, int64_t* counts,
                   moe_bf16* out, const moe_taps* taps, void* ws, size_t ws_bytes, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  moe::RouteGating rg;
  s = gating_ok(d, gating, &rg);
  if (s != MOE_OK) return s;
  if (!local_experts && d->E_local != d->E) return MOE_ERR_DIMS;
  s = weights_8bit_ok(d, w);
  if (s != MOE_OK) return s;
  s = forward_io_ok(d, logits, src, x, counts, out);
  if (s != MOE_OK) return s;
  s = check_entry(d, MOE_ENTRY_FORWARD_I8);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_FORWARD_I8, ws, ws_bytes);
  if (s != MOE_OK) return s;

  hipStream_t st = static_cast<hipStream_t>(stream);
  const ForwardWs fw = carve_forward(d, ffn_i8_ws(d, true), ws);
  return run_forward(d, rg, logits, src, local_experts, counts, out, taps, fw, st,
                     [&](const int32_t* x_rows, const int32_t* offsets) {
                       return run_ffn_i8(d, x, x_rows, offsets, w, x, fw.y_perm, fw.y_shared, fw.ffn_ws, taps, st);
                     });
}

int moe_norm_rows(const moe_norm* n, const moe_norm_io* r, int32_t T, const moe_bf16* y, int64_t ldy, void* stream) {
  const int s = norm_ok(n, r, T);
  if (s != MOE_OK) return s;
  if (y && ldy < n->H) return MOE_ERR_DIMS;
  if (y && ldy > kMaxNormStride) return MOE_ERR_UNSUPPORTED;
  if (y && T > 1 && r->x == y && r->ldx != ldy) return MOE_ERR_DIMS;
  if (!aligned2(y)) return MOE_ERR_ALIGN;
  moe::NormArgs a = norm_args(n, r, T, y, ldy);
  if (!y) a.post_weight = a.gate = nullptr;  // nothing to norm or to gate
  return status(moe::launch_norm(a, static_cast<hipStream_t>(stream)));
}

int moe_quantize_rows_f8(int32_t rows, int32_t cols, const moe_bf16* x, int64_t ldx, moe_f8* q, int64_t ldq,
                         float* scale, void* stream) {
  if (rows < 0 || cols < 1 || ldx < cols || ldq < cols) return MOE_ERR_DIMS;
  if (ldx > kMaxNormStride || ldq > kMaxNormStride || cols > kIntMax - 256) return MOE_ERR_UNSUPPORTED;
  if (ldq % 16 != 0) return MOE_ERR_ALIGN;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return MOE_ERR_NULL;
  if (!aligned2(x) || !aligned16(q) || (reinterpret_cast<uintptr_t>(scale) & 3u) != 0) return MOE_ERR_ALIGN;
  const moe::QuantF8Args a{x, q, scale, nullptr, ldx, ldq, rows, cols};
  return status(moe::launch_quantize_rows_f8(a, nullptr, static_cast<hipStream_t>(stream)));
}

int moe_quantize_blocks_f8(int32_t G, int32_t rows, int32_t cols, const moe_bf16* x, int64_t ldx, moe_f8* q,
                           int64_t ldq, float* scale, void* stream) {
  if (G < 0 || rows < 1 || cols < 1 || ldx < cols || ldq < cols) return MOE_ERR_DIMS;
  if (ldx > kMaxNormStride || ldq > kMaxNormStride || cols > kIntMax - 256 || rows > kIntMax - 256 ||
      !moe::quantize_blocks_f8_supported(G, rows, cols))
    return MOE_ERR_UNSUPPORTED;
  if (ldq % 16 != 0) return MOE_ERR_ALIGN;
  if (G == 0) return MOE_OK;
  if (!x || !q || !scale) return MOE_ERR_NULL;
  if (!aligned2(x) || !aligned16(q) || (reinterpret_cast<uintptr_t>(scale) & 3u) != 0) return MOE_ERR_ALIGN;
  return status(moe::launch_quantize_blocks_f8(G, rows, cols, x, ldx, q, ldq, scale, static_cast<hipStream_t>(stream)));
}

int moe_linear_f8(const moe_linear_dims* d, const moe_f8* xq, const float* x_scale, const moe_f8* wq,
                  const float* w_scale, moe_bf16* y, void* stream) {
  const int s = linear_ok(d, false, false, xq, x_scale, wq, w_scale, y);
  if (s != MOE_OK || d->M == 0) return s;
  const moe::Segments seg = linear_segments(d, nullptr, false);
  const moe::GemmF8 a{xq, x_scale, nullptr, 0, nullptr, d->M, 1, wq, nullptr, w_scale, nullptr, y,
                      d->K, d->N, d->ldx, d->ldw, d->ldy};
  if (!moe::gemm_f8_supported(seg, a, nullptr, false)) return MOE_ERR_UNSUPPORTED;
  return status(moe::launch_gemm_f8(seg, a, nullptr, false, static_cast<hipStream_t>(stream)));
}

int moe_grouped_linear_f8(const moe_linear_dims* d, const moe_f8* xq, const float* x_scale, const int32_t* x_rows,
                          const int32_t* offsets, const moe_f8* wq, const float* w_scale, moe_bf16* y, void* stream) {
  const int s = linear_ok(d, true, x_rows != nullptr, xq, x_scale, wq, w_scale, y);
  if (s != MOE_OK || d->M == 0) return s;
  if (!offsets) return MOE_ERR_NULL;
  if (((reinterpret_cast<uintptr_t>(offsets) | reinterpret_cast<uintptr_t>(x_rows)) & 3u) != 0) return MOE_ERR_ALIGN;
  const moe::Segments seg = linear_segments(d, offsets, true);
  const moe::GemmF8 a{xq, x_scale, x_rows, x_rows ? d->X : 0, offsets, 0, d->G, wq, nullptr, w_scale, nullptr, y,
                      d->K, d->N, d->ldx, d->ldw, d->ldy};
  if (!moe::gemm_f8_supported(seg, a, nullptr, false)) return MOE_ERR_UNSUPPORTED;
  return status(moe::launch_gemm_f8(seg, a, nullptr, false, static_cast<hipStream_t>(stream)));
}

int moe_expert_ffn_f8(const moe_dims* d, const moe_bf16* x_perm, const int32_t* offsets, const moe_weights_f8* w,
                      const moe_bf16* x, moe_bf16* y_perm, moe_bf16* y_shared, void* ws, size_t ws_bytes,
                      void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  s = weights_8bit_ok(d, w);
  if (s != MOE_OK) return s;
  if (!x_perm || !offsets || !y_perm) return MOE_ERR_NULL;
  if (d->n_shared > 0 && (!x || !y_shared)) return MOE_ERR_NULL;
  if (!aligned16(x_perm) || !aligned16(y_perm)) return MOE_ERR_ALIGN;
  if (d->n_shared > 0 && (!aligned16(x) || !aligned16(y_shared))) return MOE_ERR_ALIGN;
  s = check_entry(d, MOE_ENTRY_EXPERT_FFN_F8);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_EXPERT_FFN_F8, ws, ws_bytes);
  if (s != MOE_OK) return s;
  if (d->T == 0) return MOE_OK;
  return run_ffn_f8(d, x_perm, nullptr, nullptr, nullptr, offsets, w, x, y_perm, y_shared, ws, nullptr,
                    static_cast<hipStream_t>(stream));
}

int moe_forward_f8(const moe_dims* d, const moe_gating* gating, const float* logits, const int32_t* src,
                   const moe_bf16* x, const moe_f8* xq, const float* x_scale, const int32_t* local_experts,
                   const moe_weights_f8* w, int64_t* counts, moe_bf16* out, const moe_norm* norm,
                   const moe_norm_io* rows, const moe_taps* taps, void* ws, size_t ws_bytes, void* stream) {
  int s = check_dims(d);
  if (s != MOE_OK) return s;
  moe::RouteGating rg;
  s = gating_ok(d, gating, &rg);
  if (s != MOE_OK) return s;
  if (!local_experts && d->E_local != d->E) return MOE_ERR_DIMS;
  s = weights_8bit_ok(d, w);
  if (s != MOE_OK) return s;
  // rows in one form; an output of the layer or its end
  if ((xq == nullptr) != (x_scale == nullptr) || (norm == nullptr) != (rows == nullptr)) return MOE_ERR_NULL;
  if (x && xq) return MOE_ERR_DIMS;
  const void* some_x = x ? static_cast<const void*>(x) : xq;
  s = forward_io_ok(d, logits, src, some_x, counts, out || !rows ? out : reinterpret_cast<const moe_bf16*>(kAlign));
  if (s != MOE_OK) return s;
  if ((reinterpret_cast<uintptr_t>(x_scale) & 3u) != 0) return MOE_ERR_ALIGN;
  if (norm) {
    if (norm->H != d->H) return MOE_ERR_DIMS;
    s = norm_ok(norm, rows, d->T);
    if (s != MOE_OK) return s;
  }
  s = check_entry(d, MOE_ENTRY_FORWARD_F8);
  if (s != MOE_OK) return s;
  s = check_ws(d, MOE_ENTRY_FORWARD_F8, ws, ws_bytes);
  if (s != MOE_OK) return s;

  hipStream_t st = static_cast<hipStream_t>(stream);
  const ForwardWs fw = carve_forward(d, ffn_f8_ws(d, true), ws);
  const uint16_t* y_shared = d->n_shared > 0 ? fw.y_shared : nullptr;
  return run_forward(
      d, rg, logits, src, local_experts, counts, taps, fw, st,
      [&](const int32_t* x_rows, const int32_t* offsets) {
        return run_ffn_f8(d, x, xq, x_scale, x_rows, offsets, w, x, fw.y_perm, fw.y_shared, fw.ffn_ws, taps, st);
      },
      [&](const int32_t* inv_pos, const float* topk_w) {
        if (!norm) return moe::launch_combine(d->T, d->k, d->H, fw.y_perm, inv_pos, topk_w, y_shared, out, st);
        moe::NormArgs a = norm_args(norm, rows, d->T, nullptr, 0);
        a.k = d->k;
        a.y_perm = fw.y_perm, a.y_shared = y_shared, a.inv_pos = inv_pos, a.topk_w = topk_w, a.out = out;
        return moe::launch_norm(a, st);
      });
}

// For the tests, which assert the kernel that a shape is meant for (not part
// of include/moe.h): how the expert GEMMs of these dims are launched by
// moe_forward (rows_indexed) or moe_expert_ffn.  out[g] for g = 0 gate/up, 1
// down: kernel, tail, split_k, merged, blocks, sh_kernel, sh_blocks.
int moe_test_ffn_plan(const moe_dims* d, int rows_indexed, int64_t out[2][7]) {
  const int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (check_ffn_limits(d, rows_indexed != 0) != MOE_OK) return MOE_ERR_UNSUPPORTED;
  const FfnPlan p = plan_ffn(d, nullptr, nullptr, rows_indexed != 0, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr);
  const bool sh = d->n_shared > 0;
  const moe::Segments* seg = sh ? &p.shared : nullptr;
  const moe::GemmPlan g[2] = {moe::plan_ffn_up(p.routed, p.up, seg, sh ? &p.sh_up : nullptr),
                              moe::plan_ffn_down(p.routed, p.dn, seg, sh ? &p.sh_dn : nullptr)};
  for (int i = 0; i < 2; ++i) {
    const int64_t v[7] = {g[i].kernel, g[i].tail, g[i].split_k, g[i].merged, g[i].blocks, g[i].sh_kernel, g[i].sh_blocks};
    std::copy(v, v + 7, out[i]);
  }
  return MOE_OK;
}

// For the tests: how the 8-bit products run (moe::GemmI8Plan: kernel, parts,
// rows, half), of moe_linear_i8 or moe_grouped_linear_i8, and of
// moe_forward_i8's or moe_expert_ffn_i8's gate/up and down.
static moe::GemmI8 plan_args(const moe_linear_dims* d, const moe::Segments& seg) {
  moe::GemmI8 a{};
  a.offsets = seg.offsets;
  a.static_rows = seg.offsets ? 0 : d->M;
  a.groups = seg.groups;
  a.K = d->K, a.N = d->N;
  return a;
}

int moe_test_linear_i8_plan(const moe_linear_dims* d, int grouped, int64_t out[4]) {
  static const int32_t some = 0;  // stands for device offsets
  if (d == nullptr || d->M < 1 || d->N < 1 || d->K < 1 || (grouped && d->G < 1)) return MOE_ERR_DIMS;
  const moe::Segments seg = linear_segments(d, grouped ? &some : nullptr, grouped != 0);
  const moe::GemmI8Plan p = moe::plan_gemm_i8(seg, plan_args(d, seg), nullptr, false);
  const int64_t v[4] = {p.kernel, p.parts, p.rows, p.half};
  std::copy(v, v + 4, out);
  return MOE_OK;
}

// For the tests: moe::GemmI8Round of a product on tiles, `tiles` of which have rows.
int moe_test_linear_i8_round(const moe_linear_dims* d, int grouped, int tiles, int64_t out[2]) {
  static const int32_t some = 0;
  if (d == nullptr || d->M < 1 || d->N < 1 || d->K < 1 || tiles < 0 || (grouped && d->G < 1)) return MOE_ERR_DIMS;
  const moe::Segments seg = linear_segments(d, grouped ? &some : nullptr, grouped != 0);
  const moe::GemmI8Round r = moe::round_gemm_i8(seg, plan_args(d, seg), nullptr, false, tiles);
  out[0] = r.grid, out[1] = r.parts;
  return MOE_OK;
}

int moe_test_ffn_i8_plan(const moe_dims* d, int64_t out[2][4]) {
  const int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (d->T == 0 || check_ffn_i8_limits(d, false) != MOE_OK) return MOE_ERR_UNSUPPORTED;
  static const int32_t some = 0;     // stands for device offsets
  static const uint16_t row = 0;     // ... and rows
  FfnI8Ws fw{};
  uint16_t h = 0;
  fw.h = fw.h_sh = &h;
  FfnI8Plan p = plan_ffn_i8(d, fw, nullptr, &some, moe_weights_i8{}, nullptr, nullptr);
  quantize_in_products(d, fw, &row, &row, &p);
  const moe::GemmI8Plan g[2] = {moe::plan_gemm_i8(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true),
                                moe::plan_gemm_i8(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false)};
  for (int i = 0; i < 2; ++i) {
    const int64_t v[4] = {g[i].kernel, g[i].parts, g[i].rows, g[i].half};
    std::copy(v, v + 4, out[i]);
  }
  return MOE_OK;
}

// For the tests: how the e4m3 products run (moe::GemmF8Plan), of moe_linear_f8 or
// moe_grouped_linear_f8, and of the layer's gate/up and down (of rows that come
// quantised or not); apart from that, whether two workgroups share a CU.
static int linear_f8_plan(const moe_linear_dims* d, bool grouped, moe::GemmF8Plan* out) {
  static const int32_t some = 0;  // stands for device offsets
  if (d == nullptr || d->M < 1 || d->N < 1 || d->K < 1 || (grouped && d->G < 1)) return MOE_ERR_DIMS;
  const moe::Segments seg = linear_segments(d, grouped ? &some : nullptr, grouped);
  moe::GemmF8 a{};
  a.offsets = seg.offsets;
  a.static_rows = seg.offsets ? 0 : d->M;
  a.groups = seg.groups;
  a.K = d->K, a.N = d->N;
  *out = moe::plan_gemm_f8(seg, a, nullptr, false);
  return MOE_OK;
}

static int ffn_f8_plan(const moe_dims* d, bool quantised, moe::GemmF8Plan out[2]) {
  const int s = check_dims(d);
  if (s != MOE_OK) return s;
  if (d->T == 0 || check_ffn_f8_limits(d, false) != MOE_OK) return MOE_ERR_UNSUPPORTED;
  static const int32_t some = 0;
  static const uint16_t row = 0;
  FfnF8Ws fw{};
  uint16_t h = 0;
  fw.h = fw.h_sh = &h;
  FfnF8Plan p = plan_ffn_f8(d, fw, nullptr, &some, moe_weights_f8{}, nullptr, nullptr);
  quantize_in_f8_products(d, fw, quantised ? nullptr : &row, quantised ? nullptr : &row, &p);
  out[0] = moe::plan_gemm_f8(p.routed, p.up, p.sh ? &p.sh_up : nullptr, true);
  out[1] = moe::plan_gemm_f8(p.routed, p.dn, p.sh ? &p.sh_dn : nullptr, false);
  return MOE_OK;
}

int moe_test_linear_f8_plan(const moe_linear_dims* d, int grouped, int64_t out[4]) {
  moe::GemmF8Plan p;
  const int s = linear_f8_plan(d, grouped != 0, &p);
  if (s != MOE_OK) return s;
  const int64_t v[4] = {p.kernel, p.parts, p.rows, p.half};
  std::copy(v, v + 4, out);
  return MOE_OK;
}

int moe_test_linear_f8_pair(const moe_linear_dims* d, int grouped, int64_t* out) {
  moe::GemmF8Plan p;
  const int s = linear_f8_plan(d, grouped != 0, &p);
  if (s == MOE_OK) *out = p.pair;
  return s;
}

int moe_test_ffn_f8_plan(const moe_dims* d, int quantised, int64_t out[2][4]) {
  moe::GemmF8Plan g[2];
  const int s = ffn_f8_plan(d, quantised != 0, g);
  if (s != MOE_OK) return s;
  for (int i = 0; i < 2; ++i) {
    const int64_t v[4] = {g[i].kernel, g[i].parts, g[i].rows, g[i].half};
    std::copy(v, v + 4, out[i]);
  }
  return MOE_OK;
}

int moe_test_ffn_f8_pair(const moe_dims* d, int quantised, int64_t out[2]) {
  moe::GemmF8Plan g[2];
  const int s = ffn_f8_plan(d, quantised != 0, g);
  if (s != MOE_OK) return s;
  for (int i = 0; i < 2; ++i) out[i] = g[i].pair;
  return MOE_OK;
}

// For the tests: workgroups of the norms (moe::norm_blocks).
int moe_test_norm_blocks(int T, int rows, int most) { return moe::norm_blocks(T, rows, most); }

// For the tests: pairs per thread in moe_route_stats.
int moe_test_stats_per(int n_pairs, int S, int E) { return moe::stats_per(n_pairs, S, E); }

// For the tests: waves of a layer's workgroup in moe_place_experts.
int moe_test_place_waves(int L, int S, int E, int G) { return moe::place_waves(L, S, E, G); }

size_t moe_place_slots(const moe_place_dims* pd, const int32_t* cap) {
  if (pd == nullptr || cap == nullptr || pd->E < 1 || pd->G < 1) return 0;
  int slots = 0;
  for (int g = 0; g < pd->G; ++g) slots = std::max(slots, std::min(std::max(cap[g], 0), pd->E));
  return static_cast<size_t>(slots);
}

int moe_place_experts(const moe_place_dims* pd, const int32_t* cap, const int64_t* A,
                      const int64_t* B, const double* D, const double* M, const int32_t* x0,
                      int32_t* x, int32_t* rank_experts, double* cost, void* stream) {
  if (pd == nullptr || cap == nullptr) return MOE_ERR_NULL;
  if (pd->L < 0 || pd->S < 1 || pd->E < 1 || pd->G < 1) return MOE_ERR_DIMS;
  if (pd->E > moe::kPlaceMaxExperts || pd->G > moe::kPlaceMaxRanks ||
      static_cast<int64_t>(pd->S) * pd->G > moe::kPlaceMaxSourceRanks ||
      moe::place_lds_bytes(pd->S, pd->E, pd->G) > static_cast<size_t>(moe::kPlaceMaxLdsBytes))
    return MOE_ERR_UNSUPPORTED;
  int64_t room = 0;
  for (int g = 0; g < pd->G; ++g) {
    if (cap[g] < 0) return MOE_ERR_DIMS;
    room += std::min(cap[g], pd->E);
  }
  if (room < pd->E) return MOE_ERR_DIMS;  // some expert would have no rank
  if (static_cast<int64_t>(pd->L) * pd->S * pd->E > (int64_t{1} << 40)) return MOE_ERR_UNSUPPORTED;
  if (pd->L == 0) return MOE_OK;
  if (!A || !D || !x0 || !x) return MOE_ERR_NULL;
  auto al = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  if (!al(A, 8) || !al(B, 8) || !al(D, 8) || !al(M, 8) || !al(cost, 8) || !al(x0, 4) || !al(x, 4) ||
      !al(rank_experts, 4))
    return MOE_ERR_ALIGN;
  moe::PlaceArgs a{};
  a.L = pd->L;
  a.S = pd->S;
  a.E = pd->E;
  a.G = pd->G;
  a.slots = static_cast<int>(moe_place_slots(pd, cap));
  a.alpha = pd->alpha;
  a.beta = pd->beta;
  a.gamma = pd->gamma;
  a.m_uniform = pd->m_uniform;
  a.cap = cap;
  a.A = A;
  a.B = B;
  a.D = D;
  a.M = M;
  a.x0 = x0;
  a.x = x;
  a.rank_experts = rank_experts;
  a.cost = cost;
  return status(moe::launch_place(a, static_cast<hipStream_t>(stream)));
}

int moe_window_stats(const moe_window_dims* wd, const int64_t* A, const int64_t* B, const int32_t* x,
                     const int32_t* home, const int32_t* engine, int64_t* remote, int64_t* total,
                     int64_t* rank_load, double* pressure, void* stream) {
  if (wd == nullptr) return MOE_ERR_NULL;
  if (wd->L < 0 || wd->S < 1 || wd->E < 1 || wd->G < 1 || wd->n_engines < 1) return MOE_ERR_DIMS;
  if (engine == nullptr && wd->n_engines != wd->G) return MOE_ERR_DIMS;
  if (wd->E > moe::kWindowMaxExperts || wd->G > moe::kWindowMaxRanks ||
      wd->n_engines > moe::kWindowMaxEngines ||
      static_cast<int64_t>(wd->L) * wd->S * wd->E > (int64_t{1} << 40))
    return MOE_ERR_UNSUPPORTED;
  if (wd->L > 0 && (!A || !x || !home || !remote || !total || !rank_load)) return MOE_ERR_NULL;
  auto al = [](const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  if (!al(A, 8) || !al(B, 8) || !al(remote, 8) || !al(total, 8) || !al(rank_load, 8) || !al(pressure, 8) ||
      !al(x, 4) || !al(home, 4) || !al(engine, 4))
    return MOE_ERR_ALIGN;
  moe::WindowArgs a{wd->L, wd->S, wd->E, wd->G, wd->n_engines, A, B, x, home, engine,
                    remote, total, rank_load, pressure};
  return status(moe::launch_window(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
