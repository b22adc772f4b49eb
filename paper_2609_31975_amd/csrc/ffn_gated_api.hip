// Host side of include/ffn_gated.h: argument checks, workspace carve-up and kernel sequencing.  No
// allocation, no synchronization.
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "ffn_gated.h"
#include "ffn_gated_internal.h"

namespace ffn {
namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxElems = (int64_t)1 << 31;
// A tile's byte offsets from its first row stay below 2^31: 256 rows of 2^20 fp32.
constexpr int kMaxRow = 1 << 20;
constexpr int kMaxRank = 1 << 16;

bool aligned(const void* p, uintptr_t a = 16) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int round_up_to(int v, int a) { return (v + a - 1) / a * a; }
size_t esize(ffn_dtype_t w) { return w == FFN_F32 ? 4 : 2; }
int chunk(ffn_dtype_t w) { return w == FFN_F32 ? 4 : 8; }
bool known(ffn_dtype_t w) { return w == FFN_F32 || w == FFN_BF16; }

int check_shape(int T, int d, int d_ff) {
  if (T < 1 || d < 1 || d_ff < 1 || d > kMaxRow || d_ff > kMaxRow) return FFN_ERR_SHAPE;
  if ((int64_t)d_ff * d >= kMaxElems || (int64_t)T * d >= kMaxElems) return FFN_ERR_SHAPE;
  return FFN_OK;
}
int check_rank(int d, int d_ff, int n, int r) {
  if (n < 1 || r < 1 || r > kMaxRank) return FFN_ERR_SHAPE;
  return (int64_t)r * std::max(d, d_ff) >= kMaxElems ? FFN_ERR_SHAPE : FFN_OK;
}

BlockShape shape_of(ffn_dtype_t w, int T, int d, int d_ff) {
  return BlockShape{T, d, d_ff, round_up_to(d, chunk(w)), round_up_to(d_ff, 64)};
}

// the call's tokens from t0 on, `piece` or fewer, and row t0 of rows of n elements
BlockShape tokens_of(BlockShape s, int64_t t0, int64_t piece) {
  s.T = (int)std::min(piece, s.T - t0);
  return s;
}
const void* rows_from(ffn_dtype_t w, const void* p, int64_t t0, int n) {
  return static_cast<const char*>(p) + t0 * n * (int64_t)esize(w);
}
void* rows_from(ffn_dtype_t w, void* p, int64_t t0, int n) { return static_cast<char*>(p) + t0 * n * (int64_t)esize(w); }

struct Carver {
  char* base;
  size_t off = 0;
  void* take(size_t bytes) {
    void* p = base ? base + off : nullptr;
    off += (bytes + kAlign - 1) / kAlign * kAlign;
    return p;
  }
};

// g, v (fp32) and z of a forward call, [T][ldf] each
struct Save {
  float *g, *v;
  void* z;
};
size_t save_layout(ffn_dtype_t w, int T, int d_ff, void* base, Save* out) {
  const size_t n = (size_t)T * round_up_to(d_ff, 64);
  Carver c{static_cast<char*>(base)};
  Save s;
  s.g = static_cast<float*>(c.take(4 * n));
  s.v = static_cast<float*>(c.take(4 * n));
  s.z = c.take(esize(w) * n);
  if (out) *out = s;
  return c.off;
}

// The regions below grow with T and with rp, so a workspace serves calls of fewer tokens and lower ranks too.
struct ForwardWs {
  void *z, *v[2], *v2, *x, *w_gate, *w_up, *w_down;
  float *part, *shares;
  int32_t* plan;
};
size_t forward_layout(ffn_dtype_t w, const BlockShape& s, int rp, void* base, ForwardWs* out) {
  Carver c{static_cast<char*>(base)};
  ForwardWs f{};
  const size_t e = esize(w);
  f.z = c.take(e * s.T * s.ldf);
  if (rp) {
    for (void*& v : f.v) v = c.take(e * s.T * rp);
    f.v2 = c.take(e * s.T * rp);
    f.plan = static_cast<int32_t*>(c.take(4 * plan_ints(s.T)));
    f.shares = static_cast<float*>(c.take(adapter_share_bytes_most(s.T, rp, 2)));
  }
  f.part = static_cast<float*>(c.take(share_bytes_most(w == FFN_F32, 1, s.T, std::max(s.d, 2 * s.d_ff), true)));
  if (s.dp != s.d) {
    f.x = c.take(e * s.T * s.dp);
    f.w_gate = c.take(e * s.d_ff * s.dp);
    f.w_up = c.take(e * s.d_ff * s.dp);
    f.w_down = c.take(e * s.d_ff * s.dp);
  }
  if (out) *out = f;
  return c.off;
}

struct BackwardWs {
  void *dg, *dv, *x, *dy, *w_gate, *w_up, *w_down;
  float* part;
};
size_t backward_layout(ffn_dtype_t w, const BlockShape& s, void* base, BackwardWs* out) {
  Carver c{static_cast<char*>(base)};
  BackwardWs b{};
  const size_t e = esize(w);
  b.dg = c.take(e * s.T * s.ldf);
  b.dv = c.take(e * s.T * s.ldf);
  // dz and dx, and the weight gradients
  b.part = static_cast<float*>(c.take(std::max(share_bytes_most(w == FFN_F32, 1, s.T, std::max(s.d, s.ldf), true),
                                               share_bytes_most(w == FFN_F32, 3, s.d_ff, s.d, false))));
  if (s.dp != s.d) {
    b.x = c.take(e * s.T * s.dp);
    b.dy = c.take(e * s.T * s.dp);
    b.w_gate = c.take(e * s.d_ff * s.dp);
    b.w_up = c.take(e * s.d_ff * s.dp);
    b.w_down = c.take(e * s.d_ff * s.dp);
  }
  if (out) *out = b;
  return c.off;
}

struct AdapterWs {
  void *v, *x, *w;
  float *part, *shares;
  int32_t* plan;
};
size_t adapter_layout(ffn_dtype_t w, const BlockShape& s, int rp, void* base, AdapterWs* out) {
  Carver c{static_cast<char*>(base)};
  AdapterWs a{};
  const size_t e = esize(w);
  a.v = c.take(e * s.T * rp);
  a.plan = static_cast<int32_t*>(c.take(4 * plan_ints(s.T)));
  a.shares = static_cast<float*>(c.take(adapter_share_bytes_most(s.T, rp, 1)));
  a.part = static_cast<float*>(c.take(share_bytes_most(w == FFN_F32, 1, s.T, s.d_ff, true)));
  if (s.dp != s.d) {
    a.x = c.take(e * s.T * s.dp);
    a.w = c.take(e * s.d_ff * s.dp);
  }
  if (out) *out = a;
  return c.off;
}

int check_form(const ffn_options_t* o, float t, BlockForm* f) {
  *f = BlockForm{FFN_ACT_RELU, 0, t};
  if (!o) return FFN_OK;
  if (o->act != FFN_ACT_RELU && o->act != FFN_ACT_RSPLUS && o->act != FFN_ACT_SILU) return FFN_ERR_OPTION;
  if (o->silu_up != 0 && o->silu_up != 1) return FFN_ERR_OPTION;
  if (o->g_idx || o->g_sign || o->rms_norm || o->rms_gain) return FFN_ERR_OPTION;
  f->act = o->act;
  f->silu_up = o->silu_up;
  return FFN_OK;
}

// The stacks a call may use (the projection call: the gate's alone), checked.
int check_adapters(const ffn_adapters_t* a, ffn_dtype_t w, int d, int d_ff, bool block, AdapterSet* out) {
  if (!a->ids) return FFN_ERR_NULL;
  const void* s[3][2] = {{a->gate_a, a->gate_b}, {a->up_a, a->up_b}, {a->down_a, a->down_b}};
  bool any = false;
  for (const auto& p : s) {
    if ((p[0] == nullptr) != (p[1] == nullptr)) return FFN_ERR_NULL;
    any = any || p[0];
  }
  if (!any || (!block && !a->gate_a)) return FFN_ERR_NULL;
  if (!block && (a->up_a || a->down_a)) return FFN_ERR_OPTION;
  if (const int rc = check_rank(d, d_ff, a->n, a->r)) return rc;
  for (const auto& p : s)
    if (!aligned(p[0]) || !aligned(p[1])) return FFN_ERR_ALIGN;
  if (!aligned(a->ids, 4) || !aligned(a->scale, 4)) return FFN_ERR_ALIGN;
  *out = AdapterSet{a->n, a->r, round_up_to(a->r, chunk(w)), a->ids, a->scale};
  return FFN_OK;
}

// `p` itself, or its rows copied to padded ones
hipError_t padded(bool f32, const BlockShape& s, int64_t rows, const void** p, void* room, hipStream_t st) {
  if (s.dp == s.d) return hipSuccess;
  const hipError_t e = launch_pad_rows(f32, rows, s.d, s.dp, *p, room, st);
  *p = room;
  return e;
}

}  // namespace
}  // namespace ffn

using namespace ffn;

#define FFN_TRY(call)                                  \
  do {                                                 \
    if ((call) != hipSuccess) return FFN_ERR_HIP;      \
  } while (0)

extern "C" {

size_t ffn_gated_save_bytes(ffn_dtype_t wdt, int T, int d_ff) {
  if (!known(wdt) || check_shape(T, 1, d_ff) != FFN_OK) return 0;
  return save_layout(wdt, T, d_ff, nullptr, nullptr);
}

size_t ffn_gated_workspace_bytes(ffn_dtype_t wdt, int T, int d, int d_ff, int r, int backward) {
  if (!known(wdt) || check_shape(T, d, d_ff) != FFN_OK || r < 0 || (r && check_rank(d, d_ff, 1, r) != FFN_OK)) return 0;
  const BlockShape s = shape_of(wdt, T, d, d_ff);
  const size_t f = forward_layout(wdt, s, round_up_to(r, chunk(wdt)), nullptr, nullptr);
  return backward ? std::max(f, backward_layout(wdt, s, nullptr, nullptr)) : f;
}

size_t ffn_adapter_workspace_bytes(ffn_dtype_t wdt, int T, int d, int n_out, int r) {
  if (!known(wdt) || check_shape(T, d, n_out) != FFN_OK || check_rank(d, n_out, 1, r) != FFN_OK) return 0;
  return adapter_layout(wdt, shape_of(wdt, T, d, n_out), round_up_to(r, chunk(wdt)), nullptr, nullptr);
}

int ffn_gated_forward(ffn_dtype_t wdt, int T, int d, int d_ff, const void* x, const void* w_gate, const void* w_up,
                      const void* w_down_t, float t, const ffn_options_t* opt, const ffn_adapters_t* ad, void* y,
                      void* save, size_t save_bytes, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!x || !w_gate || !w_up || !w_down_t || !y || !ws) return FFN_ERR_NULL;
  if (!known(wdt)) return FFN_ERR_DTYPE;
  if (const int rc = check_shape(T, d, d_ff)) return rc;
  if (!aligned(x) || !aligned(w_gate) || !aligned(w_up) || !aligned(w_down_t) || !aligned(y) || !aligned(save) ||
      !aligned(ws))
    return FFN_ERR_ALIGN;
  BlockForm form;
  if (const int rc = check_form(opt, t, &form)) return rc;
  AdapterSet set;
  if (ad) {
    if (save) return FFN_ERR_OPTION;
    if (const int rc = check_adapters(ad, wdt, d, d_ff, true, &set)) return rc;
  }
  const BlockShape s = shape_of(wdt, T, d, d_ff);
  ForwardWs f;
  if (ws_bytes < forward_layout(wdt, s, set.rp, ws, &f)) return FFN_ERR_WORKSPACE;
  Save sv{nullptr, nullptr, f.z};
  if (save && save_bytes < save_layout(wdt, T, d_ff, save, &sv)) return FFN_ERR_WORKSPACE;
  set.plan = f.plan;
  set.part = f.shares;

  const bool f32 = wdt == FFN_F32;
  FFN_TRY(padded(f32, s, T, &x, f.x, stream));
  FFN_TRY(padded(f32, s, d_ff, &w_gate, f.w_gate, stream));
  FFN_TRY(padded(f32, s, d_ff, &w_up, f.w_up, stream));
  FFN_TRY(padded(f32, s, d_ff, &w_down_t, f.w_down, stream));

  const void* b2[2] = {ad ? ad->gate_b : nullptr, ad ? ad->up_b : nullptr};
  const void* v2[2] = {f.v[0], f.v[1]};
  const bool down = ad && ad->down_b;
  const int64_t piece = tokens_a_launch(std::max<int64_t>(d, 2 * (int64_t)d_ff), ad != nullptr);
  for (int64_t t0 = 0; t0 < T; t0 += piece) {
    const BlockShape p = tokens_of(s, t0, piece);
    const void* xp = rows_from(wdt, x, t0, s.dp);
    void* z = rows_from(wdt, sv.z, t0, s.ldf);
    float *g = sv.g ? sv.g + t0 * s.ldf : nullptr, *v = sv.v ? sv.v + t0 * s.ldf : nullptr;
    if (ad) set.ids = ad->ids + t0;
    if (b2[0] || b2[1]) {
      const void* a[2] = {b2[0] ? ad->gate_a : ad->up_a, ad->up_a};
      void* vs[2] = {b2[0] ? f.v[0] : f.v[1], f.v[1]};
      FFN_TRY(launch_adapter_v(f32, p.T, d, s.dp, xp, set, b2[0] && b2[1] ? 2 : 1, a, vs, hidden_plan(f32, p, true).tile, stream));
    }
    const AdapterSet hidden = b2[0] || b2[1] ? set : AdapterSet{};
    FFN_TRY(launch_block_hidden(f32, p, xp, w_gate, w_up, form, hidden, v2, b2, z, g, v, f.part, stream));
    if (down) {
      const void* a[2] = {ad->down_a, nullptr};
      void* vs[2] = {f.v2, nullptr};
      FFN_TRY(launch_adapter_v(f32, p.T, d_ff, s.ldf, z, set, 1, a, vs, token_plan(f32, p.T, d, d_ff, 1, true).tile, stream));
    }
    const TokenProduct q{{z, nullptr}, {w_down_t, nullptr}, 1, p.T, d, d_ff, s.ldf, s.dp, d, rows_from(wdt, y, t0, d),
                         f.part, down ? set : AdapterSet{}, f.v2, down ? ad->down_b : nullptr};
    FFN_TRY(launch_token_product_ks(f32, q, stream));
  }
  return FFN_OK;
}

int ffn_gated_backward(ffn_dtype_t wdt, int T, int d, int d_ff, const void* x, const void* w_gate, const void* w_up,
                       const void* w_down_t, const ffn_options_t* opt, const void* dy, const void* save,
                       size_t save_bytes, void* dx, void* dw_gate, void* dw_up, void* dw_down_t, void* ws,
                       size_t ws_bytes, hipStream_t stream) {
  if (!x || !w_gate || !w_up || !w_down_t || !dy || !save || !ws) return FFN_ERR_NULL;
  if (!dx && !dw_gate && !dw_up && !dw_down_t) return FFN_ERR_NULL;
  if (!known(wdt)) return FFN_ERR_DTYPE;
  if (const int rc = check_shape(T, d, d_ff)) return rc;
  if (!aligned(x) || !aligned(w_gate) || !aligned(w_up) || !aligned(w_down_t) || !aligned(dy) || !aligned(save) ||
      !aligned(dx) || !aligned(dw_gate) || !aligned(dw_up) || !aligned(dw_down_t) || !aligned(ws))
    return FFN_ERR_ALIGN;
  BlockForm form;
  if (const int rc = check_form(opt, 0.f, &form)) return rc;
  const BlockShape s = shape_of(wdt, T, d, d_ff);
  BackwardWs b;
  if (ws_bytes < backward_layout(wdt, s, ws, &b)) return FFN_ERR_WORKSPACE;
  Save sv;
  if (save_bytes < save_layout(wdt, T, d_ff, const_cast<void*>(save), &sv)) return FFN_ERR_WORKSPACE;

  const bool f32 = wdt == FFN_F32, hidden = dx || dw_gate || dw_up;
  if (dw_gate || dw_up) FFN_TRY(padded(f32, s, T, &x, b.x, stream));
  FFN_TRY(padded(f32, s, T, &dy, b.dy, stream));
  if (hidden) {
    FFN_TRY(padded(f32, s, d_ff, &w_down_t, b.w_down, stream));
    FFN_TRY(launch_block_dz(f32, s, dy, w_down_t, form, sv.g, sv.v, b.dg, b.dv, b.part, stream));
  }
  if (dx) {
    FFN_TRY(padded(f32, s, d_ff, &w_gate, b.w_gate, stream));
    FFN_TRY(padded(f32, s, d_ff, &w_up, b.w_up, stream));
    const TokenProduct p{{b.dg, b.dv}, {w_gate, w_up}, 2, T, d, d_ff, s.ldf, s.dp, d, dx, b.part,
                         AdapterSet{}, nullptr, nullptr};
    FFN_TRY(launch_token_product_ks(f32, p, stream));
  }
  const void *wa[3] = {}, *wb[3] = {};
  void* wo[3] = {};
  int n = 0;
  auto want = [&](void* out, const void* a, const void* bb) {
    if (!out) return;
    wa[n] = a;
    wb[n] = bb;
    wo[n++] = out;
  };
  want(dw_gate, b.dg, x);
  want(dw_up, b.dv, x);
  want(dw_down_t, sv.z, dy);
  if (n) FFN_TRY(launch_block_dw(f32, s, n, wa, wb, wo, b.part, stream));
  return FFN_OK;
}

int ffn_adapter_forward(ffn_dtype_t wdt, int T, int d, int n_out, const void* x, const void* w,
                        const ffn_adapters_t* ad, void* y, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!x || !w || !ad || !y || !ws) return FFN_ERR_NULL;
  if (!known(wdt)) return FFN_ERR_DTYPE;
  if (const int rc = check_shape(T, d, n_out)) return rc;
  if (!aligned(x) || !aligned(w) || !aligned(y) || !aligned(ws)) return FFN_ERR_ALIGN;
  AdapterSet set;
  if (const int rc = check_adapters(ad, wdt, d, n_out, false, &set)) return rc;
  const BlockShape s = shape_of(wdt, T, d, n_out);
  AdapterWs a;
  if (ws_bytes < adapter_layout(wdt, s, set.rp, ws, &a)) return FFN_ERR_WORKSPACE;
  set.plan = a.plan;
  set.part = a.shares;
  const bool f32 = wdt == FFN_F32;
  FFN_TRY(padded(f32, s, T, &x, a.x, stream));
  FFN_TRY(padded(f32, s, n_out, &w, a.w, stream));
  const void* aa[2] = {ad->gate_a, nullptr};
  void* v[2] = {a.v, nullptr};
  const int64_t piece = tokens_a_launch(n_out, true);
  for (int64_t t0 = 0; t0 < T; t0 += piece) {
    const BlockShape p = tokens_of(s, t0, piece);
    const void* xp = rows_from(wdt, x, t0, s.dp);
    set.ids = ad->ids + t0;
    FFN_TRY(launch_adapter_v(f32, p.T, d, s.dp, xp, set, 1, aa, v, token_plan(f32, p.T, n_out, d, 1, true).tile, stream));
    const TokenProduct q{{xp, nullptr}, {w, nullptr}, 1, p.T, n_out, d, s.dp, s.dp, n_out, rows_from(wdt, y, t0, n_out),
                         a.part, set, a.v, ad->gate_b};
    FFN_TRY(launch_token_product_kc(f32, q, stream));
  }
  return FFN_OK;
}

}  // extern "C"
