// Host side of include/ffn_group_q.h: argument checks, the choice of tiles, the launches for 64 tokens: the products, before
// them x taken apart (17 tokens and more), behind them a join (windows in shares).  No allocation, no synchronization.
#include <algorithm>

#include "ffn_group_q.h"
#include "ffn_group_q_internal.h"
#include "ffn_step_host.h"

namespace ffn {

// The windows of x that a workgroup's waves take at once (wk u) have to fit in LDS.
GqPlan gq_plan(bool xf32, bool gated, int group, int T, int n_in, int n_out) {
  GqPlan p{};
  p.nt = T == 1 ? 0 : ceil_div(T, 16);
  p.ns = group % kWindow == 0 ? 1 : n_in % kWindow ? 8 : group == 64 ? 2 : group == 32 ? 4 : 8;
  const int windows = ceil_div(n_in, p.nt ? kWindow : 2 * kWindow);
  auto share = [&] {
    const int unit = p.wk * p.u, units = ceil_div(windows, unit);
    p.blocks = ceil_div(n_out, 8 / p.wk * 16);
    // Rows for fewer workgroups than the card holds at once (one to a CU with more than one token tile, else two): the
    // windows in shares, which a second launch joins, where that launch (about 5 us) is little beside the rest: eight
    // rounds of the waves or more, and four to a share.  us without shares, so, and with one round to a share, bf16: 16384 -> 512, 3
    // tokens 13.4, 10.7, 7.3; 28672 -> 2048, one token 13.2, 12.1, 11.8; 4096 -> 1024, 20 tokens 20.0, 11.6, 9.9; 14336 -> 1024, 40
    // tokens 61, 16.4, 16.4; the other way round 14336 -> 4096, 8 tokens 16.7, 18.0, 17.9 (fp32 29, 23, 23).
    const int room = p.nt > 1 ? 256 : 512;
    p.shares = units < 8 ? 1 : std::max(1, std::min({room / p.blocks, units / 4, kGqSharesMost}));
    p.per_share = ceil_div(units, p.shares) * unit;
    p.shares = ceil_div(windows, p.per_share);
    p.chunk = p.per_share;
    return gq_lds(xf32, p, T) <= kGqLds;
  };
  if (p.nt <= 1) {
    // Few tokens: all workgroups at once on the card, two to a CU, rather than rounds of them.
    const int tiles = ceil_div(n_out, 16);
    p.wk = tiles <= 512 ? 8 : tiles <= 1024 ? 4 : 2;
    p.u = p.nt ? gq_batch(gated, p.ns) : 1;
    p.whole = share();
    if (p.whole) return p;
    if (!p.nt) {
      const int unit = p.wk * p.u;
      p.chunk = unit;
      while (true) {
        p.chunk += unit;
        if (gq_lds(xf32, p, 1) > kGqLds) break;
      }
      p.chunk -= unit;
      return p;
    }
  }
  p.u = 1;
  if (p.nt > 1) {
    p.wk = kGqWaves;
    share();
    p.chunk = p.wk;
  } else {
    // pieces of x that the threads hold while they are on their way: windows that they have room for
    const int most = 512 * gq_units(xf32) / (T * (kWindow / 8));
    p.wk = most >= 8 ? 8 : 4;
    share();
    p.chunk = most / p.wk * p.wk;
  }
  return p;
}

namespace {

int check_gq_shape(int T, int n_in, int n_out) {
  if (T < 1 || n_in < 1 || n_out < 1 || n_in > 1 << 20 || n_out > 1 << 20) return FFN_ERR_SHAPE;
  if ((int64_t)T * n_in >= kMaxElems || (int64_t)T * n_out >= kMaxElems || (int64_t)n_in * n_out >= kMaxElems) return FFN_ERR_SHAPE;
  return FFN_OK;
}
// Rows of partial sums a token and matrix, shares x n_out at most whatever T: gq_plan makes shares only of rows for half the
// card's workgroups or fewer (512 of 32 rows at most, or 256 of 64), and no more of them than fill it.
constexpr size_t kGqShareRows = 512 * 32;
size_t gq_share_rows(int n_out) {
  return 2 * (size_t)n_out <= kGqShareRows ? std::min(kGqSharesMost * (size_t)n_out, kGqShareRows) : 0;
}
// A pass's shares, and x in parts with the table of its sums: every region grows with T.
struct GqWs {
  float* part;
  uint4* planes;
  float* sums;
  size_t bytes;
};
GqWs gq_layout(int T, int n_in, int n_out, bool gated, void* base) {
  const size_t tokens = std::min(T, kGqTokens), columns = (size_t)ceil_div(n_in, kGqWaves * kWindow) * kGqWaves * kWindow;
  Carver c{static_cast<char*>(base)};
  GqWs w;
  w.part = static_cast<float*>(c.take(sizeof(float) * (gated ? 2 : 1) * tokens * gq_share_rows(n_out)));
  w.planes = static_cast<uint4*>(c.take(3 * 2 * ceil_div<size_t>(tokens, 16) * 16 * columns));
  w.sums = static_cast<float*>(c.take(sizeof(float) * columns / 32 * kGqTokens));
  w.bytes = c.off;
  return w;
}
int check_matrix(const ffn_group_q_t* w, int n_in) {
  if (!w->codes || !w->scales) return FFN_ERR_NULL;
  if (!known(w->sdt)) return FFN_ERR_DTYPE;
  if (w->group < 32 || w->group % 32 || n_in % w->group) return FFN_ERR_SHAPE;
  if (!aligned(w->codes) || !aligned(w->scales) || !aligned(w->offsets)) return FFN_ERR_ALIGN;
  return FFN_OK;
}

int gq_call(ffn_dtype_t xdt, int T, int n_in, int n_out, const void* x, const ffn_group_q_t* w, const ffn_group_q_t* w2,
            const ActForm& form, void* y, void* ws, size_t ws_bytes, hipStream_t st) {
  if (!x || !w || !y || !ws) return FFN_ERR_NULL;
  if (!known(xdt)) return FFN_ERR_DTYPE;
  if (const int rc = check_gq_shape(T, n_in, n_out)) return rc;
  if (!aligned(x) || !aligned(y) || !aligned(ws)) return FFN_ERR_ALIGN;
  if (const int rc = check_matrix(w, n_in)) return rc;
  if (w2) {
    if (const int rc = check_matrix(w2, n_in)) return rc;
    if (w->sdt != w2->sdt || w->group != w2->group || (w->offsets != nullptr) != (w2->offsets != nullptr)) return FFN_ERR_OPTION;
  }
  if (ws_bytes < ffn_group_q_workspace_bytes(T, n_in, n_out, w2 != nullptr)) return FFN_ERR_WORKSPACE;
  const bool xf32 = xdt == FFN_F32, sf32 = w->sdt == FFN_F32;
  const size_t xs = xf32 ? 4 : 2;
  for (int t0 = 0; t0 < T; t0 += kGqTokens) {
    GqArgs a{};
    a.T = std::min(kGqTokens, T - t0);
    const GqPlan p = gq_plan(xf32, w2 != nullptr, w->group, a.T, n_in, n_out);
    a.n_in = n_in;
    a.n_out = n_out;
    a.windows = ceil_div(n_in, p.nt ? kWindow : 2 * kWindow);
    a.per_share = p.per_share;
    a.chunk = p.chunk;
    a.div_group = (uint32_t)(((uint64_t)1 << 31) / (w->group / 32) + 1);
    a.groups = n_in / w->group;
    a.x = static_cast<const char*>(x) + (size_t)t0 * n_in * xs;
    a.w[0] = GqMatrix{w->codes, w->scales, w->offsets};
    if (w2) a.w[1] = GqMatrix{w2->codes, w2->scales, w2->offsets};
    a.act = form.act;
    a.silu_up = form.silu_up;
    a.t = form.t;
    a.y = static_cast<char*>(y) + (size_t)t0 * n_out * xs;
    const GqWs room = gq_layout(T, n_in, n_out, w2 != nullptr, ws);
    a.part = p.shares > 1 ? room.part : nullptr;
    a.planes = room.planes;
    a.sums = room.sums;
    const hipError_t e = (xf32 ? launch_group_q_f32 : launch_group_q_bf16)(sf32, w2 != nullptr, a, p, st);
    if (e != hipSuccess) return FFN_ERR_HIP;
  }
  return FFN_OK;
}

}  // namespace
}  // namespace ffn

using namespace ffn;

extern "C" {

size_t ffn_group_q_workspace_bytes(int T, int n_in, int n_out, int gated) {
  if (check_gq_shape(T, n_in, n_out) != FFN_OK || (gated != 0 && gated != 1)) return 0;
  return gq_layout(T, n_in, n_out, gated != 0, nullptr).bytes;
}

int ffn_group_q_forward(ffn_dtype_t xdt, int T, int n_in, int n_out, const void* x, const ffn_group_q_t* w, void* y,
                        void* ws, size_t ws_bytes, hipStream_t stream) {
  return gq_call(xdt, T, n_in, n_out, x, w, nullptr, ActForm{}, y, ws, ws_bytes, stream);
}

int ffn_group_q_gated_forward(ffn_dtype_t xdt, int T, int n_in, int n_out, const void* x, const ffn_group_q_t* w_gate,
                              const ffn_group_q_t* w_up, float t, const ffn_options_t* opt, void* z, void* ws,
                              size_t ws_bytes, hipStream_t stream) {
  if (!w_up) return FFN_ERR_NULL;
  ActForm form;
  const int rc = check_act(opt, t, &form);
  if (rc) return rc;
  return gq_call(xdt, T, n_in, n_out, x, w_gate, w_up, form, z, ws, ws_bytes, stream);
}

}  // extern "C"
