// include/ffn_moe.h: a mixture-of-experts layer for a decode step's tokens.
//
// The chosen experts' three matrices bound it: each is read once for every 16, 32 or 64 of its expert's tokens, by the mean number of
// them (launch_moe).  Launches:
//   1. k_moe_logits  the router's products in 64 bits, a wave to an expert
//      k_moe_choose  the choice, a wave to a token; up to 4 tokens' is made by every workgroup of k_moe_hidden instead (a
//                    launch less)
//   2. k_moe_hidden  z = A(x W1^T - t) U(x W3^T), 16 hidden neurons of an expert to a workgroup
//   3. k_moe_down    z W2 in pieces of neurons, 16-byte columns x 16 lanes of an expert to a workgroup
//   4. k_moe_join    the pieces and the experts, weighted, in a fixed order
// The matrix products have tokens as the A operand and weights as the B operand, so that one token costs
// what 16 do; the weights go from memory to registers and enter as they lie (W1, W3: rows along the summed
// dimension) or after an exchange of half-words in the lane (W2's rows are neurons: 8 of them, 8 columns each).
#include <math.h>

#include <algorithm>

#include "ffn_mfma.h"
#include "ffn_moe.h"
#include "ffn_moe_internal.h"
#include "ffn_step_device.h"

namespace ffn {
namespace {

constexpr int kMoeTokens = 256, kMoeK = 16, kMoeExperts = 512;
// Workgroups of k_moe_down, where the neurons go in pieces to come to so many (bf16: 8 experts of 4096 x 14336, 16 tokens, 458 us with
// 256, 434 to 440 with 512 to 4096; 64 of 2048 x 1408, 64 tokens, 198 with 256 to 1024, 203 and 208 with 2048 and 4096).
constexpr int kDownGroups = 1024;
constexpr int kRouteTokens = 8;  // tokens of a wave that computes logits
// Tokens that k_moe_hidden chooses for itself, a wave each (64 experts of 2048 x 256 bf16, one token: a launch of its own 24.3 us, so
// 22.3; four tokens 32.8 and 30.9, of 512 experts 38.2 and 38.1).
constexpr int kChooseTokens = 4;

struct RouteArgs {
  int T, d, E, k;
  const void *x, *w;
  const float* bias;
  int sigmoid, normalize;
  float scale;
  double* logits;  // [T][E]
  int32_t* ids;
  float* weights;
};

struct MoeArgs {
  int T, d, d_ff, E, k, ldz;
  int slots;   // T k places (each place's first use of its expert works), or the experts
  int pieces;  // of the neurons, in k_moe_down
  const void *x, *w[3];
  ActForm form;
  const int32_t* ids;
  const float* weights;
  void* z;      // [T k][ldz], with bf16 twice: the values, and behind them what their rounding leaves
  size_t z_plane;
  float* part;  // [pieces][T k][d]
  void* y;
};

// A 16-byte chunk's worth of elements from element i on, `left` of them there: one load, or narrower ones.  VEC: 2, rows are
// whole lines of 128 bytes (weights are streamed past the caches); 1, whole chunks; 3, rows start at whole dwords, which
// is all that a 16-byte load needs, but end inside a chunk; 0, bf16 rows of odd length.
template <bool F32, int VEC, bool WEIGHTS = false>
__device__ __forceinline__ uint4 ld_chunk(const Buf& b, uint32_t i, int left) {
  if constexpr (VEC == 3) {
    if (left >= (F32 ? 4 : 8)) return ldb(b, i * (F32 ? 4u : 2u));
    return ld_chunk<F32, 0>(b, i, left);
  } else if constexpr (VEC) {
    const uint32_t o = left > 0 ? i * (F32 ? 4u : 2u) : kOOB;
    return WEIGHTS && VEC == 2 ? ldb_nt(b, o) : ldb(b, o);
  } else if constexpr (F32) {
    return make_uint4(ldb32(b, left > 0 ? i * 4 : kOOB), ldb32(b, left > 1 ? i * 4 + 4 : kOOB),
                      ldb32(b, left > 2 ? i * 4 + 8 : kOOB), ldb32(b, left > 3 ? i * 4 + 12 : kOOB));
  } else {
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, left > j ? i * 2 + j * 2 : kOOB, 0, 0);
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}
// ------------------------------------------------------------------ the router
template <int CTRL>
__device__ __forceinline__ double dpp_move64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double lane64(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)u, lane), hi = __builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// every lane's v joined, as group_sum joins floats
template <class F>
__device__ __forceinline__ double wave_join64(double v, const F& f) {
  v = f(v, dpp_move64<kDppXor1>(v));
  v = f(v, dpp_move64<kDppXor2>(v));
  v = f(v, dpp_move64<kDppHalfMirror>(v));
  v = f(v, dpp_move64<kDppMirror>(v));
  return f(f(lane64(v, 0), lane64(v, 16)), f(lane64(v, 32), lane64(v, 48)));
}
__device__ __forceinline__ double wave_sum64(double v) {
  return wave_join64(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double wave_max64(double v) {
  return wave_join64(v, [](double a, double b) { return b > a ? b : a; });
}

// The choice of one token, by one wave: k of lanes 0 ... k - 1.  A lane has the scores of experts lane, 64 + lane, ...
// (N of them).
struct Chosen {
  int id;
  float weight;
};
template <int N>
__device__ __forceinline__ Chosen choose_of(const RouteArgs& a, int tok) {
  const int lane = lane_id();
  double score[N], key[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * kWave + lane;
    score[i] = e < a.E ? a.logits[(size_t)tok * a.E + e] : -INFINITY;
    key[i] = score[i];
  }
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < N; ++i) score[i] = 1.0 / (1.0 + exp(-score[i]));
  } else {
    double top = -INFINITY, total = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = score[i] > top ? score[i] : top;
    top = wave_max64(top);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      score[i] = exp(score[i] - top);
      total += i * kWave + lane < a.E ? score[i] : 0.0;
    }
    total = wave_sum64(total);
#pragma unroll
    for (int i = 0; i < N; ++i) score[i] /= total;
  }
  uint32_t open = 0;  // experts of this lane that are not chosen yet
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = i * kWave + lane;
    if (e >= a.E) continue;
    if (a.bias) key[i] = score[i] + (double)a.bias[e];
    key[i] = key[i] == key[i] ? key[i] : -INFINITY;
    open |= 1u << i;
  }
  double sum = 0.0, mine = 0.0;
  int mine_e = 0;
  for (int j = 0; j < a.k; ++j) {
    double best = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) best = (open >> i & 1) && key[i] > best ? key[i] : best;
    best = wave_max64(best);
    // the lowest of the open experts that have it
    int at = -1, from = 0;
#pragma unroll
    for (int i = N - 1; i >= 0; --i) {
      const uint64_t m = __ballot((open >> i & 1) && key[i] == best);
      at = m ? i : at;
      from = m ? __builtin_ctzll(m) : from;
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i == at) s = lane64(score[i], from);
    if (lane == from) open &= ~(1u << at);
    sum += s;
    if (lane == j) {
      mine = s;
      mine_e = at * kWave + from;
    }
  }
  return Chosen{mine_e, (float)((double)a.scale * (a.normalize ? mine / sum : mine))};
}
__device__ __forceinline__ Chosen choose(const RouteArgs& a, int tok) {
  if (a.E <= kWave) return choose_of<1>(a, tok);
  if (a.E <= 2 * kWave) return choose_of<2>(a, tok);
  return choose_of<kMoeExperts / kWave>(a, tok);
}
__device__ __forceinline__ void put_choice(const RouteArgs& a, int tok, const Chosen& c) {
  if (lane_id() < a.k) {
    a.ids[(size_t)tok * a.k + lane_id()] = c.id;
    a.weights[(size_t)tok * a.k + lane_id()] = c.weight;
  }
}
__global__ __launch_bounds__(64) void k_moe_choose(RouteArgs a) { put_choice(a, blockIdx.x, choose(a, blockIdx.x)); }

// A wave takes one expert's logits of NT tokens.  Latency: 64 experts of 2048, one token 2.8 us, 64 tokens 4.6.
template <bool F32, int VEC, int NT>
__global__ __launch_bounds__(256) void k_moe_logits(RouteArgs a) {
  constexpr int E = F32 ? 4 : 8;
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), e = blockIdx.x * 4 + wave, t0 = blockIdx.y * NT;
  const int nt = min(a.T - t0, NT);
  if (e >= a.E) return;
  {
    const size_t es = F32 ? 4 : 2;
    const Buf wb = make_buf(static_cast<const char*>(a.w) + (size_t)e * a.d * es, a.d * (uint32_t)es);
    const Buf xb = make_buf(static_cast<const char*>(a.x) + (size_t)t0 * a.d * es, nt * a.d * (uint32_t)es);
    // U chunks' loads at once; the same order of additions whatever NT
    constexpr int U = VEC ? (NT == 1 ? 4 : 2) : 1;
    double s[NT] = {};
    for (int k0 = lane * E; k0 < a.d; k0 += U * kWave * E) {
      uint4 wv[U], xv[U][NT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + u * kWave * E;
        wv[u] = ld_chunk<F32, VEC>(wb, k, a.d - k);
#pragma unroll
        for (int t = 0; t < NT; ++t) xv[u][t] = ld_chunk<F32, VEC>(xb, t * a.d + k, t < nt ? a.d - k : 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float w[E], x[E];
        if constexpr (F32) unpack(WF32{}, wv[u], w);
        else unpack(WBf16{}, wv[u], w);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if constexpr (F32) unpack(WF32{}, xv[u][t], x);
          else unpack(WBf16{}, xv[u][t], x);
#pragma unroll
          for (int j = 0; j < E; ++j) s[t] = fma((double)w[j], (double)x[j], s[t]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const double v = wave_sum64(s[t]);
      if (lane == 0 && t < nt) a.logits[(size_t)(t0 + t) * a.E + e] = v;
    }
  }
}

// ------------------------------------------------------------------ the experts
// The expert of a slot, or -1.  With a slot a place, a place whose expert an earlier one names has no work.
__device__ __forceinline__ int slot_expert(const MoeArgs& a, const int32_t* ids, int slot) {
  if (a.slots == a.E && a.slots != a.T * a.k) return slot;
  const int e = uniform(ids[slot]);
  if (e < 0 || e >= a.E) return -1;
  for (int b = 0; b < slot; b += kWave) {
    const int at = b + lane_id();
    if (__ballot(at < slot && ids[at] == e)) return -1;
  }
  return e;
}
// The places of expert e, in order, into list; every wave calls it and gets their number.
__device__ __forceinline__ int list_places(const MoeArgs& a, const int32_t* ids, int e, uint16_t* list, int* count) {
  if (threadIdx.x < kWave) {
    const int n = a.T * a.k;
    int have = 0;
    for (int b = 0; b < n; b += 8 * kWave) {
      int id[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = b + j * kWave + lane_id();
        id[j] = at < n ? ids[at] : -1;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint64_t m = __ballot(id[j] == e);
        if (id[j] == e) list[have + rank_in_mask(m)] = (uint16_t)(b + j * kWave + lane_id());
        have += __popcll(m);
      }
    }
    if (lane_id() == 0) *count = have;
  }
  __syncthreads();
  return uniform(*count);
}

// Lanes 8 apart exchange halves: a keeps its own in lanes n < 8 and gets b's of lane n - 8 in the others; b the other way round.
__device__ __forceinline__ void exchange8(uint4& a, uint4& b) {
  auto one = [](uint32_t& x, uint32_t& y) {  // 0x128: row_ror:8, written in the upper or the lower 8 lanes of each 16
    const uint32_t u = __builtin_amdgcn_update_dpp((int)x, (int)y, 0x128, 0xF, 0xC, false);
    y = __builtin_amdgcn_update_dpp((int)y, (int)x, 0x128, 0xF, 0x3, false);
    x = u;
  };
  one(a.x, b.x);
  one(a.y, b.y);
  one(a.z, b.z);
  one(a.w, b.w);
}

// One value of z: fp32, or with bf16 weights two bf16 parts that hold 16 of its bits, a plane each.  Rounded to one part, z would
// put as much error into y as y's own rounding does (2.3e-3 of its norm, so 1.65e-3), and the second product, which the weights'
// bytes bound, has room for both parts: 8 experts of 4096 x 14336, 16 tokens 433 us, so 441; 64 of 2048 x 1408, one token 34.7 and 34.9,
// 64 tokens 198 and 203, 256 tokens 322 and 336.  An Inf or NaN has no second part.
template <bool F32>
__device__ __forceinline__ void put_z(const MoeArgs& a, size_t i, float v) {
  store_as<F32>(a.z, i, v);
  if constexpr (!F32) {
    const float hi = bf_to_f(f_to_bf(v));
    static_cast<uint16_t*>(a.z)[a.z_plane + i] = f_to_bf(hi - hi == 0.f ? v - hi : 0.f);
  }
}

// Four waves share the summed dimension of 16 hidden neurons' two rows.  NT: 16-token tiles at a time.  CHOOSE: the
// tokens' choice is made here, from the logits.  Bound by the weights' bytes: 8 experts of 4096 x 14336, 16 tokens 1.88 GB in
// 272 us (6.9 TB/s); 64 of 2048 x 1408, 64 tokens 738 MB in 121 us (6.1); 8 of 64, 2048 x 1024, one token 67 MB in 17 us, of
// which the choice and the first loads are about 7.
template <bool F32, int VEC, int NT, bool CHOOSE>
__global__ __launch_bounds__(256) void k_moe_hidden(MoeArgs a, RouteArgs route) {
  constexpr int E = F32 ? 4 : 8, U = 4, STEP = 4 * E * U;  // elements of a row that a wave takes at once
  __shared__ uint16_t list[CHOOSE ? kChooseTokens * kMoeK : kMoeTokens * kMoeK];
  __shared__ float red[4][2][4][kWave];
  __shared__ int32_t chosen[CHOOSE ? kChooseTokens * kMoeK : 1];
  __shared__ int count;
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int32_t* ids = a.ids;
  if constexpr (CHOOSE) {
    if (wave < a.T) {
      const Chosen c = choose(route, wave);
      if (lane < a.k) chosen[wave * a.k + lane] = c.id;
      if (blockIdx.x == 0 && blockIdx.y == 0) put_choice(route, wave, c);
    }
    __syncthreads();
    ids = chosen;
  }
  const int e = slot_expert(a, ids, blockIdx.y);
  if (e < 0) return;
  const int row0 = blockIdx.x * 16, rows = min(16, a.d_ff - row0);
  const size_t es = F32 ? 4 : 2;
  Buf wb[2];
#pragma unroll
  for (int m = 0; m < 2; ++m)
    wb[m] = make_buf(static_cast<const char*>(a.w[m]) + ((size_t)e * a.d_ff + (rows > 0 ? row0 : 0)) * a.d * es,
                     rows > 0 ? (uint32_t)(rows * a.d * es) : 0u);
  const Buf xb = make_buf(a.x, (uint32_t)a.T * a.d * es);
  // A load takes whole lines, 128 bytes of 8 rows, streamed past the caches where the rows are whole lines (7.0 TB/s over 1.9
  // GB; 16 rows of 64 bytes, as the operands have them, 6.3 through the caches and less past them): lane (n, g) has chunk
  // g + 4 (n / 8) of row n % 8, and of row n % 8 + 8 in a second load.  The operands' lanes (n, g) want row n's chunks g and
  // 4 + g: lanes 8 apart exchange halves.  Columns behind a row's end are zeros; rows behind the last are behind the buffer.
  uint4 w[U][2];
  auto load = [&](int k0) {
    if (k0 >= a.d) return;
    const bool tail = k0 + STEP > a.d;
#pragma unroll
    for (int q = 0; q < U; q += 2) {
      const int k = k0 + (q * 4 + g + (n >> 3) * 4) * E, left = tail ? a.d - k : E;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = (n & 7) + 8 * h;
          w[q + h][m] = ld_chunk<F32, VEC, true>(wb[m], (uint32_t)r * a.d + k, (VEC && VEC != 3) || r < rows ? left : 0);
        }
    }
  };
  // The workgroups go through the rows from different places on: with rows of 2^n bytes all of them would be on the
  // same few memory channels at any time (rows of 4096 bytes: 4.3 TB/s, so 5.25).
  const int turns = (a.d + 4 * STEP - 1) / (4 * STEP), start = (int)((blockIdx.x * 5 + (blockIdx.x >> 3)) % (uint32_t)turns);
  load((start * 4 + wave) * STEP);
  const int cnt = list_places(a, ids, e, list, &count);

  for (int p0 = 0; p0 < cnt; p0 += 16 * NT) {
    uint32_t xo[NT];  // a token's row: tokens past the last one repeat it, and are not stored
#pragma unroll
    for (int t = 0; t < NT; ++t) xo[t] = (uint32_t)(list[min(p0 + t * 16 + n, cnt - 1)] / a.k) * a.d;
    const int tiles = min(NT, (cnt - p0 + 15) / 16);
    f32x4_t acc[NT][2] = {};
    int turn = start;
    if (p0) load((start * 4 + wave) * STEP);
    for (int i = 0; i < turns; ++i) {
      const int k0 = (turn * 4 + wave) * STEP;
      turn = turn + 1 == turns ? 0 : turn + 1;
      // 8 loads of weights in flight, and three or more other waves of the SIMD at theirs
      if (k0 < a.d) {
        const bool tail = k0 + STEP > a.d;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t >= tiles) break;
          uint4 x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int k = k0 + (u * 4 + g) * E;
            x[u] = ld_chunk<F32, VEC>(xb, xo[t] + k, tail ? a.d - k : E);
          }
          if (t == 0) {
#pragma unroll
            for (int q = 0; q < U; q += 2)
#pragma unroll
              for (int m = 0; m < 2; ++m) exchange8(w[q][m], w[q + 1][m]);
          }
          f32x4_t s[2] = {};
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              if constexpr (F32) {
                s[m] = mfma16f(comp<0>(x[u]), comp<0>(w[u][m]), s[m]);
                s[m] = mfma16f(comp<1>(x[u]), comp<1>(w[u][m]), s[m]);
                s[m] = mfma16f(comp<2>(x[u]), comp<2>(w[u][m]), s[m]);
                s[m] = mfma16f(comp<3>(x[u]), comp<3>(w[u][m]), s[m]);
              } else {
                s[m] = mfma16(bf8(x[u]), bf8(w[u][m]), s[m]);
              }
            }
          acc[t][0] += s[0];
          acc[t][1] += s[1];
        }
      }
      if (i + 1 < turns) load((turn * 4 + wave) * STEP);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t >= tiles) break;
      __syncthreads();
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][m][i][lane] = acc[t][m][i];
      __syncthreads();
      const int p = p0 + t * 16 + g * 4 + wave, row = row0 + n;  // thread (wave, lane): result register `wave` of `lane`
      if (p < cnt) {
        float h = 0.f, v = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          h += red[w][0][wave][lane];
          v += red[w][1][wave][lane];
        }
        // rows up to ldz are zeros for the next product
        put_z<F32>(a, (size_t)list[p] * a.ldz + row, row < a.d_ff ? act_product(a.form, h, v) : 0.f);
      }
    }
  }
}

// Columns of a workgroup: 16 lanes of 16 bytes.
template <bool F32>
constexpr int down_columns() {
  return F32 ? 64 : 128;
}

// Four waves take turns at the piece's neurons, 32 at once: a lane has 16 bytes of 8 neurons' rows.  Bound by the weights'
// bytes, rows of 256 bytes at a time: 939 MB in 149 us (6.3 TB/s), 369 in 59-74, 34 in 9.5 (the calls named at k_moe_hidden).
// Where rows end inside a chunk (VEC 3 and 0) the narrow loads of a row's end are in every workgroup's loop, and the kernels
// spill, 63 to 73 registers with one tile of bf16: 52 tokens, 16 experts of 1728 x 6272 243 us, of 1716 325, of 1715 775.
template <bool F32, int VEC, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 4 : 2) void k_moe_down(MoeArgs a) {
  constexpr int E = F32 ? 4 : 8, COLS = down_columns<F32>();
  __shared__ uint16_t list[kMoeTokens * kMoeK];
  __shared__ float red[4][4][4][kWave];
  __shared__ int count;
  const int e = slot_expert(a, a.ids, blockIdx.y);
  if (e < 0) return;
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int col = blockIdx.x * COLS + n * E;
  // the piece's neurons: whole steps of 32
  const int steps = a.ldz / 32, s0 = (int)((int64_t)steps * blockIdx.z / a.pieces), s1 = (int)((int64_t)steps * (blockIdx.z + 1) / a.pieces);
  const size_t es = F32 ? 4 : 2;
  const Buf zb = make_buf(a.z, (uint32_t)(a.T * a.k * a.ldz) * 4u);  // fp32, or two planes of bf16
  const uint32_t vo = col < a.d ? (uint32_t)((g * 8 * (size_t)a.d + col) * es) : kOOB;
  const char* wbase = static_cast<const char*>(a.w[2]) + (size_t)e * a.d_ff * a.d * es;

  uint4 w[8];
  auto load = [&](int s) {
    if (s >= s1) return;
    // rows behind the last are behind the buffer
    const int rows = min(32, a.d_ff - s * 32);
    const Buf wb = make_buf(wbase + (size_t)s * 32 * a.d * es, rows > 0 ? (uint32_t)(rows * a.d * es) : 0u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // the whole offset in the lane's: a wave's own, behind the buffer's end, is no part of the bounds that are checked
      if constexpr (VEC == 1 || VEC == 2) w[j] = ldb_nt(wb, vo + (uint32_t)(j * a.d * es));
      else w[j] = ld_chunk<F32, VEC>(wb, (uint32_t)(g * 8 + j) * a.d + col, g * 8 + j < rows ? a.d - col : 0);
    }
  };
  load(s0 + wave);
  const int cnt = list_places(a, a.ids, e, list, &count);

  for (int p0 = 0; p0 < cnt; p0 += 16 * NT) {
    uint32_t zo[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) zo[t] = (uint32_t)list[min(p0 + t * 16 + n, cnt - 1)] * a.ldz;
    const int tiles = min(NT, (cnt - p0 + 15) / 16);
    f32x4_t acc[NT][E] = {};
    if (p0) load(s0 + wave);
    for (int s = s0 + wave; s < s1; s += 4) {
      uint4 b[E];
      if constexpr (!F32) {
        // column 2q (and 2q + 1) of neurons 2p, 2p + 1: the low (high) halves of dword q of both rows
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t lo[4], hi[4];
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint4 &r0 = w[2 * p], &r1 = w[2 * p + 1];
            const uint32_t d0 = q == 0 ? r0.x : q == 1 ? r0.y : q == 2 ? r0.z : r0.w;
            const uint32_t d1 = q == 0 ? r1.x : q == 1 ? r1.y : q == 2 ? r1.z : r1.w;
            lo[p] = __builtin_amdgcn_perm(d1, d0, 0x05040100u);
            hi[p] = __builtin_amdgcn_perm(d1, d0, 0x07060302u);
          }
          b[2 * q] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          b[2 * q + 1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (t >= tiles) break;
        const uint32_t zi = (zo[t] + s * 32 + g * 8) * (uint32_t)es;
        const uint4 z0 = ldb(zb, zi);
        if constexpr (F32) {
          const uint4 z1 = ldb(zb, zi + 16);
          const float z[8] = {comp<0>(z0), comp<1>(z0), comp<2>(z0), comp<3>(z0), comp<0>(z1), comp<1>(z1), comp<2>(z1), comp<3>(z1)};
          f32x4_t sum[E] = {};
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sum[0] = mfma16f(z[j], comp<0>(w[j]), sum[0]);
            sum[1] = mfma16f(z[j], comp<1>(w[j]), sum[1]);
            sum[2] = mfma16f(z[j], comp<2>(w[j]), sum[2]);
            sum[3] = mfma16f(z[j], comp<3>(w[j]), sum[3]);
          }
#pragma unroll
          for (int c = 0; c < E; ++c) acc[t][c] += sum[c];
        } else {
          const uint4 z1 = ldb(zb, zi + (uint32_t)a.z_plane * 2u);
#pragma unroll
          for (int c = 0; c < E; ++c) acc[t][c] = mfma16(bf8(z0), bf8(b[c]), mfma16(bf8(z1), bf8(b[c]), acc[t][c]));
        }
      }
      load(s + 4);
    }
    // The waves' sums joined, four of a lane's columns at a time; neighbouring threads have neighbouring columns
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t >= tiles) break;
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) red[wave][c][i][lane] = acc[t][h * 4 + c][i];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = threadIdx.x & 3, l16 = threadIdx.x >> 2 & 15, tok = j * 4 + wave;
          const int p = p0 + t * 16 + tok, at = blockIdx.x * COLS + l16 * E + h * 4 + c;
          if (p >= cnt || at >= a.d) continue;
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) v += red[w][c][tok & 3][(tok >> 2) * 16 + l16];
          a.part[((size_t)blockIdx.z * a.T * a.k + list[p]) * a.d + at] = v;
        }
      }
    }
  }
}

// 64 columns of a token to a workgroup; four waves take turns at its places' pieces.  4 to 5 us, latency.
template <bool F32>
__global__ __launch_bounds__(256) void k_moe_join(MoeArgs a) {
  __shared__ float red[4][kWave];
  const int t = blockIdx.y, wave = uniform(threadIdx.x >> 6), lane = lane_id(), c = blockIdx.x * kWave + lane;
  const size_t rows = (size_t)a.T * a.k;
  float y = 0.f;
  for (int j = wave; j < a.k; j += 4) {
    const int p = t * a.k + j, e = uniform(a.ids[p]);
    if (e < 0 || e >= a.E || c >= a.d) continue;
    const float w = a.weights[p];
    float v[kMoePieces];
#pragma unroll
    for (int s = 0; s < kMoePieces; ++s) v[s] = s < a.pieces ? a.part[(s * rows + p) * a.d + c] : 0.f;
#pragma unroll
    for (int s = 1; s < kMoePieces; ++s) v[0] += v[s];
    y += w * v[0];
  }
  red[wave][lane] = y;
  __syncthreads();
  if (wave == 0 && c < a.d) store_as<F32>(a.y, (size_t)t * a.d + c, (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]));
}

// ------------------------------------------------------------------ host side
struct MoeWs {
  double* logits;
  void* z;
  float* part;
};
size_t moe_layout(bool f32, int T, int d, int d_ff, int E, int k, void* base, MoeWs* out) {
  Carver c{static_cast<char*>(base)};
  MoeWs w;
  w.logits = static_cast<double*>(c.take(sizeof(double) * T * E));
  w.z = c.take(sizeof(float) * T * k * (size_t)moe_ldz(d_ff));
  w.part = static_cast<float*>(c.take(sizeof(float) * moe_part_rows(f32, T, d, d_ff, E, k) * (size_t)d));
  if (out) *out = w;
  return c.off;
}

int check_moe_shape(int T, int d, int d_ff, int E, int k) {
  if (T < 1 || d < 1 || d_ff < 1 || T > kMoeTokens || d > 1 << 20 || d_ff > 1 << 20) return FFN_ERR_SHAPE;
  if ((int64_t)d_ff * d >= kMaxElems) return FFN_ERR_SHAPE;
  if (E < 1 || E > kMoeExperts || k < 1 || k > kMoeK || k > E) return FFN_ERR_SHAPE;
  // z is read through one buffer of less than 2^31 bytes
  if ((int64_t)T * k * moe_ldz(d_ff) >= kMaxElems / 4) return FFN_ERR_SHAPE;
  return FFN_OK;
}

template <bool F32, int VEC, int NT, bool CHOOSE>
hipError_t launch_hidden(const RouteArgs& r, const MoeArgs& a, hipStream_t st) {
  k_moe_hidden<F32, VEC, NT, CHOOSE><<<dim3(a.ldz / 16, a.slots), 256, 0, st>>>(a, r);
  return hipGetLastError();
}
template <bool F32, int VEC, int NT>
hipError_t launch_experts(const RouteArgs& r, const MoeArgs& a, bool choose, hipStream_t st) {
  hipError_t e;
  if constexpr (NT == 1) e = choose ? launch_hidden<F32, VEC, 1, true>(r, a, st) : launch_hidden<F32, VEC, 1, false>(r, a, st);
  else e = launch_hidden<F32, VEC, NT, false>(r, a, st);
  if (e != hipSuccess) return e;
  k_moe_down<F32, VEC, NT><<<dim3(ceil_div(a.d, down_columns<F32>()), a.slots, a.pieces), 256, 0, st>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_moe_join<F32><<<dim3(ceil_div(a.d, kWave), a.T), 256, 0, st>>>(a);
  return hipGetLastError();
}
template <bool F32, int VEC>
hipError_t launch_moe(const RouteArgs& r, const MoeArgs& a, hipStream_t st) {
  const bool choose = r.w && a.T <= kChooseTokens;
  if (r.w) {
    // Waves of one token while there are few of them: 8 tokens of a wave save its expert's row 7 times, one after the
    // other (8 experts, 16 tokens of 4096: 10.9 us, so 4.4).  Layers of 64 hidden neurons, bf16, T E = 4096: 64 tokens of 4096 47.2
    // us, so 42.5, of 1024 22.5 and 21.9; 8192: 52.8 and 51.3, 24.2 and 25.1; 16384: 65.4 and 67.9, 28.5 and 31.5.
    if (a.T * a.E <= 4096) k_moe_logits<F32, VEC, 1><<<dim3(ceil_div(a.E, 4), a.T), 256, 0, st>>>(r);
    else k_moe_logits<F32, VEC, kRouteTokens><<<dim3(ceil_div(a.E, 4), ceil_div(a.T, kRouteTokens)), 256, 0, st>>>(r);
    if (!choose) k_moe_choose<<<a.T, kWave, 0, st>>>(r);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  // An expert of more tokens than the tiles hold reads its weights again.  With every choice as likely, that is one in
  // two hundred experts of a mean of 8 tokens and 16 a pass, and fewer with 20 and 32.
  const int tokens = a.T * a.k;
  if (a.T <= 16 || tokens <= 8 * a.E) return launch_experts<F32, VEC, 1>(r, a, choose, st);
  return a.T <= 32 || tokens <= 20 * a.E ? launch_experts<F32, VEC, 2>(r, a, false, st) : launch_experts<F32, VEC, 4>(r, a, false, st);
}

}  // namespace

int moe_slots(int T, int E, int k) { return std::min(T * k, E); }
int moe_ldz(int d_ff) { return ceil_div(d_ff, 32) * 32; }
// Enough workgroups for the card, each with a step of 32 for every wave.
static int moe_groups(bool f32, int d) { return ceil_div(kDownGroups, ceil_div(d, f32 ? 64 : 128)); }
static int moe_pieces_most(int d_ff) { return std::max(1, std::min(moe_ldz(d_ff) / 128, kMoePieces)); }
int moe_pieces(bool f32, int T, int d, int d_ff, int E, int k) {
  return std::min(ceil_div(moe_groups(f32, d), moe_slots(T, E, k)), moe_pieces_most(d_ff));
}
// With g groups to find and s slots, pieces = ceil(g / s): up to E places, places times pieces are s + g - 1 at most; with more of
// them pieces stay what they are with E slots.
size_t moe_part_rows(bool f32, int T, int d, int d_ff, int E, int k) {
  const size_t places = (size_t)T * k, slots = moe_slots(T, E, k);
  const size_t few = std::min(slots * moe_pieces_most(d_ff), slots + moe_groups(f32, d) - 1);
  return std::max(few, places > slots ? places * moe_pieces(f32, T, d, d_ff, E, k) : 0);
}

}  // namespace ffn

using namespace ffn;

extern "C" {

size_t ffn_moe_workspace_bytes(ffn_dtype_t wdt, int T, int d, int d_ff, int experts, int k) {
  if (!known(wdt) || check_moe_shape(T, d, d_ff, experts, k) != FFN_OK) return 0;
  return moe_layout(wdt == FFN_F32, T, d, d_ff, experts, k, nullptr, nullptr);
}

int ffn_moe_forward(ffn_dtype_t wdt, int T, int d, int d_ff, const ffn_router_t* router, const void* x,
                    const void* w_gate, const void* w_up, const void* w_down_t, float t, const ffn_options_t* opt,
                    int32_t* ids, float* weights, void* y, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!router || !x || !w_gate || !w_up || !w_down_t || !ids || !weights || !y || !ws) return FFN_ERR_NULL;
  if (!known(wdt)) return FFN_ERR_DTYPE;
  const int E = router->experts, k = router->k;
  if (const int rc = check_moe_shape(T, d, d_ff, E, k)) return rc;
  if (!aligned(x) || !aligned(w_gate) || !aligned(w_up) || !aligned(w_down_t) || !aligned(y) || !aligned(ws) ||
      !aligned(router->w) || !aligned(router->bias, 4) || !aligned(ids, 4) || !aligned(weights, 4))
    return FFN_ERR_ALIGN;
  if ((router->sigmoid != 0 && router->sigmoid != 1) || (router->normalize != 0 && router->normalize != 1)) return FFN_ERR_OPTION;
  if (router->w ? !isfinite(router->scale)
                : router->bias || router->sigmoid || router->normalize || router->scale != 0.f)
    return FFN_ERR_OPTION;
  ActForm form;
  if (const int rc = check_act(opt, t, &form)) return rc;
  const bool f32 = wdt == FFN_F32;
  MoeWs w;
  if (ws_bytes < moe_layout(f32, T, d, d_ff, E, k, ws, &w)) return FFN_ERR_WORKSPACE;

  const RouteArgs r{T, d, E, k, x, router->w, router->bias, router->sigmoid, router->normalize, router->scale,
                    w.logits, ids, weights};
  const MoeArgs a{T, d, d_ff, E, k, moe_ldz(d_ff), moe_slots(T, E, k), moe_pieces(f32, T, d, d_ff, E, k),
                  x, {w_gate, w_up, w_down_t}, form, ids, weights, w.z, (size_t)T * k * moe_ldz(d_ff), w.part, y};
  const bool lines = d % (f32 ? 32 : 64) == 0, chunks = d % (f32 ? 4 : 8) == 0;
  hipError_t e;
  if (f32) e = lines ? launch_moe<true, 2>(r, a, stream) : chunks ? launch_moe<true, 1>(r, a, stream) : launch_moe<true, 3>(r, a, stream);
  else e = lines ? launch_moe<false, 2>(r, a, stream) : chunks ? launch_moe<false, 1>(r, a, stream)
         : d % 2 == 0 ? launch_moe<false, 3>(r, a, stream) : launch_moe<false, 0>(r, a, stream);
  return e == hipSuccess ? FFN_OK : FFN_ERR_HIP;
}

}  // extern "C"
