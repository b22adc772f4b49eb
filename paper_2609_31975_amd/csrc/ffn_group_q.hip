// include/ffn_group_q.h: products of a decode step's tokens with 4-bit weights that have a scale (and an
// offset) for every group of codes along the summed dimension.
//
// The codes' bytes bound it, and the work a byte brings: two codes to turn into matrix operands.  So:
//   - The codes enter v_mfma_f32_16x16x32_bf16 unscaled.  Two nibbles of a dword become two bf16 of value
//     24 + code with a shift and an and-or (16 + u has u in its top mantissa bits; u = code + 8): 9 operations
//     for 8 codes.  What the 24 add, 24 times the sum of the same x, one product with the constant -24
//     takes away again, and that product serves every row tile.  A group's sum is then multiplied by its row's scale.
//   - Tokens are the A operand, weight rows the B operand: a lane's results are of one weight row, whose scale it
//     holds.
//   - A lane loads 16 bytes, 32 codes of a row; the four lanes of a row 128 (a window).  Where a window lies in one
//     group, MFMA f takes dword f of every lane, and x in the same order.  Else the four dwords are transposed between
//     the lanes (two v_permlane32_swap, two v_permlane16_swap), and each MFMA has 32 codes in a row.
//   - x lies in LDS, as bf16 in the order of the operands; fp32 x as three bf16 parts, three products.
#include <algorithm>

#include "ffn_group_q.h"
#include "ffn_mfma.h"
#include "ffn_step_device.h"

namespace ffn {
namespace {

constexpr int kWindow = 128;             // codes of a row that four lanes load at once
constexpr int kGqTokens = 64;            // tokens of a pass
constexpr size_t kGqLds = 64 * 1024;     // two workgroups to a CU
constexpr uint32_t kBias = 0xC1C0C1C0u;  // -24, twice

struct GqMatrix {
  const void *codes, *scales, *offsets;
};
struct GqArgs {
  int T, n_in, n_out;
  int windows;        // of a row
  int per_share;      // windows of a workgroup: a multiple of the chunk's
  int chunk;          // windows of x in LDS at a time
  uint32_t div_group; // q = (n div_group) >> 31 divides a count of 32 codes by group / 32
  int groups;         // of a row
  const void* x;
  GqMatrix w[2];
  ActForm form;
  void* y;
  float* part;        // [share][matrix][T][n_out], or null: one share
};

// four codes pairs of a dword: elements (0, 4), (1, 5), (2, 6), (3, 7) as 24 + code
__device__ __forceinline__ bf16x8_t codes8(uint32_t w) {
  const uint32_t u = w ^ 0x88888888u;
  constexpr uint32_t m = 0x00780078u, s = 0x41804180u;
  return bf8(make_uint4((u << 3 & m) | s, (u >> 1 & m) | s, (u >> 5 & m) | s, (u >> 9 & m) | s));
}

// dword f of lane group g <- dword g of lane group f
__device__ __forceinline__ uint4 transpose4(const uint4& v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  const u2 a = __builtin_bit_cast(u2, __builtin_amdgcn_permlane32_swap(v.x, v.z, false, false));
  const u2 b = __builtin_bit_cast(u2, __builtin_amdgcn_permlane32_swap(v.y, v.w, false, false));
  const u2 c = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false));
  const u2 d = __builtin_bit_cast(u2, __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false));
  return make_uint4(c[0], c[1], d[0], d[1]);
}

// Windows [w0, w0 + chunk) of x's T rows into LDS: rows of chunk * 256 + 16 bytes (the 16 spread the rows over the
// banks), plane after plane.  Columns past n_in are zero.
template <bool XF32, int THREADS>
__device__ __forceinline__ void stage_x(const GqArgs& a, char* lds, int w0) {
  const int units = a.chunk * (kWindow / 8), stride = a.chunk * 2 * kWindow + 16;
  const Buf xb = make_buf(a.x, (uint32_t)a.T * a.n_in * (XF32 ? 4 : 2));
  for (int i = threadIdx.x; i < a.T * units; i += THREADS) {
    const int t = i / units, c = i - t * units, k = w0 * kWindow + c * 8;
    const uint32_t o = k < a.n_in ? ((uint32_t)t * a.n_in + k) * (XF32 ? 4 : 2) : kOOB;
    char* p = lds + t * stride + c * 16;
    if constexpr (XF32) {
      const uint4 lo = ldb(xb, o), hi = ldb(xb, k < a.n_in ? o + 16 : kOOB);
      // elements (0, 4), (1, 5), (2, 6), (3, 7)
      float v[8] = {comp<0>(lo), comp<0>(hi), comp<1>(lo), comp<1>(hi), comp<2>(lo), comp<2>(hi), comp<3>(lo), comp<3>(hi)};
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        uint32_t d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[j] = f_to_bf2(v[2 * j], v[2 * j + 1]);
          v[2 * j] -= __uint_as_float(d[j] << 16);
          v[2 * j + 1] -= __uint_as_float(d[j] & 0xffff0000u);
        }
        *reinterpret_cast<uint4*>(p + q * a.T * stride) = make_uint4(d[0], d[1], d[2], d[3]);
      }
    } else {
      const uint4 v = ldb(xb, o);
      *reinterpret_cast<uint4*>(p) = make_uint4(__builtin_amdgcn_perm(v.z, v.x, 0x05040100u), __builtin_amdgcn_perm(v.z, v.x, 0x07060302u),
                                                __builtin_amdgcn_perm(v.w, v.y, 0x05040100u), __builtin_amdgcn_perm(v.w, v.y, 0x07060302u));
    }
  }
}

// 8 waves: WK of them share a row tile's windows, 8 / WK row tiles of 16 to a workgroup.  NT: 16-token
// tiles.  U: windows that a wave has in flight.  TR: windows do not lie in one group.
template <bool XF32, bool SF32, bool GATED, bool TR, int NT, int WK, int U>
__global__ __launch_bounds__(512, 4) void k_group_q(GqArgs a) {
  constexpr int M = GATED ? 2 : 1, WR = 8 / WK, P = XF32 ? 3 : 1, NS = TR ? 4 : 1;
  extern __shared__ __align__(16) char lds[];
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int wk = wave % WK, row0 = (blockIdx.x * WR + wave / WK) * 16, row = row0 + n;
  const bool row_ok = row < a.n_out;
  const int first = blockIdx.y * a.per_share, last = min(a.windows, first + a.per_share);
  const uint32_t row_bytes = (uint32_t)a.n_in / 2, ss = SF32 ? 4 : 2;

  Buf cb[M], sb[M], ob[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    cb[m] = make_buf(a.w[m].codes, row_bytes * a.n_out);
    sb[m] = make_buf(a.w[m].scales, (uint32_t)a.n_out * a.groups * ss);
    ob[m] = make_buf(a.w[m].offsets, a.w[m].offsets ? (uint32_t)a.n_out * a.groups * ss : 0u);
  }
  const bool off = a.w[0].offsets != nullptr;

  struct Batch {
    uint4 c[U][M];
    float s[U][M][NS], o[U][M][NS];
  };
  auto value = [&](const Buf& b, uint32_t i) -> float {
    if constexpr (SF32) return __builtin_bit_cast(float, ldb32(b, i));
    else return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, i, 0, 0) << 16);
  };
  auto load = [&](int w_first, Batch& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int w = w_first + u * WK + wk;
      const bool in = row_ok && w < last;
#pragma unroll
      for (int m = 0; m < M; ++m)
        b.c[u][m] = ldb_nt(cb[m], in && w * kWindow + g * 32 < a.n_in ? row * row_bytes + w * (kWindow / 2) + g * 16 : kOOB);
#pragma unroll
      for (int f = 0; f < NS; ++f) {
        const uint32_t k32 = w * 4 + f, gi = (uint32_t)((uint64_t)k32 * a.div_group >> 31);
        const uint32_t at = in && (int)(k32 * 32) < a.n_in ? ((uint32_t)row * a.groups + gi) * ss : kOOB;
#pragma unroll
        for (int m = 0; m < M; ++m) {
          b.s[u][m][f] = value(sb[m], at);
          b.o[u][m][f] = off ? value(ob[m], at) : 0.f;
        }
      }
    }
  };

  f32x4_t acc[NT][M] = {};
  Batch cur;
  load(first, cur);
  const int stride = a.chunk * 2 * kWindow + 16;
  const bf16x8_t bias = bf8(make_uint4(kBias, kBias, kBias, kBias));
  for (int c0 = first; c0 < last; c0 += a.chunk) {
    if (c0 != first) __syncthreads();
    stage_x<XF32, 512>(a, lds, c0);
    __syncthreads();
    const int end = min(a.chunk, last - c0);
    for (int b0 = 0; b0 < end; b0 += WK * U) {
      Batch nxt;
      load(c0 + b0 + WK * U, nxt);
      issue_barrier();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int w = b0 + u * WK + wk;  // within the chunk: the chunk is a multiple of WK U
#pragma unroll
        for (int m = 0; m < M; ++m)
          if constexpr (TR) cur.c[u][m] = transpose4(cur.c[u][m]);
        bf16x8_t wf[M][4];
#pragma unroll
        for (int m = 0; m < M; ++m) {
          wf[m][0] = codes8(cur.c[u][m].x);
          wf[m][1] = codes8(cur.c[u][m].y);
          wf[m][2] = codes8(cur.c[u][m].z);
          wf[m][3] = codes8(cur.c[u][m].w);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          // results of tokens past the last one are not stored, and depend on nothing but their own rows
          const char* xp = lds + min(t * 16 + n, a.T - 1) * stride + w * 2 * kWindow;
          f32x4_t sum[M] = {}, gone = {};
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            bf16x8_t x[P];
#pragma unroll
            for (int p = 0; p < P; ++p)
              x[p] = bf8(*reinterpret_cast<const uint4*>(xp + p * a.T * stride + (TR ? f * 64 + g * 16 : g * 64 + f * 16)));
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {
              gone = mfma16(x[p], bias, gone);
#pragma unroll
              for (int m = 0; m < M; ++m) sum[m] = mfma16(x[p], wf[m][f], sum[m]);
            }
            if (TR || f == 3) {
              const int q = TR ? f : 0;
#pragma unroll
              for (int m = 0; m < M; ++m) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  acc[t][m][i] += cur.s[u][m][q] * (sum[m][i] + gone[i]);
                  if (off) acc[t][m][i] += cur.o[u][m][q] * (gone[i] * (-1.f / 24.f));
                }
                sum[m] = f32x4_t{};
              }
              gone = f32x4_t{};
            }
          }
        }
      }
      cur = nxt;
    }
  }

  // The WK waves' sums joined in LDS, in their order; one token tile at a time.
  float* red = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[((wave * M + m) * 4 + i) * 64 + lane] = acc[t][m][i];
    __syncthreads();
    for (int e = threadIdx.x; e < WR * 256; e += 512) {
      const int r = e >> 8, i = e >> 6 & 3, l = e & 63;
      const int tok = t * 16 + (l >> 4) * 4 + i, o = (blockIdx.x * WR + r) * 16 + (l & 15);
      if (tok >= a.T || o >= a.n_out) continue;
      float v[M] = {};
#pragma unroll
      for (int k = 0; k < WK; ++k)
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] += red[(((r * WK + k) * M + m) * 4 + i) * 64 + l];
      if (a.part) {
#pragma unroll
        for (int m = 0; m < M; ++m) a.part[(((size_t)blockIdx.y * M + m) * a.T + tok) * a.n_out + o] = v[m];
      } else {
        const float z = GATED ? act_product(a.form, v[0], v[M - 1]) : v[0];
        store_as<XF32>(a.y, (size_t)tok * a.n_out + o, z);
      }
    }
  }
}

template <bool XF32, bool GATED>
__global__ __launch_bounds__(256) void k_group_q_join(GqArgs a, int shares) {
  constexpr int M = GATED ? 2 : 1;
  const size_t count = (size_t)a.T * a.n_out;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < count; e += (size_t)gridDim.x * 256) {
    float v[M] = {};
    for (int s = 0; s < shares; ++s)
#pragma unroll
      for (int m = 0; m < M; ++m) v[m] += a.part[((size_t)s * M + m) * count + e];
    store_as<XF32>(a.y, e, GATED ? act_product(a.form, v[0], v[M - 1]) : v[0]);
  }
}

// Tiles of a pass, by its tokens: the windows of x that a workgroup's waves take at once have to fit in LDS.
struct GqPlan {
  int nt, wk, u;
  int chunk, per_share, shares, blocks;
};
GqPlan gq_plan(bool xf32, bool gated, int T, int n_in, int n_out) {
  const int planes = xf32 ? 3 : 1, windows = ceil_div(n_in, kWindow);
  auto bytes = [&](int chunk) { return (size_t)planes * T * (chunk * 2 * kWindow + 16); };
  GqPlan p{};
  p.nt = T <= 16 ? 1 : T <= 32 ? 2 : 4;
  if (p.nt == 1) {
    p.wk = 8;
    p.u = gated ? 2 : 4;
    if (bytes(p.wk * p.u) > kGqLds) p.u = 1;
    if (bytes(p.wk * p.u) > kGqLds) p.wk = 4;
  } else {
    p.wk = (xf32 ? 4 : 8) / p.nt;
    p.u = 1;
  }
  const int unit = p.wk * p.u;
  p.blocks = ceil_div(n_out, 8 / p.wk * 16);
  p.shares = 1;
  p.per_share = ceil_div(windows, unit) * unit;
  p.chunk = unit;
  while (p.chunk < p.per_share && bytes(p.chunk + unit) <= kGqLds) p.chunk += unit;
  p.per_share = ceil_div(p.per_share, p.chunk) * p.chunk;
  return p;
}
constexpr int kGqSharesMost = 1;

template <bool XF32, bool SF32, bool GATED, bool TR>
hipError_t launch_gq(const GqArgs& a, const GqPlan& p, hipStream_t st) {
  const size_t x = (size_t)(XF32 ? 3 : 1) * a.T * (p.chunk * 2 * kWindow + 16);
  const size_t lds = std::max<size_t>(x, 8 * (GATED ? 2 : 1) * 1024);
  const dim3 grid(p.blocks, p.shares);
  auto go = [&](auto nt, auto wk, auto u) {
    k_group_q<XF32, SF32, GATED, TR, nt.value, wk.value, u.value><<<grid, 512, lds, st>>>(a);
    return hipGetLastError();
  };
  constexpr int kU = GATED ? 2 : 4;
  if (p.nt == 1 && p.wk == 8 && p.u == kU) return go(Int<1>{}, Int<8>{}, Int<kU>{});
  if (p.nt == 1 && p.wk == 8) return go(Int<1>{}, Int<8>{}, Int<1>{});
  if constexpr (XF32) {
    if (p.nt == 1) return go(Int<1>{}, Int<4>{}, Int<1>{});
    if (p.nt == 2) return go(Int<2>{}, Int<2>{}, Int<1>{});
    return go(Int<4>{}, Int<1>{}, Int<1>{});
  } else {
    if (p.nt == 2) return go(Int<2>{}, Int<4>{}, Int<1>{});
    return go(Int<4>{}, Int<2>{}, Int<1>{});
  }
}

int check_gq_shape(int T, int n_in, int n_out) {
  if (T < 1 || n_in < 1 || n_out < 1 || n_in > 1 << 20 || n_out > 1 << 20) return FFN_ERR_SHAPE;
  if ((int64_t)T * n_in >= kMaxElems || (int64_t)T * n_out >= kMaxElems || (int64_t)n_in * n_out >= kMaxElems) return FFN_ERR_SHAPE;
  return FFN_OK;
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
  const bool xf32 = xdt == FFN_F32, sf32 = w->sdt == FFN_F32, tr = w->group % kWindow != 0;
  const size_t xs = xf32 ? 4 : 2;
  for (int t0 = 0; t0 < T; t0 += kGqTokens) {
    GqArgs a{};
    a.T = std::min(kGqTokens, T - t0);
    const GqPlan p = gq_plan(xf32, w2 != nullptr, a.T, n_in, n_out);
    a.n_in = n_in;
    a.n_out = n_out;
    a.windows = ceil_div(n_in, kWindow);
    a.per_share = p.per_share;
    a.chunk = p.chunk;
    a.div_group = (uint32_t)(((uint64_t)1 << 31) / (w->group / 32) + 1);
    a.groups = n_in / w->group;
    a.x = static_cast<const char*>(x) + (size_t)t0 * n_in * xs;
    a.w[0] = GqMatrix{w->codes, w->scales, w->offsets};
    if (w2) a.w[1] = GqMatrix{w2->codes, w2->scales, w2->offsets};
    a.form = form;
    a.y = static_cast<char*>(y) + (size_t)t0 * n_out * xs;
    a.part = p.shares > 1 ? static_cast<float*>(ws) : nullptr;
    hipError_t e;
    auto pick = [&](auto xf, auto sf, auto gated) {
      return tr ? launch_gq<xf.value, sf.value, gated.value, true>(a, p, st)
                : launch_gq<xf.value, sf.value, gated.value, false>(a, p, st);
    };
    auto pick2 = [&](auto xf, auto sf) { return w2 ? pick(xf, sf, Int<1>{}) : pick(xf, sf, Int<0>{}); };
    if (xf32) e = sf32 ? pick2(Int<1>{}, Int<1>{}) : pick2(Int<1>{}, Int<0>{});
    else e = sf32 ? pick2(Int<0>{}, Int<1>{}) : pick2(Int<0>{}, Int<0>{});
    if (e == hipSuccess && p.shares > 1) {
      const int blocks = (int)std::min<size_t>(ceil_div<size_t>((size_t)a.T * n_out, 256), 4096);
      if (xf32 && w2) k_group_q_join<true, true><<<blocks, 256, 0, st>>>(a, p.shares);
      else if (xf32) k_group_q_join<true, false><<<blocks, 256, 0, st>>>(a, p.shares);
      else if (w2) k_group_q_join<false, true><<<blocks, 256, 0, st>>>(a, p.shares);
      else k_group_q_join<false, false><<<blocks, 256, 0, st>>>(a, p.shares);
      e = hipGetLastError();
    }
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
  return sizeof(float) * kGqSharesMost * (gated ? 2 : 1) * (size_t)std::min(T, kGqTokens) * n_out;
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
