// include/ffn_norm.h: the norms before and after a block with its gate and residual, and their backward
// pass.  Both move bytes: a token's row is read once into registers, its one or two means are summed
// across the threads that hold it, and the outputs are written from the registers.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ffn_norm.h"
#include "ffn_norm_internal.h"
#include "ffn_step_device.h"

namespace ffn {
namespace {

// Threads to a row (TPR) and elements to a thread (EPT).  A wave or a workgroup holds a row of up to
// TPR EPT elements; 64 threads take 4 rows to a workgroup and need no barrier.
constexpr int kMaxNormRow = 16384;

struct NormArgs {
  int T, d;
  float alpha, eps;
  int post, sigmoid, gate_rows;
  const void *x, *f, *gate, *post_gain, *pre_gain;
  void *x_out, *n_out;
  float* rstd;
};

// Sixteen bytes at any element's address: a load or store of that width needs no alignment, and a wave's neighbours
// still share their lines.
typedef uint32_t any4_t __attribute__((ext_vector_type(4), aligned(2)));

// The elements of a row that a thread holds: 16-byte chunks, a row's chunks dealt out over its threads.  VEC: rows
// are whole chunks, and a row is a buffer, behind whose end loads give zeros and stores nothing (with compares of
// each element and 64-bit addresses instead, the vector ALUs were busy for 87% of 8192 x 8192's forward call).
// Otherwise a row starts anywhere, and the chunk that it ends in goes by elements (4096 rows of 4097 bf16: 51 us, all of
// it by elements 133, rows of 4096 29; forward and backward 157, 600 and 92).
template <bool F32, int TPR, int EPT, bool VEC>
struct Part {
  static constexpr int E = F32 ? 4 : 8, N = EPT / E, ES = F32 ? 4 : 2;
  static __device__ __forceinline__ int at(int t, int i) { return (i * TPR + t) * E; }

  static __device__ __forceinline__ float element(const void* p, int64_t o) {
    return F32 ? static_cast<const float*>(p)[o] : bf_to_f(static_cast<const uint16_t*>(p)[o]);
  }
  // row: the same for a wave
  template <bool STREAM = false>
  static __device__ __forceinline__ void load(const void* p, int64_t row, int d, int t, float (&v)[EPT]) {
    uint4 c[N];
    if constexpr (VEC) {
      const Buf b = make_buf(static_cast<const char*>(p) + row * d * ES, (uint32_t)d * ES);
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = STREAM ? ldb_nt(b, (uint32_t)at(t, i) * ES) : ldb(b, (uint32_t)at(t, i) * ES);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = at(t, i);
        const char* from = static_cast<const char*>(p) + (row * d + (e < d ? e : 0)) * ES;
        any4_t u = {0, 0, 0, 0};
        if (e + E <= d) u = STREAM ? __builtin_nontemporal_load(reinterpret_cast<const any4_t*>(from)) : *reinterpret_cast<const any4_t*>(from);
        c[i] = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float u[E];
      if constexpr (F32) unpack(WF32{}, c[i], u);
      else unpack(WBf16{}, c[i], u);
#pragma unroll
      for (int j = 0; j < E; ++j) v[i * E + j] = u[j];
      if constexpr (!VEC) {
        const int e = at(t, i);
        if (e < d && e + E > d) {
#pragma unroll
          for (int j = 0; j < E - 1; ++j)
            if (e + j < d) v[i * E + j] = element(p, row * d + e + j);
        }
      }
    }
  }
  static __device__ __forceinline__ void store(void* p, int64_t row, int d, int t, const float (&v)[EPT]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = at(t, i);
      any4_t w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (F32) w[j] = __float_as_uint(v[i * 4 + j]);
        else w[j] = f_to_bf2(v[i * 8 + 2 * j], v[i * 8 + 2 * j + 1]);
      }
      if constexpr (VEC) {
        const Buf b = make_buf(static_cast<const char*>(p) + row * d * ES, (uint32_t)d * ES);
        __builtin_amdgcn_raw_buffer_store_b128(w, b.r, (uint32_t)e * ES, 0, 0);
      } else if (e + E <= d) {
        *reinterpret_cast<any4_t*>(static_cast<char*>(p) + (row * d + e) * ES) = w;
      } else if (e < d) {
        const int64_t o = row * d + e;
#pragma unroll
        for (int j = 0; j < E - 1; ++j) {
          if (e + j >= d) continue;
          if constexpr (F32) static_cast<float*>(p)[o + j] = v[i * 4 + j];
          else static_cast<uint16_t*>(p)[o + j] = f_to_bf(v[i * 8 + j]);
        }
      }
    }
  }
};

// sigma(c) = 1 / (1 + e), e = 2^(-c log2 e), the exponent in two parts and the quotient with a step of Newton's: within 3 units
// in the last place, at half of what expf and a division cost.  1 - sigma is e sigma: taken from 1 it would lose the bits that
// its slope sigma (1 - sigma) is made of (7% of it at c = 14, all from 17 on).  NaN stays NaN.  |c| up to 88, behind which
// sigma is 0 or 1 to fp32's range.
struct Logistic {
  float value, rest;  // sigma, 1 - sigma
};
__device__ __forceinline__ Logistic logistic(float c) {
  c = c > 88.f ? 88.f : c;
  c = c < -88.f ? -88.f : c;
  constexpr float kLog2e = 1.44269504f, kRest = 1.92596299e-8f;  // log2 e = their sum
  const float p = -c * kLog2e, rest = fmaf(-c, kLog2e, -p) - c * kRest;
  const float e2 = __builtin_amdgcn_exp2f(p), e = fmaf(e2, rest * 0.693147181f, e2), a = 1.f + e;
  const float r = __builtin_amdgcn_rcpf(a), s = fmaf(fmaf(-a, r, 1.f), r, r);
  return Logistic{s, e * s};
}

// Sum over the threads of a row.  `room`: TPR / 64 floats of LDS that no earlier sum of the same row used, and none
// that is still being read: the sums of a row use rooms of their own, and each row's first barrier lies between
// the last row's reads of a room and this row's writes of it.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* room) {
  v = wave_sum(v);
  if constexpr (TPR == 64) return v;
  if (lane_id() == 0) room[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < TPR / 64; ++i) s += room[i];
  return s;
}

// 1 / sqrt(mean v^2 + eps) of a row.  `room`: two of row_sum's, the second for a row whose sum of squares passes fp32's range
// (values of 2^57 and more): its values times 2^-80, of squares from 2^-46 to 2^96.  A row that holds an Inf keeps it.  The
// branch is the same for all threads of a row.
template <int TPR, int EPT>
__device__ __forceinline__ float row_rms(const float (&v)[EPT], int d, float eps, float (*room)[16]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < EPT; ++i) s += v[i] * v[i];
  s = row_sum<TPR>(s, room[0]);
  if (s == INFINITY) {
    constexpr float kDown = 0x1p-80f;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < EPT; ++i) s += (v[i] * kDown) * (v[i] * kDown);
    return kDown / sqrtf(row_sum<TPR>(s, room[1]) / (float)d + eps * kDown * kDown);
  }
  return 1.f / sqrtf(s / (float)d + eps);
}

// STREAM: rows are read past the caches.  Bound by bytes: 4096 x 4096 bf16 with a gate for each token, 168 MB, 32 us (5.2
// TB/s); 8192 x 8192, 671 MB, 109 us (6.2 TB/s); one token 3.3 us, the loads' latency twice and two sums.
template <bool F32, int TPR, int EPT, bool VEC, bool STREAM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm_fwd(NormArgs a) {
  using P = Part<F32, TPR, EPT, VEC>;
  constexpr int WG = TPR < 256 ? 256 : TPR, ROWS = WG / TPR;
  __shared__ float room[2][4][16];
  const int t = threadIdx.x % TPR;
  int turn = 0;
  for (int64_t row = (int64_t)blockIdx.x * ROWS + uniform(threadIdx.x / TPR); row < a.T; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    float x[EPT], u[EPT], c[EPT];
    P::template load<STREAM>(a.x, row, a.d, t, x);
    if (a.f) {
      P::template load<STREAM>(a.f, row, a.d, t, u);
      if (a.gate_rows) P::template load<STREAM>(a.gate, a.gate_rows == 1 ? 0 : row, a.d, t, c);
      if (a.post) {
        const float r = row_rms<TPR>(u, a.d, a.eps, room[turn]);
        if (t == 0 && a.rstd) a.rstd[row] = r;
#pragma unroll
        for (int i = 0; i < EPT; ++i) u[i] *= r;
        if (a.post_gain) {
          float w[EPT];
          P::load(a.post_gain, 0, a.d, t, w);
#pragma unroll
          for (int i = 0; i < EPT; ++i) u[i] *= w[i];
        }
      }
      if (a.gate_rows) {
        if (a.sigmoid) {
#pragma unroll
          for (int i = 0; i < EPT; ++i) c[i] = logistic(c[i]).value;
        }
#pragma unroll
        for (int i = 0; i < EPT; ++i) u[i] *= c[i];
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] = a.alpha * x[i] + u[i];
    }
    if (a.x_out) P::store(a.x_out, row, a.d, t, x);
    if (a.n_out) {
      const float r = row_rms<TPR>(x, a.d, a.eps, room[turn] + 2);
      if (t == 0 && a.rstd) a.rstd[(int64_t)a.T + row] = r;
#pragma unroll
      for (int i = 0; i < EPT; ++i) x[i] *= r;
      if (a.pre_gain) {
        float w[EPT];
        P::load(a.pre_gain, 0, a.d, t, w);
#pragma unroll
        for (int i = 0; i < EPT; ++i) x[i] *= w[i];
      }
      P::store(a.n_out, row, a.d, t, x);
    }
  }
}

struct NormBack {
  int T, d;
  float alpha;
  int post, sigmoid, gate_rows;
  const void *x_out, *f, *gate, *post_gain, *pre_gain;
  const float* rstd;
  const void *dn, *dx_out;
  void *dx, *df, *dgate;   // dgate: rows of T (of one row: summed)
  float* part[3];          // [groups][d] of dpre_gain, dpost_gain, dgate of one row; null: not wanted
};

// One group of threads takes every groups-th row and keeps its columns' sums over them in registers.  Bound by bytes: 8192 x
// 8192 bf16 with a gate for each token reads five rows and writes three, 1.07 GB, in 250 us (4.3 TB/s); a row's two means
// leave its loads waiting for the row before (those of the next row a row early, in two sets of registers, spill).  Rows of more than
// 8192 take 16 elements to each of 1024 threads, which do not fit: 76 to 155 registers spill inside the loop over the rows (2048 x
// 12288, gate of each token, forward and backward: bf16 272 us, 1.9 TB/s, fp32 373, 2.7).
template <bool F32, int TPR, int EPT, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, EPT == 8 ? 4 : 1) void k_norm_bwd(NormBack a) {
  using P = Part<F32, TPR, EPT, VEC>;
  constexpr int WG = TPR < 256 ? 256 : TPR, ROWS = WG / TPR;
  __shared__ float room[2][2][16];
  const int t = threadIdx.x % TPR;
  const int64_t group = (int64_t)blockIdx.x * ROWS + uniform(threadIdx.x / TPR);
  float sp[EPT] = {}, so[EPT] = {}, sg[EPT] = {};
  const bool block_side = a.f && (a.df || a.dgate || a.part[1] || a.part[2]);
  int turn = 0;
  for (int64_t row = group; row < a.T; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
    float g[EPT], f[EPT], c[EPT];
    if (a.dx_out) P::load(a.dx_out, row, a.d, t, g);
    if (block_side) {
      P::load(a.f, row, a.d, t, f);
      if (a.gate_rows) P::load(a.gate, a.gate_rows == 1 ? 0 : row, a.d, t, c);
    }
    if (a.dn) {
      float n[EPT], xh[EPT], w[EPT];
      P::load(a.dn, row, a.d, t, n);
      P::load(a.x_out, row, a.d, t, xh);
      if (a.pre_gain) P::load(a.pre_gain, 0, a.d, t, w);
      const float r = a.rstd[(int64_t)a.T + row];
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) xh[i] *= r;
      if (a.part[0]) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) sp[i] += n[i] * xh[i];
      }
      if (a.pre_gain) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) n[i] *= w[i];
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) s += n[i] * xh[i];
      const float m = row_sum<TPR>(s, room[turn][0]) / (float)a.d;
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const float v = r * (n[i] - xh[i] * m);
        g[i] = a.dx_out ? g[i] + v : v;
      }
    }
    if (a.dx) {
      float v[EPT];
#pragma unroll
      for (int i = 0; i < EPT; ++i) v[i] = a.alpha * g[i];
      P::store(a.dx, row, a.d, t, v);
    }
    if (!block_side) continue;
    // du = c G (in g), with dgate = G u c'
    const float rf = a.post ? a.rstd[row] : 1.f;
    float w[EPT];
    if (a.post && a.post_gain) P::load(a.post_gain, 0, a.d, t, w);
    else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) w[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < EPT; ++i) f[i] *= rf;
    if (a.gate_rows) {
      float dg[EPT];
#pragma unroll
      for (int i = 0; i < EPT; ++i) dg[i] = g[i] * (f[i] * w[i]);
      if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
          const Logistic l = logistic(c[i]);
          c[i] = l.value;
          dg[i] *= l.value * l.rest;
        }
      }
      if (a.part[2]) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) sg[i] += dg[i];
      }
#pragma unroll
      for (int i = 0; i < EPT; ++i) g[i] *= c[i];
      if (a.dgate && a.gate_rows != 1) P::store(a.dgate, row, a.d, t, dg);
    }
    if (a.post) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) so[i] += g[i] * f[i];  // a sum that is not wanted is not stored
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        g[i] *= w[i];
        s += g[i] * f[i];
      }
      if (a.df) {
        const float m = row_sum<TPR>(s, room[turn][1]) / (float)a.d;
#pragma unroll
        for (int i = 0; i < EPT; ++i) g[i] = rf * (g[i] - f[i] * m);
      }
    }
    if (a.df) P::store(a.df, row, a.d, t, g);
  }
  auto put = [&](float* p, const float(&v)[EPT]) {
    if (!p) return;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
      const int e = P::at(t, i / P::E) + i % P::E;
      if (e < a.d) p[group * a.d + e] = v[i];
    }
  };
  put(a.part[0], sp);
  put(a.part[1], so);
  put(a.part[2], sg);
}

// out[i] [d] = sum over the groups' rows of part[i], in a fixed order: 16 threads to a column take every
// 16th row each, and one joins them.
// Latency: 256 rows of 8192, two sums 5 us, 257 of 3840, three 4 us.
constexpr int kSumLoads = 8;
struct NormSums {
  int groups, d;
  const float* part[3];
  void* out[3];
};
template <bool F32>
__global__ __launch_bounds__(1024) void k_norm_sums(NormSums a) {
  __shared__ float s[16][64];
  const int c = blockIdx.x * 64 + lane_id(), w = threadIdx.x >> 6;
  const float* p = a.part[blockIdx.y];
  float v = 0.f;
  if (c < a.d) {
    for (int r0 = w; r0 < a.groups; r0 += 16 * kSumLoads) {  // so many loads in flight
      float u[kSumLoads];
#pragma unroll
      for (int i = 0; i < kSumLoads; ++i) {
        const int r = r0 + 16 * i;
        u[i] = r < a.groups ? p[(int64_t)r * a.d + c] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < kSumLoads; ++i) v += u[i];
    }
  }
  s[w][lane_id()] = v;
  __syncthreads();
  if (w == 0 && c < a.d) {
    float u = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) u += s[i][lane_id()];
    if constexpr (F32) static_cast<float*>(a.out[blockIdx.y])[c] = u;
    else static_cast<uint16_t*>(a.out[blockIdx.y])[c] = f_to_bf(u);
  }
}

// go(threads, elements) of the plan; the plans of either call are all listed
template <int TPR, int EPT, int... REST, class F>
hipError_t with_plan(const NormPlan& p, const F& go) {
  if (p.tpr == TPR && p.ept == EPT) return go(std::integral_constant<int, TPR>{}, std::integral_constant<int, EPT>{});
  if constexpr (sizeof...(REST) > 0) return with_plan<REST...>(p, go);
  return hipErrorInvalidValue;
}

template <bool F32, bool VEC>
hipError_t launch_fwd(const NormArgs& a, hipStream_t st) {
  // Rows that no backward call reads again, or too many to find them in a cache then, are streamed (4096 x 4096 bf16: 35.7
  // us through the caches, 32.4 past them, 5.2 TB/s; 8192 x 8192 118 and 108; 513 x 3840 fp32, forward and backward: 3 us
  // more past them).
  const bool stream = !a.rstd || (int64_t)a.T * a.d * (F32 ? 4 : 2) >= (int64_t)64 << 20;
  return with_plan<64, 8, 64, 16, 256, 8, 256, 16, 512, 16, 1024, 16>(norm_forward_plan(a.d), [&](auto tpr, auto ept) {
    constexpr int WG = tpr.value < 256 ? 256 : tpr.value;
    const int blocks = norm_blocks(a.T, a.d);
    if (stream) k_norm_fwd<F32, tpr.value, ept.value, VEC, true><<<blocks, WG, 0, st>>>(a);
    else k_norm_fwd<F32, tpr.value, ept.value, VEC, false><<<blocks, WG, 0, st>>>(a);
    return hipGetLastError();
  });
}
template <bool F32, bool VEC>
hipError_t launch_bwd(const NormBack& a, int groups, hipStream_t st) {
  return with_plan<64, 8, 256, 8, 512, 8, 1024, 8, 1024, 16>(norm_backward_plan(a.d), [&](auto tpr, auto ept) {
    constexpr int WG = tpr.value < 256 ? 256 : tpr.value, ROWS = WG / tpr.value;
    k_norm_bwd<F32, tpr.value, ept.value, VEC><<<groups / ROWS, WG, 0, st>>>(a);
    return hipGetLastError();
  });
}

int check_norm_shape(int T, int d) {
  if (T < 1 || d < 1 || d > kMaxNormRow || (int64_t)T * d >= kMaxElems) return FFN_ERR_SHAPE;
  return FFN_OK;
}
int check_norm_form(const ffn_norm_t* n, int T, bool f) {
  if (!isfinite(n->alpha) || !isfinite(n->eps) || !(n->eps > 0.f)) return FFN_ERR_OPTION;
  if ((n->post != 0 && n->post != 1) || (n->gate_sigmoid != 0 && n->gate_sigmoid != 1)) return FFN_ERR_OPTION;
  if (n->gate_rows != 0 && n->gate_rows != 1 && n->gate_rows != T) return FFN_ERR_OPTION;
  if ((n->gate_rows != 0) != (n->gate != nullptr) || (n->gate_sigmoid && !n->gate)) return FFN_ERR_OPTION;
  if (n->post_gain && !n->post) return FFN_ERR_OPTION;
  if (!f && (n->alpha != 1.f || n->post || n->gate)) return FFN_ERR_OPTION;
  if (!aligned(n->gate) || !aligned(n->post_gain) || !aligned(n->pre_gain)) return FFN_ERR_ALIGN;
  return FFN_OK;
}

}  // namespace

NormPlan norm_forward_plan(int d) {
  const int tpr = d <= 1024 ? 64 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024;
  return NormPlan{tpr, d <= tpr * 8 ? 8 : 16};
}
// The backward call holds six rows and up to three sums: 8 elements to a thread leave room for twice the waves (8192 x 8192
// bf16: 256 us with 16, so 252).
NormPlan norm_backward_plan(int d) {
  const int tpr = d <= 512 ? 64 : d <= 2048 ? 256 : d <= 4096 ? 512 : 1024;
  return NormPlan{tpr, d <= 8192 ? 8 : 16};
}
int norm_blocks(int T, int d) { return std::min(ceil_div(T, norm_forward_plan(d).tpr == 64 ? 4 : 1), 1 << 20); }
// Rows in flight in the backward call: what the card holds at once (8192 x 8192 bf16: twice as many 309 us forward and
// backward, so 292).  Of more than 128 wide rows no more than leave every group two: the partial sums are read and written
// once more (300 x 8192 bf16: 49 us with a row each, so 33; 40 x 6000 23 with two, so 21).
int norm_groups(int T, int d) {
  const NormPlan p = norm_backward_plan(d);
  if (p.tpr == 64) return std::min(512, ceil_div(T, 4)) * 4;
  return std::min(p.tpr == 256 ? 1024 : p.tpr == 512 ? 512 : 256, std::max(ceil_div(T, 2), std::min(T, 128)));
}

}  // namespace ffn

using namespace ffn;

extern "C" {

int ffn_norm_forward(ffn_dtype_t dt, int T, int d, const void* x, const void* f, const ffn_norm_t* form, void* x_out,
                     void* n_out, float* rstd, hipStream_t stream) {
  if (!x || !form || (!x_out && !n_out)) return FFN_ERR_NULL;
  if (!known(dt)) return FFN_ERR_DTYPE;
  if (const int rc = check_norm_shape(T, d)) return rc;
  if (!aligned(x) || !aligned(f) || !aligned(x_out) || !aligned(n_out) || !aligned(rstd, 4)) return FFN_ERR_ALIGN;
  if (const int rc = check_norm_form(form, T, f != nullptr)) return rc;
  if ((!f && x_out) || (!n_out && form->pre_gain)) return FFN_ERR_OPTION;
  const NormArgs a{T, d, form->alpha, form->eps, form->post, form->gate_sigmoid, form->gate_rows, x, f,
                   form->gate, form->post_gain, form->pre_gain, x_out, n_out, rstd};
  const hipError_t e = dt == FFN_F32 ? (d % 4 ? launch_fwd<true, false>(a, stream) : launch_fwd<true, true>(a, stream))
                                     : (d % 8 ? launch_fwd<false, false>(a, stream) : launch_fwd<false, true>(a, stream));
  return e == hipSuccess ? FFN_OK : FFN_ERR_HIP;
}

size_t ffn_norm_workspace_bytes(int T, int d) {
  if (check_norm_shape(T, d) != FFN_OK) return 0;
  Carver c{nullptr};
  for (int i = 0; i < 3; ++i) c.take(sizeof(float) * norm_groups(T, d) * (size_t)d);
  return c.off;
}

int ffn_norm_backward(ffn_dtype_t dt, int T, int d, const void* x_out, const void* f, const ffn_norm_t* form,
                      const float* rstd, const void* dn, const void* dx_out, void* dx, void* df, void* dgate,
                      void* dpost_gain, void* dpre_gain, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!form || !ws || (!dn && !dx_out) || (!dx && !df && !dgate && !dpost_gain && !dpre_gain)) return FFN_ERR_NULL;
  if (!known(dt)) return FFN_ERR_DTYPE;
  if (const int rc = check_norm_shape(T, d)) return rc;
  for (const void* p : {x_out, f, dn, dx_out, (const void*)dx, (const void*)df, (const void*)dgate,
                        (const void*)dpost_gain, (const void*)dpre_gain, (const void*)ws})
    if (!aligned(p)) return FFN_ERR_ALIGN;
  if (!aligned(rstd, 4)) return FFN_ERR_ALIGN;
  if (const int rc = check_norm_form(form, T, f != nullptr)) return rc;
  if ((!f && df) || (!form->gate && dgate) || (!form->post && dpost_gain) || (!dn && dpre_gain)) return FFN_ERR_OPTION;
  if ((dn && !x_out) || ((dn || form->post) && !rstd)) return FFN_ERR_NULL;
  if (ws_bytes < ffn_norm_workspace_bytes(T, d)) return FFN_ERR_WORKSPACE;

  const int groups = norm_groups(T, d);
  Carver c{static_cast<char*>(ws)};
  float* room[3];
  for (float*& p : room) p = static_cast<float*>(c.take(sizeof(float) * groups * (size_t)d));
  const bool row_gate = dgate && form->gate_rows == 1;
  NormBack a{T, d, form->alpha, form->post, form->gate_sigmoid, form->gate_rows, x_out, f, form->gate, form->post_gain,
             form->pre_gain, rstd, dn, dx_out, dx, df, dgate,
             {dpre_gain ? room[0] : nullptr, dpost_gain ? room[1] : nullptr, row_gate ? room[2] : nullptr}};
  const bool f32 = dt == FFN_F32;
  hipError_t e = f32 ? (d % 4 ? launch_bwd<true, false>(a, groups, stream) : launch_bwd<true, true>(a, groups, stream))
                     : (d % 8 ? launch_bwd<false, false>(a, groups, stream) : launch_bwd<false, true>(a, groups, stream));
  if (e != hipSuccess) return FFN_ERR_HIP;
  NormSums s{groups, d, {}, {}};
  int n = 0;
  void* outs[3] = {dpre_gain, dpost_gain, row_gate ? dgate : nullptr};
  for (int i = 0; i < 3; ++i)
    if (outs[i]) {
      s.part[n] = a.part[i];
      s.out[n++] = outs[i];
    }
  if (n) {
    const dim3 grid(ceil_div(d, 64), n);
    if (f32) k_norm_sums<true><<<grid, 1024, 0, stream>>>(s);
    else k_norm_sums<false><<<grid, 1024, 0, stream>>>(s);
    e = hipGetLastError();
  }
  return e == hipSuccess ? FFN_OK : FFN_ERR_HIP;
}

}  // extern "C"
