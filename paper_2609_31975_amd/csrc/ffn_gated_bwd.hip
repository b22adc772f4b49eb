// The gated block's backward pass: the gradients of the hidden layer, dz = dy W2 with the activations'
// derivatives in its epilogue, and the weight gradients.
#include "ffn_gemm_host.h"

namespace ffn {
namespace {

// dg and dv are rounded once, to the type of the products that read them.  The derivative is taken where g is
// in fp32, so a neuron is on exactly where the forward call had it on.  8192 tokens, 4096 -> 14336: 1070 us, pipes
// 43% busy; a tile's epilogue reads 512 KB and writes 256 KB.
template <class E>
struct EpiDz {
  BlockForm form;
  int d_ff, ldf;
  const float *g, *v;
  typename E::T *dg, *dv;

  __device__ __forceinline__ void select(GemmArgs&) const {}
  __device__ __forceinline__ void pair(int, int, f32x4_t, f32x4_t) const {}
  __device__ __forceinline__ void put(const GemmArgs&, int m, int n, f32x4_t dz) const {
    if (n >= ldf) return;
    const size_t at = (size_t)m * ldf + n;
    const f32x4_t gg = *reinterpret_cast<const f32x4_t*>(g + at), vv = *reinterpret_cast<const f32x4_t*>(v + at);
    f32x4_t og, ov;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, da, u, du;
      block_act_grad(form.act, gg[i], a, da);
      up_grad(form.silu_up, vv[i], u, du);
      const bool in = n + i < d_ff;  // the rest pads the next products' k
      og[i] = in ? dz[i] * u * da : 0.f;
      ov[i] = in ? dz[i] * a * du : 0.f;
    }
    store4<E>(dg + at, og);
    store4<E>(dv + at, ov);
  }
};

// Weight gradient i of a launch: blockIdx.y.  All of them in one launch fill more rounds of the CUs (three of 14336 x
// 4096 over 8192 tokens: 2100 to 2200 us, 1.3 PFLOP/s).
template <class E>
struct EpiDw {
  const void *a[3], *b[3];
  typename E::T* out[3];
  int ldo;
  bool vec;

  __device__ __forceinline__ void select(GemmArgs& g) const {
    g.a.p[0] = a[blockIdx.y];
    g.b.p[0] = b[blockIdx.y];
  }
  __device__ __forceinline__ void pair(int, int, f32x4_t, f32x4_t) const {}
  __device__ __forceinline__ void put(const GemmArgs& g, int m, int n, f32x4_t v) const {
    if (n >= g.N) return;
    typename E::T* o = out[blockIdx.y] + (size_t)m * ldo + n;
    if (vec) {
      store4<E>(o, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < g.N) o[i] = (typename E::T)v[i];
    }
  }
};

template <class E>
hipError_t dz(const BlockShape& s, const void* dy, const void* w_down_t, const BlockForm& form, const float* g,
              const float* v, void* dg, void* dv, float* part, hipStream_t st) {
  GemmArgs a{};
  a.a = Operand{{dy, nullptr}, s.dp, s.T};
  a.b = Operand{{w_down_t, nullptr}, s.dp, s.d_ff};
  a.M = s.T;
  a.N = s.ldf;
  a.K = s.d;
  a.products = 1;
  a.part = part;
  const EpiDz<E> epi{form, s.d_ff, s.ldf, g, v, static_cast<typename E::T*>(dg), static_cast<typename E::T*>(dv)};
  const Plan p = choose_tile(E::EPC == 4, 1, s.T, s.ldf, ceil_div(s.d, step_k<E>()), false, true);
  return with_tile<E>(p.tile, [&](auto c) {
    return launch_gemm<E, decltype(c), Lay::KC, Lay::KC, false, false>(a, epi, p, 1, st);
  });
}

template <class E>
hipError_t dw(const BlockShape& s, int count, const void* const a[3], const void* const b[3], void* const out[3],
              float* part, hipStream_t st) {
  GemmArgs g{};
  g.a = Operand{{nullptr, nullptr}, s.ldf, s.ldf};
  g.b = Operand{{nullptr, nullptr}, s.dp, s.dp};
  g.M = s.d_ff;
  g.N = s.d;
  g.K = s.T;
  g.products = 1;
  g.part = part;
  EpiDw<E> epi{};
  for (int i = 0; i < count; ++i) {
    epi.a[i] = a[i];
    epi.b[i] = b[i];
    epi.out[i] = static_cast<typename E::T*>(out[i]);
  }
  epi.ldo = s.d;
  epi.vec = s.d % 4 == 0;
  const Plan p = choose_tile(E::EPC == 4, count, s.d_ff, s.d, ceil_div(s.T, step_k<E>()), false, false);
  return with_tile<E>(p.tile, [&](auto c) {
    typedef decltype(c) C;
    if constexpr (C::BM >= 64) return launch_gemm<E, C, Lay::KS, Lay::KS, false, false>(g, epi, p, count, st);
    else return hipErrorInvalidValue;  // not reached
  });
}

}  // namespace

hipError_t launch_block_dz(bool f32, const BlockShape& s, const void* dy, const void* w_down_t, const BlockForm& form,
                           const float* g, const float* v, void* dg, void* dv, float* part, hipStream_t st) {
  return f32 ? dz<EF32>(s, dy, w_down_t, form, g, v, dg, dv, part, st) : dz<EBf16>(s, dy, w_down_t, form, g, v, dg, dv, part, st);
}
hipError_t launch_block_dw(bool f32, const BlockShape& s, int count, const void* const a[3], const void* const b[3],
                           void* const out[3], float* part, hipStream_t st) {
  return f32 ? dw<EF32>(s, count, a, b, out, part, st) : dw<EBf16>(s, count, a, b, out, part, st);
}

}  // namespace ffn
