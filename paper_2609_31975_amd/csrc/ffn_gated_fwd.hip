// The hidden layer of the gated block: both projections, the activation and their product in one
// kernel, z = A(x W1^T - t) U(x W3^T).
#include "ffn_gemm_host.h"

namespace ffn {
namespace {

// z is rounded to the type of the next product, which takes no other on the bf16 matrix pipes (y: 2.4e-3 of the
// norm; the output's own rounding alone 1.7e-3).  g and v are saved in fp32: in bf16 they would take 4 bytes a
// hidden value in place of 8, and dg and dv a second rounding (by arithmetic 2.9e-3 in place of 2.4e-3).
//
// What bounds it: the matrix pipes (8192 tokens, 4096 -> 14336, saving: 1600 us, 1.2 PFLOP/s, pipes 62% busy;
// without saving 1.3 PFLOP/s: the epilogue's 320 KB a tile leave while the CU's pipes idle); few tokens: the
// weights' bytes (one token: 40 us, 5.8 TB/s).
template <class E>
struct EpiGated {
  BlockForm form;
  int d_ff, ldf;
  typename E::T* z;
  float *g, *v;  // or null

  __device__ __forceinline__ void select(GemmArgs&) const {}
  __device__ __forceinline__ void put(const GemmArgs&, int, int, f32x4_t) const {}
  __device__ __forceinline__ void pair(int m, int n, f32x4_t h, f32x4_t u) const {
    if (n >= ldf) return;
    const size_t at = (size_t)m * ldf + n;
    f32x4_t gg, zz;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      gg[i] = h[i] - form.t;
      zz[i] = n + i < d_ff ? block_act(form.act, gg[i]) * up_value(form.silu_up, u[i]) : 0.f;
    }
    store4<E>(z + at, zz);
    if (g) {
      *reinterpret_cast<f32x4_t*>(g + at) = gg;
      *reinterpret_cast<f32x4_t*>(v + at) = u;
    }
  }
};

template <class E>
hipError_t hidden(const BlockShape& s, const void* x, const void* w_gate, const void* w_up, const BlockForm& form,
                  const AdapterSet& ad, const void* const v2[2], const void* const b2[2], void* z, float* g, float* v,
                  float* part, hipStream_t st) {
  GemmArgs a{};
  a.a = Operand{{x, nullptr}, s.dp, s.T};
  a.b = Operand{{w_gate, w_up}, s.dp, s.d_ff};
  a.M = s.T;
  a.N = s.d_ff;
  a.K = s.d;
  a.products = 1;
  a.part = part;
  if (ad.plan) a.lr = low_rank(ad, v2, b2, s.d_ff);
  const EpiGated<E> epi{form, s.d_ff, s.ldf, static_cast<typename E::T*>(z), g, v};
  const Plan plan = hidden_plan(E::EPC == 4, s, ad.plan != nullptr);
  return with_tile<E>(plan.tile, [&](auto c) {
    return launch_with_adapters<E, decltype(c), Lay::KC, Lay::KC, true>(a, epi, plan, st);
  });
}

}  // namespace

hipError_t launch_block_hidden(bool f32, const BlockShape& s, const void* x, const void* w_gate, const void* w_up,
                               const BlockForm& form, const AdapterSet& ad, const void* const v2[2],
                               const void* const b2[2], void* z, float* g, float* v, float* part, hipStream_t st) {
  return f32 ? hidden<EF32>(s, x, w_gate, w_up, form, ad, v2, b2, z, g, v, part, st)
             : hidden<EBf16>(s, x, w_gate, w_up, form, ad, v2, b2, z, g, v, part, st);
}

}  // namespace ffn
