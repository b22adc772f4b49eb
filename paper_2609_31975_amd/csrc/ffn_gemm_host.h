// Host side of the tiled product: tile shapes and launches.  Not part of the public ABI.
#pragma once

#include "ffn_gated_internal.h"
#include "ffn_gemm.h"

namespace ffn {
namespace {

// Tiles: tokens (or weight-gradient rows) x columns, waves, steps in LDS.
typedef Config<16, 128, 1, 4, 4> TileT16;    // a decode step: weights streamed, 3 steps in flight
typedef Config<64, 128, 1, 4, 4> TileT64;
typedef Config<128, 128, 2, 2, 2> TileT128;
typedef Config<256, 256, 2, 4, 2> TileT256;

inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

template <class E, class C, Lay LA, Lay LB, bool DUAL, bool AD, class Epi>
hipError_t launch_gemm(GemmArgs g, const Epi& epi, int problems, hipStream_t st) {
  g.ntm = ceil_div(g.M, C::BM);
  g.ntn = ceil_div(g.N, DUAL ? C::BN / 2 : C::BN);
  k_gemm<E, C, LA, LB, DUAL, AD, Epi><<<dim3(g.ntm * g.ntn * g.splits, problems), C::threads, 0, st>>>(g, epi);
  return hipGetLastError();
}

template <class E>
struct Four {
  typename E::T v[4];
};
template <class E>
__device__ __forceinline__ void store4(typename E::T* p, f32x4_t x) {
  Four<E> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = (typename E::T)x[i];
  if constexpr (E::EPC == 8) *reinterpret_cast<uint2*>(p) = __builtin_bit_cast(uint2, o);
  else *reinterpret_cast<uint4*>(p) = __builtin_bit_cast(uint4, o);
}

inline LowRank low_rank(const AdapterSet& ad, const void* const v[2], const void* const b[2], int out) {
  return LowRank{{v[0], v[1]}, {b[0], b[1]}, ad.ids, ad.n, ad.r, ad.rp, out};
}

}  // namespace
}  // namespace ffn
