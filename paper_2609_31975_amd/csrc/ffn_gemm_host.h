// Host side of the tiled product: tile shapes and launches.  Not part of the public ABI.
#pragma once

#include "ffn_gated_internal.h"
#include "ffn_gemm.h"

namespace ffn {
namespace {

// Tiles: tokens (or weight-gradient rows) x columns, waves, steps in LDS.
//   16, 64      a few tokens: the weights are streamed past them, 2 to 4 workgroups a CU (28672 x 4096 bf16
//               weights, 1..48 tokens: 36 to 38 us, 6.4 TB/s; 128 columns a tile 38 to 40)
//   64, 64x128  fp32, any number of tokens: the fp32 products bound it (512 x 28460 x
//               3840, k contiguous in both: 123 and 138 TFLOP/s, the card's library product 133; a training
//               step over 513 tokens, most of whose products read a strided operand by element, 112), and
//               small tiles waste the least of odd sizes
//   128, 128x256, 256  bf16, many tokens: 1030, 1150 and 1300 TFLOP/s where the tiles fill the chip
//               (8192 x 4096 x 14336; the card's library product reaches 1360 to 1480)
typedef Config<16, 64, 1, 2, 4> Tile16;
typedef Config<64, 64, 2, 2, 3> Tile64;
typedef Config<64, 128, 2, 4, 2> Tile64x128;
typedef Config<128, 128, 2, 2, 2> Tile128;
typedef Config<128, 256, 2, 4, 3> Tile128x256;
typedef Config<256, 256, 2, 4, 2> Tile256;

inline int ceil_div(int a, int b) { return (int)(((int64_t)a + b - 1) / b); }

// plan.cut counts the tiles of all `problems` results, each of which has its own grid row.
template <class E, class C, Lay LA, Lay LB, bool DUAL, bool AD, class Epi>
hipError_t launch_gemm(GemmArgs g, const Epi& epi, const Plan& plan, int problems, hipStream_t st) {
  g.ntm = ceil_div(g.M, C::BM);
  g.ntn = ceil_div(g.N, DUAL ? C::BN / 2 : C::BN);
  const int tiles = g.ntm * g.ntn, cut = plan.cut / problems;
  g.whole = tiles - cut;
  g.shares = plan.shares;
  const int grid = g.whole + cut * plan.shares;
  k_gemm<E, C, LA, LB, DUAL, AD, Epi><<<dim3(grid, problems), C::threads, 0, st>>>(g, epi);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || cut == 0) return e;
  k_join<C, DUAL, Epi><<<dim3(cut, problems, C::MT), C::threads, 0, st>>>(g, epi);
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

// The tiles that products with adapters are built for, and so the ones that choose_tile picks for them
// (takes_adapters): the adapters' sums beside Tile256's need more registers than there are, and Tile128 holds too few
// steps to load the adapters ahead (3000 tokens, 4096 x 4096, rank 64: the call 173 us, 131 in Tile128x256; fp32
// products take so much longer that it does not show in Tile64x128).
template <class C>
constexpr bool adapter_tile() {
  return C::S >= 3 || C::BM == 64;
}

inline LowRank low_rank(const AdapterSet& ad, const void* const v[2], const void* const b[2], int out) {
  return LowRank{{v[0], v[1]}, {b[0], b[1]}, ad.plan, ad.r, ad.rp, out};
}

// f(Config{}) for the tile that choose_tile picked; a tile of the other type is an error
template <class E, class F>
hipError_t with_tile(Tile t, F f) {
  switch (t) {
    case Tile::T16: return f(Tile16{});
    case Tile::T64: return f(Tile64{});
    default: break;
  }
  if constexpr (E::EPC == 8) {
    if (t == Tile::T128) return f(Tile128{});
    if (t == Tile::T128x256) return f(Tile128x256{});
    if (t == Tile::T256) return f(Tile256{});
  } else {
    if (t == Tile::T64x128) return f(Tile64x128{});
  }
  return hipErrorInvalidValue;
}

// The product with adapters, or without where a.lr has none.  A plan for adapters whose tile has none built is an
// error: the product without them would be a wrong result.
template <class E, class C, Lay LA, Lay LB, bool DUAL, class Epi>
hipError_t launch_with_adapters(const GemmArgs& a, const Epi& epi, const Plan& plan, hipStream_t st) {
  if (!a.lr.plan) return launch_gemm<E, C, LA, LB, DUAL, false>(a, epi, plan, 1, st);
  if constexpr (adapter_tile<C>()) return launch_gemm<E, C, LA, LB, DUAL, true>(a, epi, plan, 1, st);
  else return hipErrorInvalidValue;
}

}  // namespace
}  // namespace ffn
