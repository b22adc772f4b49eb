// Products with a row for every token: y = z W2t, dx = dg W1 + dv W3, and one shared projection
// x W^T, with adapters; the adapters' first factor A_j x; padded copies of odd rows.
#include "ffn_gemm_host.h"

namespace ffn {
namespace {

template <class E>
struct EpiTok {
  typename E::T* out;
  float* part;  // of a split sum
  int ldo, np;
  bool vec;  // rows of whole quads

  __device__ __forceinline__ void select(GemmArgs&) const {}
  __device__ __forceinline__ void pair(int, int, f32x4_t, f32x4_t) const {}
  __device__ __forceinline__ void put(const GemmArgs& g, int split, int m, int n, f32x4_t v) const {
    if (n >= g.N) return;
    if (g.splits > 1) {
      *reinterpret_cast<f32x4_t*>(part + ((size_t)split * g.M + m) * np + n) = v;
      return;
    }
    typename E::T* o = out + (size_t)m * ldo + n;
    if (vec) {
      store4<E>(o, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < g.N) o[i] = (typename E::T)v[i];
    }
  }
};

// out[m][n] = sum of the shares, in their order
template <class E>
__global__ void __launch_bounds__(kBlock) k_join(int splits, int M, int N, int np, int ldo, const float* part,
                                                 typename E::T* out) {
  const int q = np / 4;
  const size_t total = (size_t)M * q, plane = (size_t)M * np;
  for (size_t i = (size_t)blockIdx.x * kBlock + threadIdx.x; i < total; i += (size_t)gridDim.x * kBlock) {
    const int m = (int)(i / q), n = (int)(i - (size_t)m * q) * 4;
    const float* p = part + (size_t)m * np + n;
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < splits; s0 += 8) {  // 8 loads in flight
      f32x4_t u[8];
#pragma unroll
      for (int s = 0; s < 8; ++s)
        u[s] = s0 + s < splits ? *reinterpret_cast<const f32x4_t*>(p + (s0 + s) * plane) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 8; ++s) v += u[s];
    }
    typename E::T* o = out + (size_t)m * ldo + n;
    if (N % 4 == 0) {
      store4<E>(o, v);
    } else {
      for (int k = 0; k < 4; ++k)
        if (n + k < N) o[k] = (typename E::T)v[k];
    }
  }
}

template <class E, Lay LB>
hipError_t product(const TokenProduct& p, hipStream_t st) {
  GemmArgs a{};
  a.a = Operand{{p.a[0], p.a[1]}, p.lda, p.T};
  a.b = Operand{{p.b[0], p.b[1]}, p.ldb, LB == Lay::KS ? p.ldb : p.n};
  a.M = p.T;
  a.N = p.n;
  a.K = p.k;
  a.products = p.products;
  const Plan plan = token_plan(E::EPC == 4, p.T, p.n, p.k, p.products);
  a.splits = plan.splits;
  const void *v[2] = {p.v, nullptr}, *b[2] = {p.ab, nullptr};
  if (p.ad.plan) a.lr = low_rank(p.ad, v, b, p.n);
  const int np = (p.n + 3) / 4 * 4;
  const EpiTok<E> epi{static_cast<typename E::T*>(p.out), p.part, p.ldo, np, p.n % 4 == 0};
  hipError_t e = with_tile<E>(plan.tile, [&](auto c) {
    typedef decltype(c) C;
    return a.lr.plan ? launch_gemm<E, C, Lay::KC, LB, false, true>(a, epi, 1, st)
                     : launch_gemm<E, C, Lay::KC, LB, false, false>(a, epi, 1, st);
  });
  if (e == hipSuccess && a.splits > 1) {
    const int64_t quads = (int64_t)p.T * np / 4;
    const int grid = (int)(quads / kBlock + 1 < 8 * kCUs ? quads / kBlock + 1 : 8 * kCUs);
    k_join<E><<<grid, kBlock, 0, st>>>(a.splits, p.T, p.n, np, p.ldo, p.part, static_cast<typename E::T*>(p.out));
    e = hipGetLastError();
  }
  return e;
}

// ------------------------------------------------------------------ the adapters' first factor
// v[m][k] = scale_j <A_j[k], x[m]>, j the adapter of token m.  A workgroup takes 16 tokens, 16 RC of
// the ranks, and of the adapters among its tokens every lanes-th from the blockIdx.x % lanes-th on (one
// each where there are few tokens, all of them where there are many); its waves share the row, each
// with loads of its own from memory to fragments, and are joined in LDS.  A product serves all 16 tokens,
// and those with another adapter are dropped.
//
// The last workgroups (one for each tile of bm tokens) make the plan of the product that reads v.
struct AdapterV {
  const void* x;
  const void* a[2];
  void* v[2];
  const int32_t* ids;
  const float* scale;
  int32_t* plan;
  int T, k, ldx, n, r, rp, lanes, blocks, bm;
};

__device__ __forceinline__ int id_of(const AdapterV& p, int m) {
  const int id = m < p.T ? p.ids[m] : -1;
  return id >= 0 && id < p.n ? id : -1;
}

// Tile `tile` of the plan (LowRank): a token's first token with the same adapter, then that one's place
// among the firsts.
template <int THREADS>
__device__ void make_plan(const AdapterV& p, int tile) {
  __shared__ int ids[256], first[256], place[256], heads[4];
  const int t = threadIdx.x, bm = p.bm;
  if (t < 256) ids[t] = t < bm ? id_of(p, tile * bm + t) : -1;
  __syncthreads();
  if (t < 256) {
    int f = t;
    for (int s = 255; s >= 0; --s)
      if (s < bm && ids[s] == ids[t] && s < f) f = s;
    first[t] = ids[t] >= 0 ? f : -1;
    const uint64_t b = __ballot(first[t] == t);
    place[t] = rank_in_mask(b);
    if (lane_id() == 0) heads[t / kWave] = __popcll(b);
  }
  __syncthreads();
  int32_t* out = p.plan + (size_t)tile * (1 + 2 * bm);
  if (t == 0) out[0] = heads[0] + heads[1] + heads[2] + heads[3];
  if (t < bm) {
    int at = -1;
    if (first[t] >= 0) {
      at = place[first[t]];
      for (int w = 0; w < first[t] / kWave; ++w) at += heads[w];
      if (first[t] == t) out[1 + at] = ids[t];
    }
    out[1 + bm + t] = at;
  }
}

template <class E, int NW, int RC>
__global__ void __launch_bounds__(NW * kWave) k_adapter_v(AdapterV p) {
  typedef typename E::T T;
  if ((int)blockIdx.x >= p.blocks) {
    if (blockIdx.y == 0 && blockIdx.z == 0) make_plan<NW * kWave>(p, (int)blockIdx.x - p.blocks);
    return;
  }
  __shared__ f32x4_t sum[NW][RC][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int m0 = (int)blockIdx.x / p.lanes * 16, k0 = blockIdx.y * 16 * RC;
  const int m = m0 + (lane & 15), id = id_of(p, m);
  bool first = id >= 0 && lane < 16;
  for (int s = 0; s < 15; ++s)
    if (__shfl(id, s) == id && s < lane) first = false;
  uint64_t firsts = __ballot(first);
  const bool whole = p.k % E::EPC == 0;
  const int c0 = lane >> 4;
  const T* x = static_cast<const T*>(p.x) + (size_t)(m < p.T ? m : m0) * p.ldx;
  const int steps = (p.k + 4 * E::EPC - 1) / (4 * E::EPC);
  for (int w = 0; firsts; ++w) {
    const int j = __shfl(id, __ffsll((unsigned long long)firsts) - 1);
    firsts &= firsts - 1;
    if (w % p.lanes != (int)blockIdx.x % p.lanes) continue;
    const T* a[RC];
    f32x4_t acc[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c) {
      const int col = k0 + 16 * c + (lane & 15);
      a[c] = static_cast<const T*>(p.a[blockIdx.z]) + ((size_t)j * p.r + (col < p.r ? col : 0)) * p.k;
      acc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int U = RC == 1 ? 8 : 4;  // steps in flight
    for (int s0 = wave; s0 < steps; s0 += NW * U) {
      uint4 xv[U], av[U][RC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = ((s0 + u * NW) * 4 + c0) * E::EPC;
        xv[u] = k < p.k ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < RC; ++c) av[u][c] = load_part<E>(a[c] + k, p.k - k, whole);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int c = 0; c < RC; ++c) acc[c] = product<E>(av[u][c], xv[u], acc[c]);
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < RC; ++c) sum[wave][c][lane] = acc[c];
    __syncthreads();
    if (wave < RC && id == j) {
      f32x4_t v = sum[0][wave][lane];
      for (int s = 1; s < NW; ++s) v += sum[s][wave][lane];
      const float sc = p.scale ? p.scale[j] : 1.f;
      const int c = k0 + 16 * wave + 4 * c0;
      if (c < p.rp) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < p.r ? v[i] * sc : 0.f;
        store4<E>(static_cast<T*>(p.v[blockIdx.z]) + (size_t)m * p.rp + c, v);
      }
    }
  }
}

template <class E>
hipError_t adapter_v(AdapterV p, int count, hipStream_t st) {
  const int tiles = ceil_div(p.T, 16), plans = ceil_div(p.T, p.bm);
  if (tiles * count >= kCUs / 2) {
    // many tokens: a workgroup for 16 of them and 64 ranks, all their adapters in turn
    p.lanes = 1;
    p.blocks = tiles;
    k_adapter_v<E, 4, 4><<<dim3(p.blocks + plans, ceil_div(p.rp, 64), count), 4 * kWave, 0, st>>>(p);
  } else {
    p.lanes = p.T < 16 ? p.T : 16;
    p.blocks = tiles * p.lanes;
    k_adapter_v<E, 16, 1><<<dim3(p.blocks + plans, ceil_div(p.rp, 16), count), 16 * kWave, 0, st>>>(p);
  }
  return hipGetLastError();
}

template <class E>
__global__ void __launch_bounds__(kBlock) k_pad_rows(int64_t rows, int n, int np, const typename E::T* src,
                                                     typename E::T* dst) {
  const int q = np / E::EPC;
  const size_t total = (size_t)rows * q;
  for (size_t i = (size_t)blockIdx.x * kBlock + threadIdx.x; i < total; i += (size_t)gridDim.x * kBlock) {
    const size_t r = i / q;
    const int c = (int)(i - r * q) * E::EPC;
    *reinterpret_cast<uint4*>(dst + r * np + c) = load_part<E>(src + r * n + c, n - c, false);
  }
}

}  // namespace

int tile_rows(Tile t) {
  switch (t) {
    case Tile::T16: return Tile16::BM;
    case Tile::T64: return Tile64::BM;
    case Tile::T256: return Tile256::BM;
    default: return Tile128::BM;
  }
}

// By an estimate of the time, in us.  A product of more rows than a few tokens runs in rounds of tiles over
// the CUs; a step of a round takes what was measured at sizes that fill the chip (two workgroups of 128 x
// 128 share a CU; a lone one takes 0.66), a tile 6 us for its first loads and its stores.  Cutting the sum
// in shares fills rounds that would stay empty; the shares' fp32 tiles are written and read once more, and
// joined by a second launch.
Plan choose_tile(bool f32, int64_t M, int64_t n, int steps, bool split) {
  auto cut = [&](int64_t tiles, int slots, int least) {  // shares of at least `least` steps that fill the slots
    int64_t s = split ? slots / tiles : 1;
    if (s > steps / least) s = steps / least;
    return (int)(s < 1 ? 1 : s > 32 ? 32 : s);
  };
  auto tiles = [&](int bm, int bn) { return ((M + bm - 1) / bm) * ((n + bn - 1) / bn); };
  if (M <= 16) return Plan{Tile::T16, cut(tiles(16, 64), 2 * kCUs, 8)};
  if (M <= 64 || f32) return Plan{Tile::T64, cut(tiles(64, 64), 2 * kCUs, 8)};
  struct Kind {
    Tile t;
    int bm, bn, a_cu;
    double step_us, lone_us;
  };
  static const Kind kinds[] = {{Tile::T256, 256, 256, 1, 1.45, 1.45},
                               {Tile::T128x256, 128, 256, 1, 0.82, 0.82},
                               {Tile::T128, 128, 128, 2, 1.04, 0.66}};
  Plan best{Tile::T256, 1};
  double least = 1e30;
  for (const Kind& k : kinds) {
    const int64_t nt = tiles(k.bm, k.bn);
    const int s = cut(nt, kCUs * k.a_cu, 16);
    const int64_t rounds = (nt * s + kCUs * k.a_cu - 1) / (kCUs * k.a_cu);
    const double step = nt * s <= kCUs ? k.lone_us : k.step_us;
    const double us = rounds * (step * ((steps + s - 1) / s) + 6.0) + (s > 1 ? 5.0 + 8e-6 * (double)(M * n) * s / 5.0 : 0.0);
    if (us < least) {
      least = us;
      best = Plan{k.t, s};
    }
  }
  return best;
}

Plan token_plan(bool f32, int T, int n, int k, int products) {
  return choose_tile(f32, T, n, products * ceil_div(k, f32 ? step_k<EF32>() : step_k<EBf16>()), true);
}
Plan hidden_plan(bool f32, const BlockShape& s) {
  return choose_tile(f32, s.T, 2 * (int64_t)s.d_ff, ceil_div(s.d, f32 ? step_k<EF32>() : step_k<EBf16>()), false);
}

hipError_t launch_token_product_ks(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KS>(p, st) : product<EBf16, Lay::KS>(p, st);
}
hipError_t launch_token_product_kc(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KC>(p, st) : product<EBf16, Lay::KC>(p, st);
}

hipError_t launch_adapter_v(bool f32, int T, int k, int ldx, const void* x, const AdapterSet& ad, int count,
                            const void* const a[2], void* const v[2], Tile t, hipStream_t st) {
  const AdapterV p{x, {a[0], a[1]}, {v[0], v[1]}, ad.ids, ad.scale, ad.plan, T, k, ldx, ad.n, ad.r, ad.rp, 0, 0, tile_rows(t)};
  return f32 ? adapter_v<EF32>(p, count, st) : adapter_v<EBf16>(p, count, st);
}

hipError_t launch_pad_rows(bool f32, int64_t rows, int n, int np, const void* src, void* dst, hipStream_t st) {
  const int64_t want = rows * np / 8 / kBlock + 1;
  const int grid = (int)(want < 32 * kCUs ? want : 32 * kCUs);
  if (f32) k_pad_rows<EF32><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const float*>(src), static_cast<float*>(dst));
  else k_pad_rows<EBf16><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const __bf16*>(src), static_cast<__bf16*>(dst));
  return hipGetLastError();
}

}  // namespace ffn
