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
    f32x4_t v = *reinterpret_cast<const f32x4_t*>(p);
    for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4_t*>(p + s * plane);
    typename E::T* o = out + (size_t)m * ldo + n;
    if (N % 4 == 0) {
      store4<E>(o, v);
    } else {
      for (int k = 0; k < 4; ++k)
        if (n + k < N) o[k] = (typename E::T)v[k];
    }
  }
}

template <class E, class C, Lay LB>
hipError_t run(const GemmArgs& a, const EpiTok<E>& epi, hipStream_t st) {
  return a.lr.ids ? launch_gemm<E, C, Lay::KC, LB, false, true>(a, epi, 1, st)
                  : launch_gemm<E, C, Lay::KC, LB, false, false>(a, epi, 1, st);
}

enum class TokTile { T16, T64, T128, T256 };
TokTile tile_for(bool f32, int T, int n) {
  if (T <= 16) return TokTile::T16;
  if (T <= 64) return TokTile::T64;
  if (!f32 && (int64_t)ceil_div(T, 256) * ceil_div(n, 256) >= kCUs) return TokTile::T256;
  return TokTile::T128;
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
  a.splits = token_splits(E::EPC == 4, p.T, p.n, p.products * ceil_div(p.k, step_k<E>()));
  const void *v[2] = {p.v, nullptr}, *b[2] = {p.ab, nullptr};
  if (p.ad.ids) a.lr = low_rank(p.ad, v, b, p.n);
  const int np = (p.n + 3) / 4 * 4;
  const EpiTok<E> epi{static_cast<typename E::T*>(p.out), p.part, p.ldo, np, p.n % 4 == 0};
  hipError_t e;
  switch (tile_for(E::EPC == 4, p.T, p.n)) {
    case TokTile::T16: e = run<E, TileT16, LB>(a, epi, st); break;
    case TokTile::T64: e = run<E, TileT64, LB>(a, epi, st); break;
    case TokTile::T128: e = run<E, TileT128, LB>(a, epi, st); break;
    default:
      if constexpr (E::EPC == 8) e = run<E, TileT256, LB>(a, epi, st);
      else e = hipErrorInvalidValue;  // not reached: tile_for gives fp32 at most T128
  }
  if (e == hipSuccess && a.splits > 1) {
    const int64_t quads = (int64_t)p.T * np / 4;
    const int grid = (int)(quads / kBlock + 1 < 8 * kCUs ? quads / kBlock + 1 : 8 * kCUs);
    k_join<E><<<grid, kBlock, 0, st>>>(a.splits, p.T, p.n, np, p.ldo, p.part, static_cast<typename E::T*>(p.out));
    e = hipGetLastError();
  }
  return e;
}

// ------------------------------------------------------------------ the adapters' first factor
// v[m][k] = scale_j <A_j[k], x[m]>, j the adapter of token m.  A workgroup takes 16 tokens, one of
// the adapters among them (blockIdx.x % 16; most find no such adapter and end) and 16 of the ranks; its
// 16 waves share the row, each with loads of its own from memory to fragments, and are joined in LDS.
// A product serves all 16 tokens, and those with another adapter are dropped.
constexpr int kVWaves = 16;
struct AdapterV {
  const void* x;
  const void* a[2];
  void* v[2];
  const int32_t* ids;
  const float* scale;
  int T, k, ldx, n, r, rp;
};
template <class E>
__global__ void __launch_bounds__(kVWaves * kWave) k_adapter_v(AdapterV p) {
  typedef typename E::T T;
  __shared__ f32x4_t sum[kVWaves][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int m0 = (int)(blockIdx.x / 16) * 16, which = blockIdx.x % 16, k0 = blockIdx.y * 16;
  const int m = m0 + (lane & 15);
  int id = m < p.T ? p.ids[m] : -1;
  if (id < 0 || id >= p.n) id = -1;
  // the which-th adapter of the 16 tokens, in the order of its first token
  bool first = id >= 0 && lane < 16;
  for (int s = 0; s < 15; ++s)
    if (__shfl(id, s) == id && s < lane) first = false;
  uint64_t firsts = __ballot(first);
  for (int s = 0; s < which && firsts; ++s) firsts &= firsts - 1;
  if (!firsts) return;
  const int j = __shfl(id, __ffsll((unsigned long long)firsts) - 1);

  const bool whole = p.k % E::EPC == 0;
  const int col = k0 + (lane & 15), c0 = lane >> 4;
  const T* x = static_cast<const T*>(p.x) + (size_t)(m < p.T ? m : m0) * p.ldx;
  const T* a = static_cast<const T*>(p.a[blockIdx.z]) + ((size_t)j * p.r + (col < p.r ? col : 0)) * p.k;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  const int steps = (p.k + 4 * E::EPC - 1) / (4 * E::EPC);
  constexpr int U = 8;  // steps in flight
  for (int s0 = wave; s0 < steps; s0 += kVWaves * U) {
    uint4 xv[U], av[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = ((s0 + u * kVWaves) * 4 + c0) * E::EPC;
      xv[u] = k < p.k ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
      av[u] = load_part<E>(a + k, p.k - k, whole);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = product<E>(av[u], xv[u], acc);
  }
  sum[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && id == j) {
    for (int w = 1; w < kVWaves; ++w) acc += sum[w][lane];
    const float sc = p.scale ? p.scale[j] : 1.f;
    const int c = k0 + 4 * c0;
    if (c < p.rp) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = c + i < p.r ? acc[i] * sc : 0.f;
      store4<E>(static_cast<T*>(p.v[blockIdx.z]) + (size_t)m * p.rp + c, acc);
    }
  }
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

// Shares of a sum over `steps` steps: a product with too few tiles for the CUs is cut along k, so that
// about two workgroups fall on a CU, but no share is under 4 steps (a share writes its whole tile in fp32).
int token_splits(bool f32, int T, int n, int steps) {
  const TokTile t = tile_for(f32, T, n);
  if (t == TokTile::T256) return 1;
  const int bm = t == TokTile::T16 ? 16 : t == TokTile::T64 ? 64 : 128;
  const int64_t tiles = (int64_t)ceil_div(T, bm) * ceil_div(n, 128);
  if (tiles >= kCUs) return 1;
  int s = (int)(2 * kCUs / tiles);
  if (s > steps / 4) s = steps / 4;
  return s < 1 ? 1 : s > 32 ? 32 : s;
}

hipError_t launch_token_product_ks(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KS>(p, st) : product<EBf16, Lay::KS>(p, st);
}
hipError_t launch_token_product_kc(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KC>(p, st) : product<EBf16, Lay::KC>(p, st);
}

hipError_t launch_adapter_v(bool f32, int T, int k, int ldx, const void* x, const AdapterSet& ad, int count,
                            const void* const a[2], void* const v[2], hipStream_t st) {
  const AdapterV p{x, {a[0], a[1]}, {v[0], v[1]}, ad.ids, ad.scale, T, k, ldx, ad.n, ad.r, ad.rp};
  const dim3 grid(ceil_div(T, 16) * 16, ceil_div(ad.rp, 16), count);
  if (f32) k_adapter_v<EF32><<<grid, kVWaves * kWave, 0, st>>>(p);
  else k_adapter_v<EBf16><<<grid, kVWaves * kWave, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t launch_pad_rows(bool f32, int64_t rows, int n, int np, const void* src, void* dst, hipStream_t st) {
  const int64_t want = rows * np / 8 / kBlock + 1;
  const int grid = (int)(want < 32 * kCUs ? want : 32 * kCUs);
  if (f32) k_pad_rows<EF32><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const float*>(src), static_cast<float*>(dst));
  else k_pad_rows<EBf16><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const __bf16*>(src), static_cast<__bf16*>(dst));
  return hipGetLastError();
}

}  // namespace ffn
