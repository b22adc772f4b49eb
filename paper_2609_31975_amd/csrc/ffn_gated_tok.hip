// Products with a row for every token: y = z W2t, dx = dg W1 + dv W3, and one shared projection
// x W^T, with adapters; the adapters' first factor A_j x; padded copies of odd rows.
#include "ffn_gemm_host.h"

namespace ffn {

// Shares of a row, at most 8 (k_adapter_join), so that a few workgroups come to a CU; a share is at least
// half a round of loads of k_adapter_v's 16 waves, or 8 steps of k_adapter_v_tiles.
size_t adapter_share_bytes_most(int T, int rp, int count) {
  const int few = 16 * 3 * kCUs;  // beyond, one share
  return (size_t)8 * count * (T < few ? T : few) * rp * 4;
}
AdapterPlan adapter_plan(bool f32, int T, int k, int rp, int count) {
  const int groups = ceil_div(T, 16);
  AdapterPlan p;
  // through LDS tiles with many tokens, and rows of whole chunks
  p.tiles = (int64_t)groups * count >= kCUs / 2 && k % (f32 ? 4 : 8) == 0;
  // most tiles of many tokens hold a prompt's, of one request or of two
  p.lanes = p.tiles ? 2 : T < 16 ? T : 16;
  const int step = f32 ? 16 : 32;  // k of a product
  const int steps = ceil_div(k, step);
  const int64_t all = (int64_t)groups * count * (p.tiles ? ceil_div(rp, 64) : (int64_t)p.lanes * ceil_div(rp, 16));
  int64_t s = (p.tiles ? 3 : 2) * kCUs / all;
  if (s > steps / (p.tiles ? 16 : 64)) s = steps / (p.tiles ? 16 : 64);
  p.shares = (int)(s < 1 ? 1 : s > 8 ? 8 : s);
  p.blocks = groups * p.lanes * p.shares;
  return p;
}

namespace {

template <class E>
struct EpiTok {
  typename E::T* out;
  int ldo;
  bool vec;  // rows of whole quads

  __device__ __forceinline__ void select(GemmArgs&) const {}
  __device__ __forceinline__ void pair(int, int, f32x4_t, f32x4_t) const {}
  __device__ __forceinline__ void put(const GemmArgs& g, int m, int n, f32x4_t v) const {
    if (n >= g.N) return;
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

template <class E, Lay LB>
hipError_t product(const TokenProduct& p, hipStream_t st) {
  GemmArgs a{};
  a.a = Operand{{p.a[0], p.a[1]}, p.lda, p.T};
  a.b = Operand{{p.b[0], p.b[1]}, p.ldb, LB == Lay::KS ? p.ldb : p.n};
  a.M = p.T;
  a.N = p.n;
  a.K = p.k;
  a.products = p.products;
  const Plan plan = token_plan(E::EPC == 4, p.T, p.n, p.k, p.products, p.ad.plan != nullptr);
  a.part = p.part;
  const void *v[2] = {p.v, nullptr}, *b[2] = {p.ab, nullptr};
  if (p.ad.plan) a.lr = low_rank(p.ad, v, b, p.n);
  const EpiTok<E> epi{static_cast<typename E::T*>(p.out), p.ldo, p.n % 4 == 0};
  return with_tile<E>(plan.tile, [&](auto c) {
    return launch_with_adapters<E, decltype(c), Lay::KC, LB, false>(a, epi, plan, st);
  });
}

// ------------------------------------------------------------------ the adapters' first factor
// v[m][k] = scale_j <A_j[k], x[m]>, j the adapter of token m.  A workgroup takes 16 tokens, some of the
// ranks, a share of the row, and of the adapters among its tokens every lanes-th from its own on.  A product
// serves all 16 tokens, and those with another adapter are dropped.
//
// Few tokens (k_adapter_v): 16 ranks, one adapter each, the row over 16 waves with loads of their own from
// memory to fragments, joined in LDS.  One CU alone reads a row slowly, so the row is cut in `shares` over
// workgroups too: these write fp32 sums, and k_adapter_join adds them up (16 tokens with an adapter each, rank
// 16, rows of 14336: 33 us in one share, 9 + 4 us in 7).
//
// Many tokens (k_adapter_v_tiles): 64 ranks through the pipeline of the tiled product.  A fragment loaded
// from memory takes 16 bytes of 16 rows at a time, a quarter of the cache's rate, which these hit (3000
// tokens, rank 64, rows of 4096: 39 us, through LDS 16 + 5).
//
// The plan of the product that reads v is made by the last workgroups (one for each tile of bm tokens) of
// k_adapter_v with one share, else of k_adapter_join.
struct AdapterV {
  const void* x;
  const void* a[2];
  void* v[2];
  const int32_t* ids;
  const float* scale;
  int32_t* plan;
  float* part;  // [shares][count][T][rp]
  int T, k, ldx, n, r, rp, lanes, blocks, bm, shares, count;
};

__device__ __forceinline__ int id_of(const AdapterV& p, int m) {
  const int id = m < p.T ? p.ids[m] : -1;
  return id >= 0 && id < p.n ? id : -1;
}

// Tile `tile` of the plan (LowRank): a token's first token with the same adapter, then that one's place
// among the firsts.  At least 256 threads.
__device__ void make_plan(const AdapterV& p, int tile) {
  __shared__ int ids[256], place[256], heads[4];
  const int t = threadIdx.x, bm = p.bm;
  const int id = t < bm ? id_of(p, tile * bm + t) : -1;
  if (t < 256) ids[t] = id;
  __syncthreads();
  int first = -1;
  if (t < 256) {
    if (id >= 0) first = t;
#pragma unroll 8
    for (int s = bm - 1; s >= 0; --s)
      if (ids[s] == id && s < first) first = s;
    const uint64_t b = __ballot(first == t);
    place[t] = rank_in_mask(b);
    if (lane_id() == 0) heads[t / kWave] = __popcll(b);
  }
  __syncthreads();
  int32_t* out = p.plan + (size_t)tile * (1 + 2 * bm);
  if (t == 0) out[0] = heads[0] + heads[1] + heads[2] + heads[3];
  if (t < bm) {
    int at = -1;
    if (first >= 0) {
      at = place[first];
      for (int w = 0; w < first / kWave; ++w) at += heads[w];
      if (first == t) out[1 + at] = id;
    }
    out[1 + bm + t] = at;
  }
}

// v is rounded to the type of the product that reads it (bf16: an adapter that moves its projection by a fifth
// adds 0.2 x 1.7e-3 to an output whose own rounding is 1.7e-3).
template <class E>
__device__ __forceinline__ void put_v(const AdapterV& p, int which, int m, int c, int id, f32x4_t v) {
  const float sc = p.scale ? p.scale[id] : 1.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = c + i < p.r ? v[i] * sc : 0.f;
  store4<E>(static_cast<typename E::T*>(p.v[which]) + (size_t)m * p.rp + c, v);
}

// The adapters of the 16 tokens from m0 on, one after the other (the lowest token of each): a mask over
// the lanes below 16 that hold their first token.
__device__ __forceinline__ uint64_t first_tokens(int id) {
  const int lane = lane_id();
  bool first = id >= 0 && lane < 16;
#pragma unroll
  for (int s = 0; s < 15; ++s)
    if (__builtin_amdgcn_readlane(id, s) == id && s < lane) first = false;
  return __ballot(first);
}

template <class E>
__device__ __forceinline__ void put_share(const AdapterV& p, int share, int which, int m, int c, int id, f32x4_t v) {
  if (p.shares == 1)
    put_v<E>(p, which, m, c, id, v);
  else
    *reinterpret_cast<f32x4_t*>(p.part + (((size_t)share * p.count + which) * p.T + m) * p.rp + c) = v;
}

// WHOLE: rows of whole chunks
constexpr int kVWaves = 16;
template <class E, bool WHOLE>
__global__ void __launch_bounds__(kVWaves * kWave) k_adapter_v(AdapterV p) {
  typedef typename E::T T;
  if ((int)blockIdx.x >= p.blocks) {
    if (blockIdx.y == 0 && blockIdx.z == 0) make_plan(p, (int)blockIdx.x - p.blocks);
    return;
  }
  __shared__ f32x4_t sum[kVWaves][kWave];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int share = (int)blockIdx.x % p.shares, block = (int)blockIdx.x / p.shares;
  const int m0 = block / p.lanes * 16, k0 = blockIdx.y * 16;
  const int m = m0 + (lane & 15), id = id_of(p, m);
  uint64_t firsts = first_tokens(id);
  const int c0 = lane >> 4, col = k0 + (lane & 15);
  const T* x = static_cast<const T*>(p.x) + (size_t)(m < p.T ? m : m0) * p.ldx;
  const Split cut((p.k + 4 * E::EPC - 1) / (4 * E::EPC), p.shares);
  const int step0 = cut.start(share), step1 = cut.start(share + 1);
  for (int w = 0; firsts; ++w) {
    const int j = __builtin_amdgcn_readlane(id, __ffsll((unsigned long long)firsts) - 1);
    firsts &= firsts - 1;
    if (w % p.lanes != block % p.lanes) continue;
    const T* a = static_cast<const T*>(p.a[blockIdx.z]) + ((size_t)j * p.r + (col < p.r ? col : 0)) * p.k;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int U = 8;  // steps in flight
    // two steps after each other are the halves of a 128-byte line: one wave's
    for (int s0 = step0 + 2 * wave; s0 < step1; s0 += kVWaves * U) {
      uint4 xv[U], av[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s = s0 + u / 2 * 2 * kVWaves + u % 2, k = (s * 4 + c0) * E::EPC;
        const bool in = s < step1 && k < p.k;
        xv[u] = in ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
        av[u] = load_part<E>(a + k, in ? p.k - k : 0, WHOLE);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) acc = product<E>(av[u], xv[u], acc);
    }
    __syncthreads();
    sum[wave][lane] = acc;
    __syncthreads();
    const int c = k0 + 4 * c0;
    if (wave == 0 && id == j && c < p.rp) {
      for (int s = 1; s < kVWaves; ++s) acc += sum[s][lane];
      put_share<E>(p, share, blockIdx.z, m, c, j, acc);
    }
  }
}

template <class E>
__global__ void __launch_bounds__(Tile16::threads) k_adapter_v_tiles(AdapterV p) {
  typedef Tile16 C;
  __shared__ __align__(1024) char lds[C::S * C::stage];
  const int lane = lane_id(), wave = uniform(threadIdx.x / kWave);
  const int share = (int)blockIdx.x % p.shares, block = (int)blockIdx.x / p.shares;
  const int m0 = block / p.lanes * 16, n0 = blockIdx.y * C::BN;
  const int m = m0 + (lane & 15), id = id_of(p, m);
  uint64_t firsts = first_tokens(id);
  Loader<E, Lay::KC, C::BM, C::NW> la;
  Loader<E, Lay::KC, C::BN, C::NW> lb;
  la.init(p.ldx, p.T, m0, [](int r) { return r; });
  lb.init(p.k, p.r, n0, [](int r) { return r; });
  const Reader<E, Lay::KC, C::BM, C::MT> ra(0);
  const Reader<E, Lay::KC, C::BN, C::NT> rb(wave * C::WTN);
  const Split cut((p.k + step_k<E>() - 1) / step_k<E>(), p.shares);
  const int it0 = cut.start(share), it1 = cut.start(share + 1);
  const char* x = static_cast<const char*>(p.x) + (size_t)m0 * p.ldx * esz<E>();
  for (int w = 0; firsts; ++w) {
    const int j = __builtin_amdgcn_readlane(id, __ffsll((unsigned long long)firsts) - 1);
    firsts &= firsts - 1;
    if (w % p.lanes != block % p.lanes) continue;
    const char* a = static_cast<const char*>(p.a[blockIdx.z]) + ((size_t)j * p.r + n0) * p.k * esz<E>();
    f32x4_t acc[C::MT][C::NT];
#pragma unroll
    for (int i = 0; i < C::NT; ++i) acc[0][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int pa = decltype(la)::per, per = pa + decltype(lb)::per;
    meet();  // the last adapter's steps have been read
    pipeline<E, C, Lay::KC, Lay::KC, per>(lds, it0, it1, ra, rb, acc, C::BM, false, [&](int f0, int f1, int it, int buf) {
      const int left = it < it1 ? p.k - it * step_k<E>() : 0;
      char* d = lds + buf * C::stage;
#pragma unroll
      for (int f = 0; f < per; ++f) {
        if (f < f0 || f >= f1) continue;
        if (f < pa) la.issue(f, left, d, [&](int) { return x + (size_t)it * 128; });
        else lb.issue(f - pa, left, d + C::BM * 128, [&](int) { return a + (size_t)it * 128; });
      }
    });
    if (id == j) {
#pragma unroll
      for (int i = 0; i < C::NT; ++i) {
        const int c = n0 + wave * C::WTN + i * 16 + 4 * (lane >> 4);
        if (c < p.rp) put_share<E>(p, share, blockIdx.z, m, c, j, acc[0][i]);
      }
    }
  }
}

// Adds up the shares of v, in their order; the last workgroups make the plan.
template <class E>
__global__ void __launch_bounds__(kBlock) k_adapter_join(AdapterV p, int blocks) {
  if ((int)blockIdx.x >= blocks) {
    make_plan(p, (int)blockIdx.x - blocks);
    return;
  }
  const int q = p.rp / 4, i = blockIdx.x * kBlock + threadIdx.x, row = i / q, c = (i - row * q) * 4;
  if (row >= p.count * p.T) return;
  const int which = row / p.T, m = row - which * p.T, id = id_of(p, m);
  if (id < 0) return;
  const size_t plane = (size_t)p.count * p.T * p.rp;
  const float* at = p.part + (size_t)row * p.rp + c;
  f32x4_t u[8], v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 8; ++s)
    u[s] = s < p.shares ? *reinterpret_cast<const f32x4_t*>(at + s * plane) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < 8; ++s) v += u[s];
  put_v<E>(p, which, m, c, id, v);
}

template <class E>
hipError_t adapter_v(AdapterV p, hipStream_t st) {
  const int plans = ceil_div(p.T, p.bm);
  const AdapterPlan plan = adapter_plan(E::EPC == 4, p.T, p.k, p.rp, p.count);
  p.shares = plan.shares;
  p.lanes = plan.lanes;
  p.blocks = plan.blocks;
  if (plan.tiles) {
    k_adapter_v_tiles<E><<<dim3(p.blocks, ceil_div(p.rp, Tile16::BN), p.count), Tile16::threads, 0, st>>>(p);
  } else {
    const dim3 grid(p.blocks + (p.shares == 1 ? plans : 0), ceil_div(p.rp, 16), p.count);
    if (p.k % E::EPC == 0) k_adapter_v<E, true><<<grid, kVWaves * kWave, 0, st>>>(p);
    else k_adapter_v<E, false><<<grid, kVWaves * kWave, 0, st>>>(p);
  }
  if (plan.tiles || p.shares > 1) {
    const int blocks = p.shares > 1 ? ceil_div(p.count * p.T * (p.rp / 4), kBlock) : 0;
    k_adapter_join<E><<<blocks + plans, kBlock, 0, st>>>(p, blocks);
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
    case Tile::T64:
    case Tile::T64x128: return Tile64::BM;
    case Tile::T256: return Tile256::BM;
    default: return Tile128::BM;
  }
}

bool takes_adapters(Tile t) {
  switch (t) {
    case Tile::T16: return adapter_tile<Tile16>();
    case Tile::T64: return adapter_tile<Tile64>();
    case Tile::T64x128: return adapter_tile<Tile64x128>();
    case Tile::T128: return adapter_tile<Tile128>();
    case Tile::T128x256: return adapter_tile<Tile128x256>();
    default: return adapter_tile<Tile256>();
  }
}

// By an estimate of the time, in us.  Tiles run in rounds over the CUs, `a_cu` to a CU.  A step of a tile takes
// `step` of a CU that is full, and no less than `lone` where it has the CU for itself (measured at sizes that
// fill the chip, and at ones that leave CUs empty); a round's first loads and stores take 6 us.  The tiles of
// the last round, where it is not full, may be cut along k in shares that fill it; a share writes its fp32
// sums, and a second launch reads them (5 us and 4 TB/s).  (4096 tokens, d 2560, d_ff 7168: 840 tiles of the
// weight gradients are 3 rounds and 72 tiles, in 3 shares each: 449 -> 400 + 15 us.)
//
// Few tokens are bound by the weights' bytes, whatever the tile: there shares only fill CUs.
Plan choose_tile(bool f32, int problems, int M, int64_t n, int steps, bool adapters, bool tokens) {
  auto tiles = [&](int bm, int bn) { return ((int64_t)M + bm - 1) / bm * ((n + bn - 1) / bn) * problems; };
  if (tokens && M <= 64) {
    const bool few = M <= 16;
    const int64_t nt = tiles(few ? 16 : 64, 64);
    int64_t s = kCUs * 3 / 2 / nt;
    if (s > steps / 8) s = steps / 8;
    if (s > 32) s = 32;
    return Plan{few ? Tile::T16 : Tile::T64, s > 1 ? (int)nt : 0, s > 1 ? (int)s : 1};
  }
  struct Kind {
    Tile t;
    int bm, bn, a_cu;
    int most;  // shares of all cut tiles: their sums stay within share_bytes_most()
    double step, lone;
  };
  static const Kind bf16_kinds[] = {{Tile::T256, 256, 256, 1, 512, 1.45, 1.45},
                                    {Tile::T128x256, 128, 256, 1, 512, 0.82, 0.82},
                                    {Tile::T128, 128, 128, 2, 1024, 0.52, 0.66},
                                    {Tile::T64, 64, 64, 3, 2048, 0.21, 0.30}};
  static const Kind f32_kinds[] = {{Tile::T64x128, 64, 128, 3, 1024, 0.93, 1.00}, {Tile::T64, 64, 64, 3, 2048, 0.51, 0.60}};
  const Kind* kinds = f32 ? f32_kinds : bf16_kinds;
  const int count = f32 ? 2 : 4;
  Plan best{Tile::T64, 0, 1};
  double least = 1e30;
  for (int i = 0; i < count; ++i) {
    const Kind& k = kinds[i];
    if (adapters && !takes_adapters(k.t)) continue;
    const int64_t nt = tiles(k.bm, k.bn), slots = kCUs * k.a_cu, full = nt / slots;
    // the tiles of the last round, the same number of each problem's
    const int64_t last = (nt - full * slots + problems - 1) / problems * problems;
    // tiles at the last row leave empty pieces' products out, but not their loads: a third of a tile at least
    const int over = M % k.bm, rows = (M + k.bm - 1) / k.bm;
    const double part = over ? over / (double)k.bm : 1.0, used = (rows - 1 + (part > 0.35 ? part : 0.35)) / rows;
    const double whole = (double)full * (k.a_cu * k.step * steps + 6.0);
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (s > 1 && (last == 0 || s > steps / 8 || last * s > k.most)) break;
      const int64_t on = (last * s + kCUs - 1) / kCUs, rounds = (on + k.a_cu - 1) / k.a_cu;
      const double step = on * k.step > rounds * k.lone ? on * k.step : rounds * k.lone;
      const double us = used * (whole + step * ((steps + s - 1) / s) + 6.0 * rounds) +
                        (s > 1 ? 5.0 + 2e-6 * k.bm * k.bn * (double)last * s : 0.0);
      if (us < least) {
        least = us;
        best = Plan{k.t, s > 1 ? (int)last : 0, s};
      }
    }
  }
  return best;
}

size_t share_bytes_most(bool f32, int problems, int M, int64_t n, bool tokens) {
  const size_t cap = f32 ? (size_t)2048 * 64 * 64 * 4 : (size_t)512 * 256 * 256 * 4;
  if (tokens && M <= 16) return (size_t)kCUs * 3 / 2 * 16 * 64 * 4;
  if (tokens && M <= 64) return (size_t)kCUs * 3 / 2 * 64 * 64 * 4;
  const size_t all = (size_t)32 * problems * (((int64_t)M + 255) / 256 * 256) * ((n + 255) / 256 * 256) * 4;
  return all < cap ? all : cap;
}

Plan token_plan(bool f32, int T, int n, int k, int products, bool adapters) {
  return choose_tile(f32, 1, T, n, products * ceil_div(k, f32 ? step_k<EF32>() : step_k<EBf16>()), adapters, true);
}
Plan hidden_plan(bool f32, const BlockShape& s, bool adapters) {
  return choose_tile(f32, 1, s.T, 2 * (int64_t)s.d_ff, ceil_div(s.d, f32 ? step_k<EF32>() : step_k<EBf16>()), adapters, true);
}

hipError_t launch_token_product_ks(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KS>(p, st) : product<EBf16, Lay::KS>(p, st);
}
hipError_t launch_token_product_kc(bool f32, const TokenProduct& p, hipStream_t st) {
  return f32 ? product<EF32, Lay::KC>(p, st) : product<EBf16, Lay::KC>(p, st);
}

hipError_t launch_adapter_v(bool f32, int T, int k, int ldx, const void* x, const AdapterSet& ad, int count,
                            const void* const a[2], void* const v[2], Tile t, hipStream_t st) {
  const AdapterV p{x, {a[0], a[1]}, {v[0], v[1]}, ad.ids, ad.scale, ad.plan, ad.part,
                   T, k, ldx, ad.n, ad.r, ad.rp, 0, 0, tile_rows(t), 1, count};
  return f32 ? adapter_v<EF32>(p, st) : adapter_v<EBf16>(p, st);
}

hipError_t launch_pad_rows(bool f32, int64_t rows, int n, int np, const void* src, void* dst, hipStream_t st) {
  const int64_t want = rows * np / 8 / kBlock + 1;
  const int grid = (int)(want < 32 * kCUs ? want : 32 * kCUs);
  if (f32) k_pad_rows<EF32><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const float*>(src), static_cast<float*>(dst));
  else k_pad_rows<EBf16><<<grid, kBlock, 0, st>>>(rows, n, np, static_cast<const __bf16*>(src), static_cast<__bf16*>(dst));
  return hipGetLastError();
}

}  // namespace ffn
