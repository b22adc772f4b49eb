// The tiled matrix product behind the gated block, its backward pass and the adapters (gfx950).
// Not part of the public ABI.
//
//   acc[m][n] = sum over k of A(m, k) B(n, k)
//
// Either operand lies in memory with k contiguous ([rows][k]: "KC") or strided ([k][rows]: "KS"),
// so the forward products (x W^T: KC, KC; z W2t: KC, KS), the token gradient (dg W1: KC, KS) and
// the weight gradients (dg^T x: KS, KS) are one kernel.  A workgroup owns a BM x BN tile of the
// result and walks k in steps of 128 bytes (64 bf16, 32 fp32).  Both tiles of a step go from memory
// into LDS without passing through registers (buffer_load ... lds, 16 bytes a lane), S steps deep:
// the loads of step i + S - 1 are in flight while step i is multiplied, and the only waits of a step
// are for its own loads and for the workgroup to have left the buffer that is loaded next.
//
// LDS images.  A load writes 64 consecutive 16-byte chunks, so a swizzle can only choose which chunk
// of memory a lane fetches:
//   KC  row r holds its 8 chunks of the step, chunk c in place c ^ (r & 7): the 8 rows that a fragment
//       read touches at once then cover all banks.
//   KS  row k holds the tile's columns; for bf16 the 32-byte pieces are exchanged by k & 3 and bit 3
//       of k, and fragments are read with the transposing LDS read (ds_read_b64_tr_b16), whose 16 lanes
//       cover 4 rows k; for fp32 the 64-byte pieces are exchanged by bits 2..3 of k and read by element.
// Rows, columns and k beyond the operand are fetched from a buffer offset past its end, which reads
// as zero: tails need no other code.
//
// The products run as mfma(B fragment, A fragment), which leaves a lane with four consecutive n of one
// m, what a row-major store wants.  Sums are fp32 throughout.
#pragma once

#include "ffn_mfma.h"

namespace ffn {
namespace {

struct EBf16 {
  typedef __bf16 T;
  static constexpr int EPC = 8;  // elements of a 16-byte chunk
};
struct EF32 {
  typedef float T;
  static constexpr int EPC = 4;
};
template <class E>
constexpr int esz() {
  return 16 / E::EPC;
}
template <class E>
constexpr int step_k() {  // k of one step: 128 bytes of a KC row
  return 8 * E::EPC;
}

// One operand: p[0], and p[1] for a second one of the same layout (the other factor of a sum of two
// products, or W_up beside W_gate).  rows: the extent that is not k; a KS operand's rows are whole
// chunks (its memory is padded to them).
struct Operand {
  const void* p[2];
  int64_t ld;
  int rows;
};

// Adapters of a product: token m adds sum over k of v[m][k] B_j[n][k] for its adapter j, with
// v = scale_j A_j x computed before (k_adapter_v) and B_j = b + j out r, [out][r].  rp: r in whole
// chunks, the row length of v.  plan: for every tile of BM tokens 1 + 2 BM entries, the number of
// adapters among its tokens, those adapters in the order of their first token, and every token's place
// in that list (-1: none).  Index 1 of v and b is W_up's, of a dual product.
struct LowRank {
  const void* v[2];
  const void* b[2];
  const int32_t* plan;
  int r, rp, out;
};

struct GemmArgs {
  Operand a, b;
  int M, N;      // of the result (N neurons for a dual product)
  int K;         // of one product
  int products;  // 1, or 2: the sum over p[0] and p[1] of both operands
  int ntm, ntn;
  // The tiles from the `whole`-th on are cut along k: `shares` workgroups to a tile, which write their fp32
  // sums to part, [tile][share][16-row piece][16-column piece][thread], for k_join to finish.
  int whole, shares;
  float* part;
  LowRank lr;
};

template <int BM_, int BN_, int WM_, int WN_, int S_>
struct Config {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, S = S_;
  static constexpr int NW = WM * WN, threads = NW * kWave;
  static constexpr int WTM = BM / WM, WTN = BN / WN, MT = WTM / 16, NT = WTN / 16;
  static constexpr int stage = (BM + BN) * 128;
};

enum class Lay { KC, KS };

__device__ __forceinline__ void lds_load16(const Buf& b, char* dst, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b.r, (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, 0);
}

// The same from an address of each lane's own.
__device__ __forceinline__ void lds_load16(const void* p, char* dst) {
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)p,
                                   (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}
// what a lane with nothing to load reads there
__device__ const uint4 zero_chunk = {0, 0, 0, 0};

// Waits until at most n of this wave's loads are in flight and its LDS reads have returned.
template <int n>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | ((n >> 4) << 14));
}
// All waves of the workgroup; nothing of one side is moved to the other.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------------------ memory to LDS
// A tile of ROWS (not-k) x one step, loaded by NW waves: instruction j of ROWS / 8 fills the chunks
// 64 j .. 64 j + 63; a wave takes every NW-th (where there are fewer than waves, some load the same
// chunks: the wait counts of all waves are then equal).
template <class E, Lay L, int ROWS, int NW>
struct Loader {
  static constexpr int CPR = ROWS / E::EPC;  // KS: chunks of a row k
  static constexpr int total = ROWS / 8, per = (total + NW - 1) / NW;
  static_assert(total % NW == 0 || NW % total == 0, "loads divide over the waves");
  uint32_t off[per];  // byte offset from the step's base, kOOB outside the operand
  int kpos[per];      // first k of the chunk within the step

  __device__ __forceinline__ static int instr(int i, int wave) { return (i * NW + wave) % total; }
  // KS: the swizzle of row k, in chunks
  __device__ __forceinline__ static int swz(int k) {
    if constexpr (E::EPC == 8) return ((k & 3) | (CPR >= 16 ? ((k >> 3) & 1) << 2 : 0)) << 1;
    else return ((k >> 2) & 3) << 2;
  }
  // row(r): the row, from r0 on, that LDS row r holds
  template <class RowOf>
  __device__ __forceinline__ void init(int64_t ld, int rows, int r0, RowOf row) {
    const int wave = threadIdx.x / kWave, lane = lane_id();
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const int j = instr(i, wave);
      if constexpr (L == Lay::KC) {
        const int c = (lane & 7) ^ (lane >> 3), rr = row(j * 8 + (lane >> 3));
        kpos[i] = c * E::EPC;
        off[i] = rr + r0 < rows ? (uint32_t)rr * (uint32_t)(ld * esz<E>()) + c * 16 : kOOB;
      } else {
        const int s = j * kWave + lane, k = s / CPR, c = (s % CPR) ^ swz(k);
        kpos[i] = k;
        off[i] = r0 + c * E::EPC < rows ? (uint32_t)k * (uint32_t)(ld * esz<E>()) + c * 16 : kOOB;
      }
    }
  }
  // Instruction i of this wave for a step that starts at `base` with k_left of k left (none or less:
  // zeros); base(j) where the rows of instruction j lie.
  template <class Base>
  __device__ __forceinline__ void issue(int i, int k_left, char* dst, Base base) const {
    const int j = instr(i, uniform(threadIdx.x / kWave));
    lds_load16(make_buf(base(j), 0x7fffffffu), dst + j * 1024, kpos[i] < k_left ? off[i] : kOOB);
  }
  // bytes from one step to the next
  __device__ __forceinline__ static int64_t stride(int64_t ld) {
    return L == Lay::KC ? 128 : (int64_t)step_k<E>() * ld * esz<E>();
  }
};

// ------------------------------------------------------------------ LDS to fragments
// A 16-byte LDS read as a plain vector load.  Read as a struct (uint4), the load loses its type in the
// compiler, which then takes it to depend on every load into LDS still in flight and waits for all of
// them (vmcnt 0) in front of it.
__device__ __forceinline__ uint4 lds_read16(const char* p) {
  const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
// The transposing read (see lds_read_tr16), for the same reason through a pointer of its own scope.
__device__ __forceinline__ uint2 lds_read_tr(const char* __restrict__ p) { return lds_read_tr16(p); }

// Fragment of half kk (0, 1) of a step for the 16 rows from tile row r: lane l holds row r + l % 16 and
// chunk l / 16 of the half (bf16: k = 8 (l / 16) .. + 7; fp32: component j is k = 4 (l / 16) + j).
template <class E, Lay L, int ROWS, int TILES>
struct Reader {
  typedef Loader<E, L, ROWS, 1> Ld;
  static constexpr int CPR = Ld::CPR;
  int off[L == Lay::KC ? 2 : TILES];

  __device__ __forceinline__ explicit Reader(int row0) {
    const int lane = lane_id();
    if constexpr (L == Lay::KC) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        off[kk] = (row0 + (lane & 15)) * 128 + (((kk * 4 + (lane >> 4)) ^ (lane & 7)) << 4);
    } else {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        if constexpr (E::EPC == 8) {
          const int k = 8 * (lane >> 4) + ((lane >> 2) & 3), c = (row0 + t * 16) / 8 + ((lane >> 1) & 1);
          off[t] = k * CPR * 16 + ((c ^ Ld::swz(k)) << 4) + (lane & 1) * 8;
        } else {
          const int k = 4 * (lane >> 4), c = (row0 + t * 16) / 4 + ((lane >> 2) & 3);
          off[t] = k * CPR * 16 + ((c ^ Ld::swz(k)) << 4) + (lane & 3) * 4;
        }
      }
    }
  }
  __device__ __forceinline__ uint4 get(const char* s, int kk, int t) const {
    if constexpr (L == Lay::KC) {
      return lds_read16(s + off[kk] + t * 2048);
    } else if constexpr (E::EPC == 8) {
      const char* p = s + off[t] + kk * 32 * CPR * 16;
      const uint2 lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * CPR * 16);
      return make_uint4(lo.x, lo.y, hi.x, hi.y);
    } else {
      const char* p = s + off[t] + kk * 16 * CPR * 16;
      return make_uint4(*reinterpret_cast<const uint32_t*>(p), *reinterpret_cast<const uint32_t*>(p + CPR * 16),
                        *reinterpret_cast<const uint32_t*>(p + 2 * CPR * 16),
                        *reinterpret_cast<const uint32_t*>(p + 3 * CPR * 16));
    }
  }
};

template <class E>
__device__ __forceinline__ f32x4_t product(const uint4& b, const uint4& a, f32x4_t c) {
  if constexpr (E::EPC == 8) {
    return mfma16(bf8(b), bf8(a), c);
  } else {
    c = mfma16f(comp<0>(b), comp<0>(a), c);
    c = mfma16f(comp<1>(b), comp<1>(a), c);
    c = mfma16f(comp<2>(b), comp<2>(a), c);
    return mfma16f(comp<3>(b), comp<3>(a), c);
  }
}

// The fragments of half a step, and their products.
template <class E, class C, Lay LA, Lay LB>
struct Half {
  static constexpr int count = C::MT + C::NT;
  uint4 a[C::MT], b[C::NT];
  // fragments [f0, f1) in the order in which the products use them
  __device__ __forceinline__ void load(int f0, int f1, const char* stage, int kk, const Reader<E, LA, C::BM, C::MT>& ra,
                                       const Reader<E, LB, C::BN, C::NT>& rb) {
#pragma unroll
    for (int f = 0; f < count; ++f) {
      if (f < f0 || f >= f1) continue;
      if (f < C::NT) b[f] = rb.get(stage + C::BM * 128, kk, f);
      else a[f - C::NT] = ra.get(stage, kk, f - C::NT);
    }
  }
  // between(i): work to issue in front of the products of fragment a[i].  LDS reads and loads into LDS
  // are handed out among the products a few at a time: issued in one piece they fill their queues, and a
  // wave that waits for a queue issues no products either.
  // RAGGED: only the first `rows` of the 16-row pieces have any rows of the result.  J0, J1: only the products of
  // fragments b[J0] .. b[J1 - 1].
  template <bool RAGGED, int J0 = 0, int J1 = C::NT, class Between>
  __device__ __forceinline__ void multiply(f32x4_t (&acc)[C::MT][C::NT], int rows, Between between) const {
#pragma unroll
    for (int i = 0; i < C::MT; ++i) {
      between(i);
      if (!RAGGED || i < rows) {
#pragma unroll
        for (int j = J0; j < J1; ++j) acc[i][j] = product<E>(b[j], a[i], acc[i][j]);
      }
      issue_barrier();
    }
  }
};

// up to EPC elements from p, the rest zero
template <class E>
__device__ __forceinline__ uint4 load_part(const typename E::T* p, int n, bool whole) {
  if (n <= 0) return make_uint4(0, 0, 0, 0);
  if (whole) return *reinterpret_cast<const uint4*>(p);
  typename E::T v[E::EPC];
#pragma unroll
  for (int i = 0; i < E::EPC; ++i) v[i] = i < n ? p[i] : (typename E::T)0.f;
  return __builtin_bit_cast(uint4, v);
}

// ------------------------------------------------------------------ activations
// A(g), and with its derivative; the same of the up side.  A gate value that is not above zero (NaN
// too) gives zero and slope zero, but for SiLU.
__device__ __forceinline__ float block_act(int act, float g) {
  if (act == 0) return g > 0.f ? g : 0.f;
  const float a = g / (1.f + expf(-g));
  return act == 2 || g > 0.f ? a : 0.f;
}
__device__ __forceinline__ void silu_grad(float g, float& a, float& da) {
  const float s = 1.f / (1.f + expf(-g));
  a = g * s;
  da = s * (1.f + g * (1.f - s));
}
__device__ __forceinline__ void block_act_grad(int act, float g, float& a, float& da) {
  const bool on = act == 2 || g > 0.f;
  float sa, sd;
  if (act == 0) {
    sa = g;
    sd = 1.f;
  } else {
    silu_grad(g, sa, sd);
  }
  a = on ? sa : 0.f;
  da = on ? sd : 0.f;
}
__device__ __forceinline__ void up_grad(int silu, float v, float& u, float& du) {
  if (silu) {
    silu_grad(v, u, du);
  } else {
    u = v;
    du = 1.f;
  }
}

// ------------------------------------------------------------------ which tile
// Workgroups go to the 8 XCDs in turn, each with an L2 of its own: XCD x takes the x-th eighth of the
// tiles, and walks it in bands of 8 tile rows, so that the tiles it works on at one time share rows of A
// and of B.
struct TileAt {
  int m, n, cut, share;  // cut: the place among the tiles that are cut, or -1
};
__device__ __forceinline__ TileAt tile_of(const GemmArgs& g, int t) {
  constexpr int kBand = 8;
  const int band = t / (kBand * g.ntn), rows = min(kBand, g.ntm - band * kBand), u = t - band * kBand * g.ntn;
  return TileAt{band * kBand + u % rows, u / rows, -1, 0};
}
// the x-th eighth of [0, n)
__device__ __forceinline__ int eighth(int n, int b) {
  const int q = n / 8, rem = n % 8, x = b % 8;
  return x * q + min(x, rem) + b / 8;
}
__device__ __forceinline__ TileAt tile_at(const GemmArgs& g) {
  const int b = blockIdx.x;
  if (b < g.whole) return tile_of(g, eighth(g.whole, b));
  const int u = eighth((int)gridDim.x - g.whole, b - g.whole), cut = u / g.shares;
  TileAt at = tile_of(g, g.whole + cut);
  at.cut = cut;
  at.share = u - cut * g.shares;
  return at;
}

// ------------------------------------------------------------------ the pipeline
// Steps [it0, it1) into acc.  issue(f0, f1, it, buf): loads f0 .. f1 - 1 of this wave's PER for step `it`
// into buffer `buf`; from it1 on they have to be zeros or anything else that nothing uses, so that
// every step has the same loads in flight.
//
// Half a step's fragments are read while the other half's products run: the second half of step i
// during the first half's products, the first half of step i + 1, behind the barrier that frees step i's
// buffer, during the second half's, and with it step i + S is loaded into that buffer.
// rows: this wave's 16-row pieces that hold rows of the result; a tile at the last row, which has fewer than
// all, leaves the others' products out (RAGGED).
template <bool RAGGED, class E, class C, Lay LA, Lay LB, int PER, class Issue>
__device__ __forceinline__ void run_steps(char* lds, int it0, int it1, const Reader<E, LA, C::BM, C::MT>& ra,
                                          const Reader<E, LB, C::BN, C::NT>& rb, f32x4_t (&acc)[C::MT][C::NT], int rows,
                                          Issue issue) {
#pragma unroll
  for (int i = 0; i < C::S; ++i) issue(0, PER, it0 + i, i);
  wait_loads<(C::S - 1) * PER>();
  meet();
  Half<E, C, LA, LB> h0, h1;
  h0.load(0, h0.count, lds, 0, ra, rb);
  int buf = 0;
  // An fp32 product adds its terms one after the other, so every four fp32 steps are summed from zero and
  // then into the running sum: two short chains in place of a long one.
  constexpr bool chain2 = E::EPC == 4;
  f32x4_t step[chain2 ? C::MT : 1][chain2 ? C::NT : 1];
  auto& sum = [&]() -> auto& {
    if constexpr (chain2) return step;
    else return acc;
  }();
  auto flush = [&] {
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int j = 0; j < C::NT; ++j) {
        acc[i][j] += step[i][j];
        step[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
  };
  if constexpr (chain2)
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
#pragma unroll
      for (int j = 0; j < C::NT; ++j) step[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int it = it0; it < it1; ++it) {
    h0.template multiply<RAGGED>(sum, rows, [&](int i) {
      h1.load(i * h1.count / C::MT, (i + 1) * h1.count / C::MT, lds + buf * C::stage, 1, ra, rb);
    });
    wait_loads<(C::S - 2) * PER>();
    meet();
    const int next = buf + 1 == C::S ? 0 : buf + 1;
    h1.template multiply<RAGGED>(sum, rows, [&](int i) {
      h0.load(i * h0.count / C::MT, (i + 1) * h0.count / C::MT, lds + next * C::stage, 0, ra, rb);
      issue(i * PER / C::MT, (i + 1) * PER / C::MT, it + C::S, buf);
    });
    if constexpr (chain2)
      if (((it - it0) & 3) == 3) flush();
    buf = next;
  }
  if constexpr (chain2) flush();
  wait_loads<0>();  // LDS is free for others once no load into it is in flight
}
// left: rows of the result from the wave's first on
template <class E, class C, Lay LA, Lay LB, int PER, class Issue>
__device__ __forceinline__ void pipeline(char* lds, int it0, int it1, const Reader<E, LA, C::BM, C::MT>& ra,
                                         const Reader<E, LB, C::BN, C::NT>& rb, f32x4_t (&acc)[C::MT][C::NT], int left,
                                         bool ragged, Issue issue) {
  if (C::MT == 1 || !ragged) run_steps<false, E, C, LA, LB, PER>(lds, it0, it1, ra, rb, acc, C::MT, issue);
  else run_steps<true, E, C, LA, LB, PER>(lds, it0, it1, ra, rb, acc, left > 0 ? (left + 15) / 16 : 0, issue);
}

// ------------------------------------------------------------------ adapters within a product
// The low-rank part is a product over k = (adapter of the tile, rank), rp to an adapter, in chunks:
// row m of the A tile holds v[m] in its own adapter's chunks and zero in the others, row n of the B tile
// B_j[n].  A dual product runs W_gate's adapters, into W_gate's sums alone (the zeros in W_up's rows of the B
// tile would turn an Inf or NaN of v into a NaN of W_up's), then W_up's.  Both images are KC.
//
// Rows of whole chunks are loaded into LDS some steps ahead, each lane from an address of its own; odd
// ranks are read by element and written to LDS, a step at a time.  (As further steps of the main part's
// pipeline they cost its loop more than the drained pipeline between the parts does: 48 tokens, 14336 x
// 4096, rank 16, 35 against 31 us.)
template <class E, class C, bool DUAL>
struct AdapterSteps {
  typedef typename E::T T;
  static constexpr int G = C::WTN / 2;
  typedef Loader<E, Lay::KC, C::BM, C::NW> LdA;
  typedef Loader<E, Lay::KC, C::BN, C::NW> LdB;
  static constexpr int per = LdA::per + LdB::per;
  const LowRank& lr;
  const int32_t* plan;  // the tile's, in LDS
  int m0, n0, cpr, chunks, steps;  // steps of one matrix's adapters

  __device__ __forceinline__ AdapterSteps(const LowRank& l, const int32_t* lds_plan, int m0_, int n0_)
      : lr(l), plan(lds_plan), m0(m0_), n0(n0_), cpr(l.rp / E::EPC) {
    chunks = uniform(plan[0]) * cpr;
    steps = (chunks + 7) / 8;
  }
  __device__ __forceinline__ int count() const { return (lr.b[0] ? steps : 0) + (DUAL && lr.b[1] ? steps : 0); }
  // the matrix of step `it`, and the step within its adapters
  __device__ __forceinline__ int matrix(int it) const { return DUAL && (!lr.b[0] || it >= steps) ? 1 : 0; }
  __device__ __forceinline__ int within(int it) const { return lr.b[0] && it >= steps ? it - steps : it; }
  __device__ __forceinline__ const T* v_at(int which, int m, int part) const {
    return static_cast<const T*>(lr.v[which]) + (size_t)m * lr.rp + part * E::EPC;
  }
  __device__ __forceinline__ const T* b_at(int which, int j, int n, int part) const {
    return static_cast<const T*>(lr.b[which]) + ((size_t)j * lr.out + n) * lr.r + part * E::EPC;
  }
  __device__ __forceinline__ int neuron(int r) const { return n0 + (DUAL ? r / C::WTN * G + r % G : r); }
  __device__ __forceinline__ bool has(int which, int r) const { return !DUAL || (r % C::WTN >= G) == (which == 1); }

  // this wave's loads of step `it`, zeros from it1 on
  __device__ __forceinline__ void issue(int it, int it1, char* stage) const {
    const int wave = uniform(threadIdx.x / kWave), lane = lane_id(), c = (lane & 7) ^ (lane >> 3);
    const int which = matrix(it), q = within(it) * 8 + c;
    const bool on = it < it1 && q < chunks;
    const int slot = on ? q / cpr : 0, part = q - slot * cpr, j = plan[1 + slot];
#pragma unroll
    for (int f = 0; f < per; ++f) {
      if (f < LdA::per) {
        const int i = LdA::instr(f, wave), r = i * 8 + (lane >> 3);
        const bool mine = on && plan[1 + C::BM + r] == slot;
        lds_load16(mine ? static_cast<const void*>(v_at(which, m0 + r, part)) : &zero_chunk, stage + i * 1024);
      } else {
        const int i = LdB::instr(f - LdA::per, wave), r = i * 8 + (lane >> 3), n = neuron(r);
        const bool mine = on && has(which, r) && n < lr.out;
        lds_load16(mine ? static_cast<const void*>(b_at(which, j, n, part)) : &zero_chunk,
                   stage + C::BM * 128 + i * 1024);
      }
    }
  }

  // The products of half kk of step `it`.  A token's zeros do not shield it from an Inf or NaN in another
  // request's B (0 x Inf is NaN), so B's fragments are looked at first, and a half that holds such a value
  // goes chunk by chunk, each into sums of its own that only its own tokens take.
  template <class H>
  __device__ __forceinline__ void multiply(const H& h, int it, int kk, int wm, f32x4_t (&acc)[C::MT][C::NT]) const {
    if constexpr (DUAL) {  // the matrix' half of the wave's columns
      if (matrix(it) == 0) multiply_columns<0, C::NT / 2>(h, it, kk, wm, acc);
      else multiply_columns<C::NT / 2, C::NT>(h, it, kk, wm, acc);
    } else {
      multiply_columns<0, C::NT>(h, it, kk, wm, acc);
    }
  }
  template <int J0, int J1, class H>
  __device__ __forceinline__ void multiply_columns(const H& h, int it, int kk, int wm,
                                                   f32x4_t (&acc)[C::MT][C::NT]) const {
    constexpr uint32_t e = E::EPC == 8 ? 0x7f807f80u : 0x7f800000u, one = E::EPC == 8 ? 0x00800080u : 0x00800000u,
                       top = E::EPC == 8 ? 0x80008000u : 0x80000000u;
    uint32_t odd = 0;  // an exponent of all ones carries into its sign's place
#pragma unroll
    for (int j = J0; j < J1; ++j)
      odd |= ((h.b[j].x & e) + one) | ((h.b[j].y & e) + one) | ((h.b[j].z & e) + one) | ((h.b[j].w & e) + one);
    if (__ballot((odd & top) != 0) == 0) {
      h.template multiply<false, J0, J1>(acc, C::MT, [](int) {});
      return;
    }
    const int lane = lane_id();
    for (int c = 0; c < 4; ++c) {
      const int slot = (within(it) * 8 + kk * 4 + c) / cpr;
      const bool here = (lane >> 4) == c;
#pragma unroll
      for (int i = 0; i < C::MT; ++i) {
        const bool mine = plan[1 + C::BM + wm * C::WTM + i * 16 + (lane & 15)] == slot;
        const uint4 a = here ? h.a[i] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = J0; j < J1; ++j) {
          const f32x4_t v = product<E>(here ? h.b[j] : make_uint4(0, 0, 0, 0), a, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[i][j][k] = mine ? acc[i][j][k] + v[k] : acc[i][j][k];
        }
      }
    }
  }

  __device__ __forceinline__ void fill(int it, char* stage) const {
    const int which = matrix(it), q0 = within(it) * 8;
    for (int s = threadIdx.x; s < (C::BM + C::BN) * 8; s += C::threads) {
      const int row = s >> 3, c = s & 7, q = q0 + c, slot = q < chunks ? q / cpr : 0, part = q - slot * cpr;
      uint4 x = make_uint4(0, 0, 0, 0);
      if (row < C::BM) {
        if (q < chunks && plan[1 + C::BM + row] == slot) x = *reinterpret_cast<const uint4*>(v_at(which, m0 + row, part));
      } else {
        const int r = row - C::BM, n = neuron(r);
        if (q < chunks && has(which, r) && n < lr.out)
          x = load_part<E>(b_at(which, plan[1 + slot], n, part), lr.r - part * E::EPC, false);
      }
      *reinterpret_cast<uint4*>(stage + row * 128 + ((c ^ (row & 7)) << 4)) = x;
    }
  }
};

// ------------------------------------------------------------------ the end of a tile
// The sums of this wave's i-th 16 rows: lane l of a 16 x 16 piece holds m = l % 16, n = 4 (l / 16) .. + 3.
template <class C, bool DUAL, class Epi>
__device__ __forceinline__ void finish(const GemmArgs& g, const Epi& epi, int m0, int n0, int wm, int wn, int i,
                                       const f32x4_t (&acc)[C::NT]) {
  constexpr int G = C::WTN / 2;
  const int lane = lane_id(), m = m0 + wm * C::WTM + i * 16 + (lane & 15);
  if (m >= g.M) return;
  if constexpr (DUAL) {
#pragma unroll
    for (int j = 0; j < C::NT / 2; ++j) epi.pair(m, n0 + wn * G + j * 16 + 4 * (lane >> 4), acc[j], acc[j + C::NT / 2]);
  } else {
#pragma unroll
    for (int j = 0; j < C::NT; ++j) epi.put(g, m, n0 + wn * C::WTN + j * 16 + 4 * (lane >> 4), acc[j]);
  }
}
// Where this thread's sums of piece (i, j) lie, of a share of a cut tile.  Several results of one launch
// (blockIdx.y) follow each other.
template <class C>
__device__ __forceinline__ f32x4_t* share_at(const GemmArgs& g, int cut, int share, int i, int j) {
  const size_t tile = ((size_t)blockIdx.y * (g.ntm * g.ntn - g.whole) + cut) * g.shares + share;
  return reinterpret_cast<f32x4_t*>(g.part) + ((tile * C::MT + i) * C::NT + j) * C::threads + threadIdx.x;
}

// ------------------------------------------------------------------ the kernel
// DUAL: B's tile holds W_gate and W_up rows of the same BN / 2 neurons, a wave's columns being half of
// either, so that its lanes end with both values of their neurons.  AD: adapters.
template <class E, class C, Lay LA, Lay LB, bool DUAL, bool AD, class Epi>
__global__ void __launch_bounds__(C::threads) k_gemm(GemmArgs g, Epi epi) {
  // One array for all: with a second one the compiler marks the accesses of either, and with the marks it
  // takes every LDS read to wait for the loads in flight (see lds_read16).
  __shared__ __align__(1024) char lds[C::S * C::stage + (AD ? (1 + 2 * C::BM) * 4 : 0)];
  constexpr int G = C::WTN / 2;  // neurons of a wave, dual
  constexpr int BNN = DUAL ? C::BN / 2 : C::BN;
  const TileAt at = tile_at(g);
  const int m0 = at.m * C::BM, n0 = at.n * BNN;
  const int wave = uniform(threadIdx.x / kWave), wm = wave / C::WN, wn = wave % C::WN;
  epi.select(g);

  Loader<E, LA, C::BM, C::NW> la;
  Loader<E, LB, C::BN, C::NW> lb;
  la.init(g.a.ld, g.a.rows, m0, [](int r) { return r; });
  if constexpr (DUAL) {
    static_assert(LB == Lay::KC && G % 8 == 0, "an instruction loads 8 rows of one of the two matrices");
    lb.init(g.b.ld, g.b.rows, n0, [](int r) { return r / C::WTN * G + r % G; });
  } else {
    lb.init(g.b.ld, g.b.rows, n0, [](int r) { return r; });
  }
  const int64_t sa = la.stride(g.a.ld), sb = lb.stride(g.b.ld);
  const int64_t a0 = LA == Lay::KC ? (int64_t)m0 * g.a.ld * esz<E>() : (int64_t)m0 * esz<E>();
  const int64_t b0 = LB == Lay::KC ? (int64_t)n0 * g.b.ld * esz<E>() : (int64_t)n0 * esz<E>();
  const int kt = (g.K + step_k<E>() - 1) / step_k<E>();

  const int shares = at.cut >= 0 ? g.shares : 1;
  const Split steps(kt * g.products, shares);
  const int it0 = steps.start(at.share), it1 = steps.start(at.share + 1);
  // loads [f0, f1) of this wave for step `it`; past the last step they fill the buffer with zeros, which
  // nothing uses, so that every step has the same loads in flight
  constexpr int per_step = decltype(la)::per + decltype(lb)::per;
  auto issue = [&](int f0, int f1, int it, int buf) {
    const int seg = it >= kt ? 1 : 0, k = it - seg * kt, left = it < it1 ? g.K - k * step_k<E>() : 0;
    char* d = lds + buf * C::stage;
    const char* pa = static_cast<const char*>(g.a.p[seg]) + a0 + k * sa;
    const char* pb = static_cast<const char*>(g.b.p[DUAL ? 0 : seg]) + b0 + k * sb;
    const char* pb2 = static_cast<const char*>(g.b.p[1]) + b0 + k * sb;
#pragma unroll
    for (int f = 0; f < per_step; ++f) {
      if (f < f0 || f >= f1) continue;
      if (f < decltype(la)::per) la.issue(f, left, d, [&](int) { return pa; });
      else lb.issue(f - decltype(la)::per, left, d + C::BM * 128,
                    [&](int j) { return DUAL && j * 8 % C::WTN >= G ? pb2 : pb; });
    }
  };

  f32x4_t acc[C::MT][C::NT];
#pragma unroll
  for (int i = 0; i < C::MT; ++i)
#pragma unroll
    for (int j = 0; j < C::NT; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const Reader<E, LA, C::BM, C::MT> ra(wm * C::WTM);
  const Reader<E, LB, C::BN, C::NT> rb(wn * C::WTN);
  if constexpr (!AD) {
    pipeline<E, C, LA, LB, per_step>(lds, it0, it1, ra, rb, acc, g.M - m0 - wm * C::WTM, g.M - m0 < C::BM, issue);
  } else {
    typedef AdapterSteps<E, C, DUAL> Steps;
    int32_t* plan = reinterpret_cast<int32_t*>(lds + C::S * C::stage);
    for (int i = threadIdx.x; i < 1 + 2 * C::BM; i += C::threads)
      plan[i] = g.lr.plan[(size_t)at.m * (1 + 2 * C::BM) + i];
    __syncthreads();
    const Steps ad(g.lr, plan, m0, n0);
    const Split part(ad.count(), shares);
    const int ad0 = part.start(at.share), ad1 = part.start(at.share + 1);
    const bool whole = g.lr.r % E::EPC == 0;
    pipeline<E, C, LA, LB, per_step>(lds, it0, it1, ra, rb, acc, g.M - m0 - wm * C::WTM, g.M - m0 < C::BM, issue);
    meet();  // the last step has been read
    const Reader<E, Lay::KC, C::BM, C::MT> rva(wm * C::WTM);
    const Reader<E, Lay::KC, C::BN, C::NT> rvb(wn * C::WTN);
    constexpr int ahead = C::S - 1;
    if (whole && ad0 < ad1) {
#pragma unroll
      for (int i = 0; i < ahead; ++i) ad.issue(ad0 + i, ad1, lds + i * C::stage);
    }
    int buf = 0;
    for (int it = ad0; it < ad1; ++it) {
      if (whole) {
        wait_loads<(ahead - 1) * Steps::per>();
        meet();
        ad.issue(it + ahead, ad1, lds + (buf == 0 ? ahead : buf - 1) * C::stage);
      } else {
        __syncthreads();
        ad.fill(it, lds + buf * C::stage);
        __syncthreads();
      }
      Half<E, C, Lay::KC, Lay::KC> h;
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        h.load(0, h.count, lds + buf * C::stage, kk, rva, rvb);
        ad.multiply(h, it, kk, wm, acc);
      }
      buf = buf + 1 == C::S ? 0 : buf + 1;
    }
    wait_loads<0>();
  }

  if (at.cut >= 0) {
    const int left = g.M - m0 - wm * C::WTM - (lane_id() & 15);  // rows of the result from this lane's first on
#pragma unroll
    for (int i = 0; i < C::MT; ++i)
      if (i * 16 < left)
#pragma unroll
        for (int j = 0; j < C::NT; ++j) *share_at<C>(g, at.cut, at.share, i, j) = acc[i][j];
    return;
  }
#pragma unroll
  for (int i = 0; i < C::MT; ++i) finish<C, DUAL>(g, epi, m0, n0, wm, wn, i, acc[i]);
}

// Adds the shares of the cut tiles up, in their order, and finishes them: a workgroup to a tile and 16-row
// piece of its waves.
template <class C, bool DUAL, class Epi>
__global__ void __launch_bounds__(C::threads) k_join(GemmArgs g, Epi epi) {
  epi.select(g);
  const int cut = blockIdx.x, i = blockIdx.z;
  const TileAt at = tile_of(g, g.whole + cut);
  const int wave = threadIdx.x / kWave, wm = wave / C::WN, wn = wave % C::WN;
  const int m0 = at.m * C::BM, n0 = at.n * (DUAL ? C::BN / 2 : C::BN);
  if (m0 + wm * C::WTM + i * 16 + (lane_id() & 15) >= g.M) return;
  f32x4_t acc[C::NT];
#pragma unroll
  for (int j = 0; j < C::NT; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  constexpr int U = C::NT >= 4 ? 2 : 8 / C::NT;  // shares in flight
  for (int s0 = 0; s0 < g.shares; s0 += U) {
    f32x4_t v[U][C::NT];
#pragma unroll
    for (int s = 0; s < U; ++s)
#pragma unroll
      for (int j = 0; j < C::NT; ++j)
        v[s][j] = s0 + s < g.shares ? *share_at<C>(g, cut, s0 + s, i, j) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < U; ++s)
#pragma unroll
      for (int j = 0; j < C::NT; ++j) acc[j] += v[s][j];
  }
  finish<C, DUAL>(g, epi, m0, n0, wm, wn, i, acc);
}

}  // namespace
}  // namespace ffn
