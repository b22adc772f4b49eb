// The kernels of include/ffn_group_q.h: products of a decode step's tokens with 4-bit weights that have a
// scale (and an offset) for every group of codes along the summed dimension.  Not part of the public ABI.
//
// The codes' bytes bound it, and the work that a byte brings: two codes to turn into matrix operands.  So:
//   - The codes enter the bf16 products unscaled.  Two nibbles of a dword become two bf16 of value 24 + code (16 + u has
//     u in its top mantissa bits; u = code + 8): 8 operations for 8 codes.  What the 24 add, 24 times the sum of the
//     same x, is in a table in LDS that the sums start from.  A group's sum is then multiplied by its row's scale.
//     One fp32 token: a table of every eight columns' sums, see k_group_q1.
//   - More fp32 tokens: the codes enter as code / 16, exactly, from a conversion of nibbles (19 operations for 8 codes), and the
//     16 comes off the joined sums.  With 24 in them a group's sums are several times the result, for x of one sign many times,
//     and every addition rounds by that (4096 columns of one sign: 3.0e-6 of the result's norm, so 1.1e-7, a plain fp32 product 4.8e-7; 48
//     tokens of 4096 -> 14336 twice, groups of 64 with offsets: 60 us, so 61; 16 tokens, groups of 128: 31, so 35).
//   - One token: dot products on the vector ALUs (k_group_q1).  More: v_mfma_f32_16x16x32_bf16 (k_group_q).
//   - Tokens are the A operand, weight rows the B operand: a lane's results are of one weight row, whose scale it
//     holds.
//   - A lane loads 16 bytes, 32 codes of a row; the four lanes of a row 128 (a window).  Where a window lies in one
//     group, MFMA f takes dword f of every lane, and x in the same order.  Else the four dwords are transposed between
//     the lanes (two v_permlane32_swap, two v_permlane16_swap), and each MFMA has 32 codes in a row.
//   - x lies in LDS, as bf16 in the order of the operands; fp32 x as three bf16 parts, three products.
#pragma once

#include <algorithm>
#include <type_traits>

#include "ffn_group_q_internal.h"
#include "ffn_mfma.h"
#include "ffn_step_device.h"

namespace ffn {
namespace {

// The four pairs of a dword, elements (0, 4), (1, 5), (2, 6), (3, 7), as 24 + code: a shift and one three-input operation
// each (mask, and an exclusive or that sets 16's bits and turns the code's sign bit over).  An instruction takes one constant
// from the scalar side: `mask` is kMask in a vector register.
constexpr uint32_t kMask = 0x00780078u;
// A plain vector: the compiler takes LDS reads of types that it does not know to wait for all loads into LDS.
__device__ __forceinline__ bf16x8_t lds_operand(const char* p) {
  return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p));
}
// all vector memory operations of this wave, the ones into LDS among them
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }
__device__ __forceinline__ uint4 codes8(uint32_t w, uint32_t mask) {
  constexpr uint32_t s = 0x41C041C0u;
  return make_uint4((w << 3 & mask) ^ s, (w >> 1 & mask) ^ s, (w >> 5 & mask) ^ s, (w >> 9 & mask) ^ s);
}

// The same pairs as code / 16, exactly (a signed nibble's conversion divides by 16).
__device__ __forceinline__ uint4 codes8_exact(uint32_t w) {
  auto two = [&](int j) { return f_to_bf2(__builtin_amdgcn_cvt_off_f32_i4(w >> (4 * j)), __builtin_amdgcn_cvt_off_f32_i4(w >> (4 * j + 16))); };
  return make_uint4(two(0), two(1), two(2), two(3));
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

// 8 columns of a token as bf16 in the order of the operands, elements (0, 4), (1, 5), (2, 6), (3, 7), fp32 in three parts; their sum.
template <bool XF32>
__device__ __forceinline__ float split_piece(const uint4 (&v)[XF32 ? 2 : 1], uint4 (&d)[XF32 ? 3 : 1]) {
  float f[8];
  if constexpr (XF32) {
    const uint4 lo = v[0], hi = v[1];
    float r[8] = {comp<0>(lo), comp<0>(hi), comp<1>(lo), comp<1>(hi), comp<2>(lo), comp<2>(hi), comp<3>(lo), comp<3>(hi)};
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = r[e];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = f_to_bf2(r[2 * e], r[2 * e + 1]);
        r[2 * e] -= __uint_as_float(w[e] << 16);
        r[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
      }
      d[q] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    unpack(WBf16{}, v[0], f);
    d[0] = make_uint4(__builtin_amdgcn_perm(v[0].z, v[0].x, 0x05040100u), __builtin_amdgcn_perm(v[0].z, v[0].x, 0x07060302u),
                      __builtin_amdgcn_perm(v[0].w, v[0].y, 0x05040100u), __builtin_amdgcn_perm(v[0].w, v[0].y, 0x07060302u));
  }
  return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// A chunk of windows of x's T rows, on its way into LDS: rows of chunk * 256 + 16 bytes (the 16 spread the rows over the
// banks), plane after plane, in pieces of 8 columns, of which a thread holds up to gq_units.  Columns past n_in are zero.
// Behind the planes the table of -24 times the sum of x: SUMS rows for a window, of all tokens of the tiles.  fp32 x: for offsets
// alone.
template <bool XF32, int SUMS, int TOKENS>
struct XPieces {
  static constexpr int N = gq_units(XF32), THREADS = 512, SPAN = N * THREADS;
  uint4 v[N][XF32 ? 2 : 1];

  __device__ __forceinline__ void load(const GqArgs& a, int w0, int from) {
    const int units = a.chunk * (kWindow / 8);
    const Buf xb = make_buf(a.x, (uint32_t)a.T * a.n_in * (XF32 ? 4 : 2));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = from + j * THREADS + (int)threadIdx.x, t = i / units, k = w0 * kWindow + (i - t * units) * 8;
      const uint32_t o = t < a.T && k < a.n_in ? ((uint32_t)t * a.n_in + k) * (XF32 ? 4 : 2) : kOOB;
      v[j][0] = ldb(xb, o);
      if constexpr (XF32) v[j][1] = ldb(xb, o + 16);
    }
  }
  static __device__ __forceinline__ float* table(const GqArgs& a, char* lds) {
    return reinterpret_cast<float*>(lds + (XF32 ? 3 : 1) * a.T * (a.chunk * 2 * kWindow + 16));
  }
  __device__ __forceinline__ void store(const GqArgs& a, char* lds, int from) const {
    const int units = a.chunk * (kWindow / 8), stride = a.chunk * 2 * kWindow + 16;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = from + j * THREADS + (int)threadIdx.x, t = i / units;
      uint4 d[XF32 ? 3 : 1];
      const float sum = group_sum(split_piece<XF32>(v[j], d), 16 / SUMS);  // the pieces of a window lie in 16 neighbouring lanes
      if (t >= a.T) continue;
      const int c = i - t * units;
      if (c % (16 / SUMS) == 0) table(a, lds)[c / (16 / SUMS) * TOKENS + t] = -24.f * sum;
      char* p = lds + t * stride + c * 16;
#pragma unroll
      for (int q = 0; q < (XF32 ? 3 : 1); ++q) *reinterpret_cast<uint4*>(p + q * a.T * stride) = d[q];
    }
  }
};

// Two token tiles and more: x is taken apart once for all workgroups, in memory, into whole operands: for window w, MFMA f, part
// p and token tile t the 64 lanes' 16 bytes at ((4 w + f) P + p) NT + t, so that a chunk is one piece of memory and LDS reads
// have no bank conflicts; and the table [windows][NS][tokens].  Tokens past the last one are left as they are in there: a token's
// operands reach its own results alone.  48 fp32 tokens of 4096: 5 us.
template <bool XF32, int NS, int NT>
__global__ __launch_bounds__(256) void k_group_q_split(GqArgs a, int windows) {
  constexpr int P = XF32 ? 3 : 1;
  const int pieces = windows * (kWindow / 8), i = blockIdx.x * 256 + threadIdx.x, t = i / pieces, c = i - t * pieces;
  const Buf xb = make_buf(a.x, (uint32_t)a.T * a.n_in * (XF32 ? 4 : 2));
  const uint32_t o = t < a.T && c * 8 < a.n_in ? ((uint32_t)t * a.n_in + c * 8) * (XF32 ? 4 : 2) : kOOB;
  uint4 v[XF32 ? 2 : 1], d[P];
  v[0] = ldb(xb, o);
  if constexpr (XF32) v[1] = ldb(xb, o + 16);
  const float sum = group_sum(split_piece<XF32>(v, d), 16 / NS);
  if (t >= a.T) return;
  const int w = c / 16, f = NS > 1 ? c % 16 / 4 : c % 4, g = NS > 1 ? c % 4 : c % 16 / 4;
#pragma unroll
  for (int p = 0; p < P; ++p) a.planes[(((size_t)(w * 4 + f) * P + p) * NT + t / 16) * 64 + g * 16 + t % 16] = d[p];
  if (c % (16 / NS) == 0) a.sums[(size_t)(c / (16 / NS)) * (16 * NT) + t] = -24.f * sum;
}
// WK windows of it, straight into LDS.
template <bool XF32, int NS, int NT, int WK>
struct XCopy {
  static constexpr int P = XF32 ? 3 : 1, BYTES = WK * 4 * P * NT * 1024, SUMS = WK * NS * 16 * NT;  // 512 sums or fewer
  static __device__ __forceinline__ float* table(const GqArgs&, char* lds) { return reinterpret_cast<float*>(lds + BYTES); }
  static __device__ __forceinline__ void copy(const GqArgs& a, char* lds, int w0) {
    const char* from = reinterpret_cast<const char*>(a.planes) + (size_t)w0 * (BYTES / WK);
    const int wave = uniform(threadIdx.x >> 6);
#pragma unroll
    for (int j = 0; j < BYTES / 8192; ++j) {  // 8 waves, 1 KB each
      const int at = (j * 8 + wave) * 1024;
      __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(const_cast<char*>(from) + at + lane_id() * 16),
                                       (__attribute__((address_space(3))) void*)(lds + at), 16, 0, 0);
    }
    if (wave * 64 < SUMS)  // whole waves: the table's rows in memory and in LDS have room for four sums a window
      __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)(a.sums + (size_t)w0 * NS * 16 * NT + wave * 64 + lane_id()),
                                       (__attribute__((address_space(3))) void*)(lds + BYTES + wave * 256), 4, 0, 0);
  }
};

// 8 waves: WK of them share a row tile's windows, 8 / WK row tiles of 16 to a workgroup.  NT: 16-token
// tiles.  U: windows of a wave in a batch; the next batch is on its way during a batch's products.  NSX: scales of a window, 1
// (groups that are multiples of 128), 2 or 4 (of 64 and 32, a window's scales side by side in whole dwords), or 8: any other
// group, a scale for every 32 codes.  OFF: there are offsets.  WHOLE: all of a share's x is in LDS at once.
// 48 fp32 tokens of 4096 -> 14336 twice, groups of 64 with offsets: 55 us, 0.61 PFLOP/s of the three parts' products, the matrix
// pipes busy for 23% and the vector ALUs for 33%: each step's operands come from LDS behind a barrier, and the codes of a batch
// are taken apart between its products.
template <bool XF32, bool SF32, bool GATED, int NSX, bool OFF, int NT, int WK, int U, bool WHOLE>
__global__ __launch_bounds__(512, NT == 1 ? 4 : 2) void k_group_q(GqArgs a) {
  constexpr int M = GATED ? 2 : 1, WR = 8 / WK, P = XF32 ? 3 : 1, UNIT = WK * U;
  constexpr int NS = gq_scales(NSX), PER = 4 / NS;
  constexpr bool TR = NS > 1;
  extern __shared__ __align__(16) char lds[];
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int wk = wave % WK;
  // rows past the last one repeat it, and are not stored
  const uint32_t row = min((int)(blockIdx.x * WR + wave / WK) * 16 + n, a.n_out - 1);
  const int first = blockIdx.y * a.per_share, last = min(a.windows, first + a.per_share);
  const uint32_t row_bytes = (uint32_t)a.n_in / 2, ss = SF32 ? 4 : 2;

  Buf cb[M], sb[M], ob[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    cb[m] = make_buf(a.w[m].codes, row_bytes * a.n_out);
    sb[m] = make_buf(a.w[m].scales, (uint32_t)a.n_out * a.groups * ss);
    ob[m] = make_buf(a.w[m].offsets, a.w[m].offsets ? (uint32_t)a.n_out * a.groups * ss : 0u);
  }
  const uint32_t code_at = row * row_bytes + g * 16, scale_at = row * a.groups * ss;

  // A window's scales: NS floats, or with bf16 ones NS / 2 dwords of two (one of one).
  constexpr int SD = SF32 ? NS : (NS + 1) / 2;
  struct Scales {
    uint32_t v[SD];
    __device__ __forceinline__ float at(int f) const {
      if constexpr (SF32) return __uint_as_float(v[f]);
      else return __uint_as_float(f & 1 ? v[f >> 1] & 0xffff0000u : v[f >> 1] << 16);
    }
  };
  struct Batch {
    uint4 codes[U][M];
    Scales sc[U][M], of[OFF ? U : 1][M];
  };
  auto load_scales = [&](const Buf& b, int w, Scales& s) {
    if constexpr (NSX == 2 || NSX == 4) {
      // one load: a gather of 16 rows' scales costs what one of their codes does (two a group with offsets; groups of 64,
      // 48 fp32 tokens of 4096 -> 14336 twice: 77 us, so 67)
      const uint32_t at = scale_at + (w < last ? w * NS * ss : kOOB);
      if constexpr (SD == 1) {
        s.v[0] = (uint32_t)ldb32(b, at);
      } else if constexpr (SD == 2) {
        typedef uint32_t u2 __attribute__((ext_vector_type(2)));
        const u2 v = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(b.r, at, 0, 0));
        s.v[0] = v[0];
        s.v[1] = v[1];
      } else {
        const uint4 v = ldb(b, at);
        s.v[0] = v.x;
        s.v[1] = v.y;
        s.v[SD - 2] = v.z;
        s.v[SD - 1] = v.w;
      }
    } else {
      uint32_t raw[NS];
#pragma unroll
      for (int f = 0; f < NS; ++f) {
        const uint32_t k32 = w * 4 + f * PER, gi = (uint32_t)((uint64_t)k32 * a.div_group >> 31);
        const uint32_t at = scale_at + (w < last && (int)(k32 * 32) < a.n_in ? gi * ss : kOOB);
        raw[f] = SF32 ? (uint32_t)ldb32(b, at) : (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, at, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < SD; ++i) s.v[i] = SF32 ? raw[i] : NS == 1 ? raw[0] : raw[2 * i] | raw[(2 * i + 1) % NS] << 16;
    }
  };
  // Lines of 128 bytes are read in two halves, by the same wave or its neighbour: through the caches (streamed past them
  // the same reads came to 5.2 TB/s, through them to 5.6).  Codes behind the row's end, of the next row or zeros behind the
  // matrix, meet zeros of x; scales behind the share's or the row's end are zeros, never the next row's.
  auto load = [&](int w_first, Batch& b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int w = w_first + wk * U + u;
#pragma unroll
      for (int m = 0; m < M; ++m) {
        b.codes[u][m] = ldb(cb[m], code_at + w * (kWindow / 2));
        load_scales(sb[m], w, b.sc[u][m]);
        if constexpr (OFF) load_scales(ob[m], w, b.of[u][m]);
      }
    }
  };

  f32x4_t acc[NT][M] = {};
  const int stride = a.chunk * 2 * kWindow + 16;
  int xrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xrow[t] = min(t * 16 + n, a.T - 1) * stride;
  uint32_t mask = kMask;
  asm("" : "+v"(mask));

  // Where all of x lies in LDS, the workgroups go through it from different places on: with rows of 2^n bytes all of them
  // would be on the same few memory channels at any time (rows of 4096 bytes: 4.3 TB/s, so 5.25).
  const int batches = (last - first + UNIT - 1) / UNIT;
  int turn = WHOLE ? (int)((blockIdx.x * 5 + (blockIdx.x >> 3)) % (uint32_t)batches) : 0;
  Batch even, odd;
  load(first + turn * UNIT, even);
  using Pieces = std::conditional_t<NT == 1, XPieces<XF32, NS, 16>, XCopy<XF32, NS, NT, WK>>;
  std::conditional_t<NT == 1, Pieces, int> xp;
  if constexpr (NT == 1) xp.load(a, first, 0);
  constexpr int BUFFERS = NT > 1 ? gq_buffers(XF32, NT) : 1;
  char* buf = lds;
  if constexpr (BUFFERS == 2) Pieces::copy(a, buf, first);
  for (int c0 = first; c0 < last; c0 += a.chunk) {
    if constexpr (BUFFERS == 2) {
      // this chunk is here; the next one goes where the last one was, which all waves have left
      wait_loads();
      __syncthreads();
      char* other = lds + (buf == lds ? gq_buffer(XF32, NT) : 0);
      if (c0 + a.chunk < last) Pieces::copy(a, other, c0 + a.chunk);
    } else {
      if (c0 != first) __syncthreads();
      if constexpr (NT == 1) {
        xp.store(a, buf, 0);
        if constexpr (WHOLE) {
          for (int i = Pieces::SPAN; i < a.T * a.chunk * (kWindow / 8); i += Pieces::SPAN) {
            xp.load(a, c0, i);
            xp.store(a, buf, i);
          }
        }
      } else {
        Pieces::copy(a, buf, c0);
        wait_loads();
      }
      __syncthreads();
      if constexpr (NT == 1 && !WHOLE)
        if (c0 + a.chunk < last) xp.load(a, c0 + a.chunk, 0);
    }
    auto products = [&](const Batch& cur, Batch& nxt) {
      const int here = first + turn * UNIT - c0;  // a window of the chunk
      turn = turn + 1 == batches ? 0 : turn + 1;
      load(first + turn * UNIT, nxt);
      issue_barrier();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int w = here + wk * U + u;  // the chunk is a multiple of UNIT
        uint4 q[M];
#pragma unroll
        for (int m = 0; m < M; ++m) q[m] = TR ? transpose4(cur.codes[u][m]) : cur.codes[u][m];
        // The sums of tokens past the last one, and their starts, stay in their own rows, which are not stored.
        const f32x4_t* tab = reinterpret_cast<const f32x4_t*>(Pieces::table(a, buf)) + w * NS * 4 * NT + g;
        f32x4_t sum[NT][M], starts[2][NT];
        // x of an MFMA f and what its sums start from; with more than one token tile the next f's are on their way during its products
        bf16x8_t x[2][NT][P];
        auto load_x = [&](int f) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if ((!XF32 || OFF) && f % PER == 0) starts[f / PER & 1][t] = tab[f / PER * 4 * NT + t * 4];
#pragma unroll
            for (int p = 0; p < P; ++p) {
              const char* at = NT == 1 ? buf + xrow[t] + w * 2 * kWindow + (TR ? f * 64 + g * 16 : g * 64 + f * 16) + p * a.T * stride
                                       : buf + ((w * 4 + f) * P * NT + p * NT + t) * 1024 + lane * 16;
              x[f & 1][t][p] = lds_operand(at);
            }
          }
        };
        load_x(0);
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          if (f < 3) load_x(f + 1);
          if constexpr (NT > 1) issue_barrier();
          bf16x8_t wf[M];
#pragma unroll
          for (int m = 0; m < M; ++m) {
            const uint32_t w8 = f == 0 ? q[m].x : f == 1 ? q[m].y : f == 2 ? q[m].z : q[m].w;
            wf[m] = bf8(XF32 ? codes8_exact(w8) : codes8(w8, mask));
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int m = 0; m < M; ++m)
              if (f % PER == 0) sum[t][m] = XF32 ? f32x4_t{} : starts[f / PER & 1][t];
#pragma unroll
          for (int p = P - 1; p >= 0; --p)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int m = 0; m < M; ++m) sum[t][m] = mfma16(x[f & 1][t][p], wf[m], sum[t][m]);
          if (f % PER == PER - 1) {
            const int s = f / PER;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
              for (int m = 0; m < M; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  acc[t][m][i] += cur.sc[u][m].at(s) * sum[t][m][i];
              if constexpr (OFF) {
                const f32x4_t sx = starts[s & 1][t] * (XF32 ? -1.f / 384.f : -1.f / 24.f);
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                  for (int i = 0; i < 4; ++i) acc[t][m][i] += cur.of[u][m].at(s) * sx[i];
              }
            }
          }
          // one f at a time: more of them in registers spill, and with NSX 8, whose scales are 16-bit or 32-bit loads of their own,
          // gated kernels of one token tile spill all the same, 17 to 48 registers (10752 -> 10688, 8 bf16 tokens, fp32 scales and
          // offsets: groups of 128 54 us, of 32 63, of 96 223)
          if constexpr (GATED && NS == 4) issue_barrier();
        }
      }
    };
    // two batches that take turns: a copy of one to the other would wait for it
    int left = (min(a.chunk, last - c0) + UNIT - 1) / UNIT;
    if constexpr (NT == 1) {
      for (; left >= 2; left -= 2) {
        products(even, odd);
        products(odd, even);
      }
    }
    if (left) {  // all there is of a chunk with more than one token tile
      products(even, odd);
      even = odd;
    }
    if constexpr (BUFFERS == 2) buf = lds + (buf == lds ? gq_buffer(XF32, NT) : 0);
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
      if constexpr (XF32) {
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] *= 16.f;
      }
      if (a.part) {
#pragma unroll
        for (int m = 0; m < M; ++m) a.part[(((size_t)blockIdx.y * M + m) * a.T + tok) * a.n_out + o] = v[m];
      } else {
        store_as<XF32>(a.y, (size_t)tok * a.n_out + o, GATED ? act_product(ActForm{a.act, a.silu_up, a.t}, v[0], v[M - 1]) : v[0]);
      }
    }
  }
}

// One token.  A load takes 128 bytes of 8 rows (whole lines, streamed past the caches), 32 codes a lane, and those lie in
// one group whatever it is; a wave takes 16 rows, two loads, of 256 columns (a window here).  A lane's products with its
// 32 x are 16 v_dot2; 8 lanes share a row.  x in LDS: piece f (8 columns) of a window's 8 lanes side by side.  Bound by
// the codes' bytes: 28672 -> 8192, 121 MB, 22.6 us (5.4 TB/s; the vector ALUs busy for 43%), 4096 -> 14336 twice, 61 MB, 13
// us (4.7 TB/s, two or three batches a wave).
template <bool XF32, bool SF32, bool GATED, bool OFF, int WK>
__global__ __launch_bounds__(512, 4) void k_group_q1(GqArgs a) {
  constexpr int M = GATED ? 2 : 1, WR = 8 / WK, P = XF32 ? 3 : 1, UNIT = WK, WIN = 2 * kWindow;
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  extern __shared__ __align__(16) char lds[];
  const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), c = lane & 7, wk = wave % WK;
  const int row0 = (blockIdx.x * WR + wave / WK) * 16 + (lane >> 3);
  const int first = blockIdx.y * a.per_share, last = min(a.windows, first + a.per_share);
  const uint32_t row_bytes = (uint32_t)a.n_in / 2, ss = SF32 ? 4 : 2;
  uint32_t code_at[2], scale_at[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {  // rows past the last one repeat it, and are not stored
    const uint32_t row = min(row0 + 8 * s, a.n_out - 1);
    code_at[s] = row * row_bytes + c * 16;
    scale_at[s] = row * a.groups * ss;
  }
  Buf cb[M], sb[M], ob[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    cb[m] = make_buf(a.w[m].codes, row_bytes * a.n_out);
    sb[m] = make_buf(a.w[m].scales, (uint32_t)a.n_out * a.groups * ss);
    ob[m] = make_buf(a.w[m].offsets, a.w[m].offsets ? (uint32_t)a.n_out * a.groups * ss : 0u);
  }
  struct Batch {
    uint4 codes[2][M];
    uint32_t sc[2][M], of[2][M];
  };
  auto raw = [&](const Buf& b, uint32_t i) -> uint32_t {
    if constexpr (SF32) return (uint32_t)ldb32(b, i);
    else return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b.r, i, 0, 0);
  };
  auto value = [](uint32_t v) { return __uint_as_float(SF32 ? v : v << 16); };
  // codes and scales behind a row's or the share's end: as in k_group_q
  auto load = [&](int w_first, Batch& b) {
    const int w = w_first + wk;
    const uint32_t k32 = w * 8 + c, gi = __umulhi(2 * k32, a.div_group);
    const uint32_t at = w < last && (int)(k32 * 32) < a.n_in ? gi * ss : kOOB;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int m = 0; m < M; ++m) {
        b.codes[s][m] = ldb_nt(cb[m], code_at[s] + w * (WIN / 2));
        b.sc[s][m] = raw(sb[m], scale_at[s] + at);
        if constexpr (OFF) b.of[s][m] = raw(ob[m], scale_at[s] + at);
      }
  };

  float acc[2][M] = {};
  uint32_t mask = kMask;
  asm("" : "+v"(mask));
  const int plane = a.chunk * WIN * 2;
  float* tab = reinterpret_cast<float*>(lds + P * plane);
  const Buf xb = make_buf(a.x, (uint32_t)a.n_in * (XF32 ? 4 : 2));
  // the workgroups start at different places of the rows: as in k_group_q
  const int batches = (last - first + UNIT - 1) / UNIT;
  int turn = last - first <= a.chunk ? (int)((blockIdx.x * 5 + (blockIdx.x >> 3)) % (uint32_t)batches) : 0;
  Batch even, odd;
  load(first + turn * UNIT, even);
  for (int c0 = first; c0 < last; c0 += a.chunk) {
    if (c0 != first) __syncthreads();
    for (int i = threadIdx.x; i < a.chunk * (WIN / 8); i += 512) {
      const int k = c0 * WIN + i * 8;
      const uint32_t o = k < a.n_in ? (uint32_t)k * (XF32 ? 4 : 2) : kOOB;
      char* p = lds + (i >> 5) * (WIN * 2) + (i & 3) * 128 + (i >> 2 & 7) * 16;
      uint4 v[XF32 ? 2 : 1], d[P];
      v[0] = ldb(xb, o);
      if constexpr (XF32) v[1] = ldb(xb, o + 16);
      const float s = XF32 ? split_piece<XF32>(v, d) : group_sum(split_piece<XF32>(v, d), 4);
#pragma unroll
      for (int q = 0; q < P; ++q) *reinterpret_cast<uint4*>(p + q * plane) = d[q];
      if constexpr (XF32) tab[i] = -24.f * s;  // of every piece: see below
      else if ((i & 3) == 0) tab[i >> 2] = -24.f * s;
    }
    __syncthreads();
    auto products = [&](const Batch& cur, Batch& nxt) {
      const int here = first + turn * UNIT - c0;  // a window of the chunk
      turn = turn + 1 == batches ? 0 : turn + 1;
      load(first + turn * UNIT, nxt);
      issue_barrier();
      const int w = here + wk;  // the chunk is a multiple of WK
      f32x4_t starts{};
      if constexpr (XF32) starts = reinterpret_cast<const f32x4_t*>(tab)[w * 8 + c];
      const float gone = XF32 ? (starts[0] + starts[1]) + (starts[2] + starts[3]) : tab[w * 8 + c];
      uint4 x[P][4];
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int f = 0; f < 4; ++f) x[p][f] = *reinterpret_cast<const uint4*>(lds + p * plane + w * (WIN * 2) + f * 128 + c * 16);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const uint4 q = cur.codes[s][m];
          const uint4 d[4] = {codes8(q.x, mask), codes8(q.y, mask), codes8(q.z, mask), codes8(q.w, mask)};
          auto dot = [&](float sum, const uint4& l, const uint4& r) {
            auto two = [&](uint32_t a2, uint32_t b2) {
              sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, a2), __builtin_bit_cast(bf16x2_t, b2), sum, false);
            };
            two(l.x, r.x);
            two(l.y, r.y);
            two(l.z, r.z);
            two(l.w, r.w);
            return sum;
          };
          float sum = XF32 ? 0.f : gone;
#pragma unroll
          for (int p = P - 1; p >= (XF32 ? 1 : 0); --p)
#pragma unroll
            for (int f = 0; f < 4; ++f) sum = dot(sum, d[f], x[p][f]);
          if constexpr (XF32) {
            // the largest part: eight columns at a time, each sum from its own start, so that no partial sum is larger than those
            // eight make it (all 32 from one start: 1.3e-6 of the norm, so 6e-7)
            sum += (dot(starts[0], d[0], x[0][0]) + dot(starts[1], d[1], x[0][1])) +
                   (dot(starts[2], d[2], x[0][2]) + dot(starts[3], d[3], x[0][3]));
          }
          acc[s][m] += value(cur.sc[s][m]) * sum;
          if constexpr (OFF) acc[s][m] += value(cur.of[s][m]) * (gone * (-1.f / 24.f));
        }
    };
    // two batches that take turns: a copy of one to the other would wait for it
    int left = (min(a.chunk, last - c0) + UNIT - 1) / UNIT;
    for (; left >= 2; left -= 2) {
      products(even, odd);
      products(odd, even);
    }
    if (left) {
      products(even, odd);
      even = odd;
    }
  }

  // 8 lanes of a row, then the WK waves, in their order
  float* red = reinterpret_cast<float*>(lds);
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const float v = group_sum(acc[s][m], 8);
      if (c == 0) red[(wave * M + m) * 16 + s * 8 + (lane >> 3)] = v;
    }
  __syncthreads();
  const int r = threadIdx.x >> 4, o = (blockIdx.x * WR + r) * 16 + (threadIdx.x & 15);
  if (r >= WR || o >= a.n_out) return;
  float v[M] = {};
#pragma unroll
  for (int k = 0; k < WK; ++k)
#pragma unroll
    for (int m = 0; m < M; ++m) v[m] += red[((r * WK + k) * M + m) * 16 + (threadIdx.x & 15)];
  if (a.part) {
#pragma unroll
    for (int m = 0; m < M; ++m) a.part[((size_t)blockIdx.y * M + m) * a.n_out + o] = v[m];
  } else {
    store_as<XF32>(a.y, o, GATED ? act_product(ActForm{a.act, a.silu_up, a.t}, v[0], v[M - 1]) : v[0]);
  }
}

template <bool XF32, bool GATED>
__global__ __launch_bounds__(256) void k_group_q_join(GqArgs a, int shares) {
  constexpr int M = GATED ? 2 : 1;
  const size_t count = (size_t)a.T * a.n_out;
  for (size_t e = (size_t)blockIdx.x * 256 + threadIdx.x; e < count; e += (size_t)gridDim.x * 256) {
    float p[kGqSharesMost][M], v[M] = {};
#pragma unroll
    for (int s = 0; s < kGqSharesMost; ++s)
#pragma unroll
      for (int m = 0; m < M; ++m) p[s][m] = s < shares ? a.part[((size_t)s * M + m) * count + e] : 0.f;
#pragma unroll
    for (int s = 0; s < kGqSharesMost; ++s)
#pragma unroll
      for (int m = 0; m < M; ++m) v[m] += p[s][m];
    store_as<XF32>(a.y, e, GATED ? act_product(ActForm{a.act, a.silu_up, a.t}, v[0], v[M - 1]) : v[0]);
  }
}

template <bool XF32, bool SF32, bool GATED, bool OFF>
hipError_t launch_one(const GqArgs& a, const GqPlan& p, hipStream_t st) {
  const dim3 grid(p.blocks, p.shares);
  auto go = [&](auto wk) {
    k_group_q1<XF32, SF32, GATED, OFF, wk.value><<<grid, 512, gq_lds(XF32, p, 1), st>>>(a);
    return hipGetLastError();
  };
  return p.wk == 8 ? go(Int<8>{}) : p.wk == 4 ? go(Int<4>{}) : go(Int<2>{});
}

template <bool XF32, bool SF32, bool GATED, int NSX, bool OFF>
hipError_t launch_tiles(const GqArgs& a, const GqPlan& p, hipStream_t st) {
  const size_t lds = std::max<size_t>(gq_lds(XF32, p, a.T), 8 * (GATED ? 2 : 1) * 1024);
  const dim3 grid(p.blocks, p.shares);
  auto go = [&](auto nt, auto wk, auto u, auto whole) {
    k_group_q<XF32, SF32, GATED, NSX, OFF, nt.value, wk.value, u.value, whole.value><<<grid, 512, lds, st>>>(a);
    return hipGetLastError();
  };
  constexpr int U = gq_batch(GATED, NSX), NS = gq_scales(NSX);
  constexpr Int<0> no;
  constexpr Int<1> yes;
  if (p.whole) {
    if (p.wk == 8) return go(Int<1>{}, Int<8>{}, Int<U>{}, yes);
    return p.wk == 4 ? go(Int<1>{}, Int<4>{}, Int<U>{}, yes) : go(Int<1>{}, Int<2>{}, Int<U>{}, yes);
  }
  if (p.nt == 1) {
    if constexpr (XF32)  // bf16 tokens leave room for 8 waves' windows
      if (p.wk == 4) return go(Int<1>{}, Int<4>{}, Int<1>{}, no);
    return go(Int<1>{}, Int<8>{}, Int<1>{}, no);
  }
  const int windows = ceil_div(a.windows, kGqWaves) * kGqWaves, blocks = ceil_div(a.T * windows * (kWindow / 8), 256);
  if (p.nt == 2) k_group_q_split<XF32, NS, 2><<<blocks, 256, 0, st>>>(a, windows);
  else if (p.nt == 3) k_group_q_split<XF32, NS, 3><<<blocks, 256, 0, st>>>(a, windows);
  else k_group_q_split<XF32, NS, 4><<<blocks, 256, 0, st>>>(a, windows);
  if (const hipError_t e = hipGetLastError()) return e;
  constexpr Int<kGqWaves> w;
  return p.nt == 2 ? go(Int<2>{}, w, Int<1>{}, no) : p.nt == 3 ? go(Int<3>{}, w, Int<1>{}, no) : go(Int<4>{}, w, Int<1>{}, no);
}

template <bool XF32, bool GATED>
hipError_t launch_form(bool sf32, const GqArgs& a, const GqPlan& p, hipStream_t st) {
  auto by_scales = [&](auto s, auto o) {
    if (p.nt == 0) return launch_one<XF32, s.value, GATED, o.value>(a, p, st);
    return p.ns == 1 ? launch_tiles<XF32, s.value, GATED, 1, o.value>(a, p, st)
           : p.ns == 2 ? launch_tiles<XF32, s.value, GATED, 2, o.value>(a, p, st)
           : p.ns == 4 ? launch_tiles<XF32, s.value, GATED, 4, o.value>(a, p, st)
                       : launch_tiles<XF32, s.value, GATED, 8, o.value>(a, p, st);
  };
  const bool off = a.w[0].offsets != nullptr;
  const hipError_t e = sf32 ? (off ? by_scales(Int<1>{}, Int<1>{}) : by_scales(Int<1>{}, Int<0>{}))
                            : (off ? by_scales(Int<0>{}, Int<1>{}) : by_scales(Int<0>{}, Int<0>{}));
  if (e != hipSuccess || p.shares == 1) return e;
  const size_t blocks = ceil_div<size_t>((size_t)a.T * a.n_out, 256);
  k_group_q_join<XF32, GATED><<<(int)std::min<size_t>(blocks, 4096), 256, 0, st>>>(a, p.shares);
  return hipGetLastError();
}

}  // namespace
}  // namespace ffn
