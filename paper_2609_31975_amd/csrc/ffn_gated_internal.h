// Internal declarations of the gated block's and the adapters' launches.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ffn {

constexpr int kCUs = 256;

// Gate activation, threshold and the up side of one call.
struct BlockForm {
  int act, silu_up;
  float t;
};

// Adapters of one product (internal form): ids, stack sizes, and the v rows computed for them.
struct AdapterSet {
  int n = 0, r = 0, rp = 0;
  const int32_t* ids = nullptr;
  const float* scale = nullptr;
  int32_t* plan = nullptr;  // room for plan_ints(T); filled by launch_adapter_v
  float* part = nullptr;    // adapter_share_bytes_most(...)
};

// The tile of a product (or of `problems` alike, in one launch) with M rows and n columns over `steps` steps
// of 128 bytes, and how many of all its tiles, the last ones, are cut along k, in how many shares.  tokens: the
// rows are tokens (few of them take tiles of few rows).
enum class Tile { T16, T64, T64x128, T128, T128x256, T256 };
struct Plan {
  Tile tile;
  int cut, shares;
};
Plan choose_tile(bool f32, int problems, int M, int64_t n, int steps, bool adapters, bool tokens);
int tile_rows(Tile t);
bool takes_adapters(Tile t);  // products with adapters are built for it
// Room for the shares of a product of M rows or fewer and n columns, whatever its plan.
size_t share_bytes_most(bool f32, int problems, int M, int64_t n, bool tokens);
// Entries of the adapters' plan of T tokens, whatever the tile: one or more tiles of tile_rows() rows.
inline size_t plan_ints(int T) { return 2 * ((size_t)T + 256) + T / 16 + 1; }

// Tokens that one launch takes of a product with n columns, a multiple of 256, so that no grid comes to 2^32 work items:
// the tiles have at most one to 16 results, or, with few columns, 8 to a token, and A x takes 1024 to a token where its
// rows are no whole chunks.  The forward calls take more tokens in pieces.  The backward call needs none: a save and
// gradients of so many tokens are larger than the card's memory.
inline int tokens_a_launch(int64_t n, bool adapters) {
  const int64_t by_columns = ((int64_t)1 << 35) / n / 256 * 256, most = (int64_t)1 << (adapters ? 21 : 27);
  return (int)(by_columns < most ? by_columns : most);
}

// Shapes: rows of dp elements (d rounded up to whole chunks), hidden rows of ldf (d_ff rounded up to 64).
struct BlockShape {
  int T, d, d_ff, dp, ldf;
};

// part, here and below: share_bytes_most(...) of the product.
//
// z = A(x W1^T - t) U(x W3^T), and g, v in fp32 when g is not null.  v2: A_j x of the two projections'
// adapters (null: none), b2 their B stacks.
hipError_t launch_block_hidden(bool f32, const BlockShape& s, const void* x, const void* w_gate, const void* w_up,
                               const BlockForm& form, const AdapterSet& ad, const void* const v2[2],
                               const void* const b2[2], void* z, float* g, float* v, float* part, hipStream_t st);
// out [T][n] = z W (W [k][n], k strided) with adapters (b null: none), or the sum of two such products.
struct TokenProduct {
  const void* a[2];  // [T][lda]
  const void* b[2];  // KS: [k][ldb]; KC: [n][ldb]
  int products, T, n, k, lda, ldb, ldo;
  void* out;
  float* part;
  AdapterSet ad;
  const void* v;
  const void* ab;
};
Plan token_plan(bool f32, int T, int n, int k, int products, bool adapters);
Plan hidden_plan(bool f32, const BlockShape& s, bool adapters);
hipError_t launch_token_product_ks(bool f32, const TokenProduct& p, hipStream_t st);
hipError_t launch_token_product_kc(bool f32, const TokenProduct& p, hipStream_t st);
// dg, dv [T][ldf] from dz = dy W2 and the saved g, v.
hipError_t launch_block_dz(bool f32, const BlockShape& s, const void* dy, const void* w_down_t, const BlockForm& form,
                           const float* g, const float* v, void* dg, void* dv, float* part, hipStream_t st);
// up to three weight gradients out[i] [d_ff][d] = a[i]^T b[i], a [T][ldf], b [T][dp]
hipError_t launch_block_dw(bool f32, const BlockShape& s, int count, const void* const a[3], const void* const b[3],
                           void* const out[3], float* part, hipStream_t st);
// The launch of A x: tokens of k elements, 16 to a group; tiles: through LDS tiles.  A group's adapters go to `lanes`
// workgroups, a row to `shares`; blocks: groups x lanes x shares.
struct AdapterPlan {
  bool tiles;
  int lanes, shares, blocks;
};
AdapterPlan adapter_plan(bool f32, int T, int k, int rp, int count);
// Room for the shares of the sums, for T tokens or fewer and ranks up to rp.
size_t adapter_share_bytes_most(int T, int rp, int count);
// v[i] [T][rp] = scale_j A_j x for up to two stacks, and ad.plan for the product of tile `t` that reads them
hipError_t launch_adapter_v(bool f32, int T, int k, int ldx, const void* x, const AdapterSet& ad, int count,
                            const void* const a[2], void* const v[2], Tile t, hipStream_t st);
// rows of n elements to rows of np, the rest zero
hipError_t launch_pad_rows(bool f32, int64_t rows, int n, int np, const void* src, void* dst, hipStream_t st);

}  // namespace ffn
