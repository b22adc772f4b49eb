// Host check of the launches of the gated block's and the adapters' forward calls: with the tokens that
// one launch takes, fewer of them, and the last of a call's pieces, no grid comes to 2^32 work items, the
// largest that HIP takes in a dimension.  Prints the number of grids and exits 0, or the first that is too large
// and exits 1.
#include <cstdint>
#include <cstdio>

#include "ffn_gated_internal.h"

namespace {

int64_t g_grids = 0;

bool fits(const char* what, int T, int64_t n, int k, int64_t blocks, int threads) {
  ++g_grids;
  const bool ok = blocks > 0 && blocks * threads < ((int64_t)1 << 32);
  if (!ok) std::printf("%s: T %d n %lld k %d: %lld workgroups of %d\n", what, T, (long long)n, k, (long long)blocks, threads);
  return ok;
}

bool product_fits(bool f32, int T, int64_t n, int steps, bool adapters) {
  const ffn::Plan p = ffn::choose_tile(f32, 1, T, n, steps, adapters, true);
  int bm = ffn::tile_rows(p.tile), bn = 256, threads = 512;
  if (p.tile == ffn::Tile::T16) bn = 64, threads = 128;
  if (p.tile == ffn::Tile::T64) bn = 64, threads = 256;
  if (p.tile == ffn::Tile::T64x128) bn = 128;
  if (p.tile == ffn::Tile::T128) bn = 128, threads = 256;
  const int64_t tiles = ((int64_t)T + bm - 1) / bm * ((n + bn - 1) / bn);
  return fits("product", T, n, steps, tiles - p.cut + (int64_t)p.cut * p.shares, threads) &&
         (p.cut == 0 || fits("join", T, n, steps, p.cut, threads));
}

// A x and its join, beside a product of `bm` rows a tile
bool adapters_fit(bool f32, int T, int k, int rp, int count, int bm) {
  const ffn::AdapterPlan p = ffn::adapter_plan(f32, T, k, rp, count);
  const int64_t plans = ((int64_t)T + bm - 1) / bm, lanes = p.tiles ? 2 : T < 16 ? T : 16;
  if (p.lanes != lanes || p.blocks != ((int64_t)T + 15) / 16 * lanes * p.shares || p.shares < 1 || p.shares > 8) {
    std::printf("T %d k %d rp %d: %d lanes, %d shares, %d blocks\n", T, k, rp, p.lanes, p.shares, p.blocks);
    return false;
  }
  const size_t sums = (size_t)p.shares * count * T * rp * 4;
  if (p.shares > 1 && sums > ffn::adapter_share_bytes_most(T, rp, count)) {
    std::printf("T %d k %d rp %d: the shares take %zu bytes\n", T, k, rp, sums);
    return false;
  }
  const int64_t join = p.shares > 1 ? ((int64_t)count * T * (rp / 4) + 255) / 256 : 0;
  return fits("A x", T, rp, k, p.blocks + (p.tiles ? 0 : plans), p.tiles ? 128 : 1024) &&
         fits("its join", T, rp, k, join + plans, 256);
}

}  // namespace

int main() {
  static const int64_t columns[] = {1, 2, 8, 63, 64, 65, 100, 128, 129, 255, 256, 257, 1000, 2048, 4097, 14336, 57344, 1 << 20, 1 << 21};
  for (int f32 = 0; f32 < 2; ++f32)
    for (int a = 0; a < 2; ++a)
      for (int64_t n : columns) {
        const int piece = ffn::tokens_a_launch(n, a);
        if (piece < 256 || piece % 256) {
          std::printf("%lld columns: pieces of %d tokens\n", (long long)n, piece);
          return 1;
        }
        // a whole piece, less, and the last pieces of calls of up to 2^31 - 1 tokens
        for (int T : {piece, piece - 1, piece - 255, piece / 2 + 1, piece / 3, (int)((((int64_t)1 << 31) - 1) % piece), 257, 64, 1}) {
          if (T < 1) continue;
          for (int steps : {1, 2, 8, 33, 448})
            if (!product_fits(f32, T, n, steps, a)) return 1;
          if (a)
            for (int k : {1, 7, 8, 64, 999, 1000, 4096, 1 << 20})
              for (int rp : {8, 16, 24, 128, 65536})
                for (int count = 1; count <= 2; ++count)
                  for (int bm : {64, 128})
                    if (!adapters_fit(f32, T, k, rp, count, bm)) return 1;
        }
      }
  std::printf("%lld\n", (long long)g_grids);
  return 0;
}
