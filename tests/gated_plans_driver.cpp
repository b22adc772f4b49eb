// Host check of the plans of the gated block's products: whatever the sizes, the tiles that are cut along k
// are among the launch's, the same number of each problem's, every share has steps, the shares' sums fit the
// room that is set aside for products of as many rows or more, and so do the adapters' plans.  Prints
// "plans cut" and exits 0, or the first plan that does not fit and exits 1.
#include <cstdint>
#include <cstdio>

#include "ffn_gated_internal.h"

namespace {

int64_t g_plans = 0, g_cut = 0;

void tile_size(ffn::Tile t, int* bm, int* bn) {
  switch (t) {
    case ffn::Tile::T16: *bm = 16, *bn = 64; return;
    case ffn::Tile::T64: *bm = 64, *bn = 64; return;
    case ffn::Tile::T64x128: *bm = 64, *bn = 128; return;
    case ffn::Tile::T128: *bm = 128, *bn = 128; return;
    case ffn::Tile::T128x256: *bm = 128, *bn = 256; return;
    default: *bm = 256, *bn = 256; return;
  }
}

bool check(bool f32, int problems, int M, int64_t n, int steps, bool adapters, bool tokens) {
  const ffn::Plan p = ffn::choose_tile(f32, problems, M, n, steps, adapters, tokens);
  int bm, bn;
  tile_size(p.tile, &bm, &bn);
  const int64_t each = (int64_t)((M + bm - 1) / bm) * ((n + bn - 1) / bn);
  const int64_t bytes = (int64_t)p.cut * p.shares * bm * bn * 4;
  ++g_plans;
  g_cut += p.cut > 0;
  const bool few = tokens && M <= 64;
  const bool ok = ffn::tile_rows(p.tile) == bm && p.shares >= 1 && p.cut >= 0 && p.cut % problems == 0 &&
                  p.cut / problems <= each && (p.cut == 0) == (p.shares == 1) && (p.cut == 0 || p.shares <= steps) &&
                  (p.cut == 0 || bytes <= (int64_t)ffn::share_bytes_most(f32, problems, M, n, tokens)) &&
                  (few || p.tile != ffn::Tile::T16) && !(adapters && p.tile == ffn::Tile::T256) &&
                  each * problems * p.shares < ((int64_t)1 << 31) &&
                  // the adapters' plan of the tile's rows
                  (int64_t)((M + bm - 1) / bm) * (1 + 2 * bm) <= (int64_t)ffn::plan_ints(M);
  if (!ok)
    std::printf("f32 %d problems %d M %d n %lld steps %d adapters %d: tile %dx%d cut %d shares %d\n", f32, problems, M,
                (long long)n, steps, adapters, bm, bn, p.cut, p.shares);
  return ok;
}

}  // namespace

int main() {
  static const int sizes[] = {1,   2,   8,   15,  16,  17,   48,   63,   64,   65,   100,  127,  128,   129,   200,  255,  256,
                              257, 300, 513, 520, 777, 1000, 1365, 2000, 2560, 3840, 4096, 7168, 8192, 14231, 14336, 28672};
  static const int more[] = {57344, 65536, 600000, 1 << 20};
  for (int f32 = 0; f32 < 2; ++f32)
    for (int a = 0; a < 2; ++a)
      for (int M : sizes)
        for (int n : sizes)
          for (int steps : {1, 3, 7, 8, 9, 16, 40, 64, 129, 224, 448, 896, 3000})
            for (int problems = 1; problems <= 3; ++problems)
              if (!check(f32, problems, M, n, steps, a, problems == 1) || !check(f32, problems, M, n, steps, false, false))
                return 1;
  for (int f32 = 0; f32 < 2; ++f32)
    for (int M : more)
      for (int n : sizes)
        for (int steps : {1, 8, 64, 448})
          if (!check(f32, 1, M, n, steps, false, true) || !check(f32, 1, n, M, steps, true, true) ||
              !check(f32, 3, M, n, steps, false, false))
            return 1;
  // room for M rows is room for fewer
  for (int f32 = 0; f32 < 2; ++f32)
    for (int64_t n : {1, 64, 520, 4096, 57344}) {
      size_t low = 0;
      for (int M : sizes) {
        const size_t b = ffn::share_bytes_most(f32, 1, M, n, true);
        if (b < low) {
          std::printf("room for %d rows of %lld: %zu, for fewer %zu\n", M, (long long)n, b, low);
          return 1;
        }
        low = b;
      }
    }
  std::printf("%lld %lld\n", (long long)g_plans, (long long)g_cut);
  return 0;
}
