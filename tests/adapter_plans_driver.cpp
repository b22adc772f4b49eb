// Host check of the tiles of products with adapters: every plan for adapters has a tile that they are built
// for, and every plan a tile of its type.  Prints how often each tile was planned with adapters, in the order
// of ffn::Tile, and exits 0, or the first plan that is wrong and exits 1.
#include <cstdint>
#include <cstdio>

#include "ffn_gated_internal.h"

int main() {
  using ffn::Tile;
  static const int sizes[] = {1, 2, 8, 16, 17, 48, 64, 65, 100, 129, 200, 256, 300, 520, 777, 1365, 2100, 4096, 8192, 14336, 28672, 65536, 600000};
  long seen[6] = {};
  for (int f32 = 0; f32 < 2; ++f32)
    for (int a = 0; a < 2; ++a)
      for (int M : sizes)
        for (int n : sizes)
          for (int steps : {1, 3, 8, 16, 40, 64, 129, 448, 3000}) {
            const Tile t = ffn::choose_tile(f32, 1, M, n, steps, a, true).tile;
            const bool of_type = t == Tile::T16 || t == Tile::T64 || (t == Tile::T64x128) == (bool)f32;
            const bool built = t != Tile::T128 && t != Tile::T256;
            if (!of_type || (a && !built) || built != ffn::takes_adapters(t)) {
              std::printf("f32 %d M %d n %d steps %d adapters %d: tile %d\n", f32, M, n, steps, a, (int)t);
              return 1;
            }
            if (a) ++seen[(int)t];
          }
  for (long s : seen) std::printf("%ld ", s);
  std::printf("\n");
  return 0;
}
