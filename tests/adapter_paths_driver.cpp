// The paths that calls with adapters take, from the library's own host arithmetic.  Reads lines "b|p f32 T d n r":
// the block with adapters on all three projections (n: d_ff), or the projection call (n: n_out).  Prints for each
// its products as "name tile cut" and its A x launches as "name tiles shares stacks", cut and shares as 0 or 1 for
// none or some, separated by ';'.
#include <cstdio>

#include "ffn_gated_internal.h"

namespace {

void product(const char* name, const ffn::Plan& p) {
  static const char* tiles[] = {"16", "64", "64x128", "128", "128x256", "256"};
  std::printf("%s %s %d;", name, tiles[(int)p.tile], p.cut > 0);
}
void first_factor(const char* name, bool f32, int T, int k, int r, int stacks) {
  const int c = f32 ? 4 : 8;
  const ffn::AdapterPlan p = ffn::adapter_plan(f32, T, k, (r + c - 1) / c * c, stacks);
  std::printf("%s %d %d %d;", name, p.tiles, p.shares > 1, stacks);
}

}  // namespace

int main() {
  char op;
  int f32, T, d, n, r;
  while (std::scanf(" %c %d %d %d %d %d", &op, &f32, &T, &d, &n, &r) == 6) {
    if (op == 'b') {
      const int c = f32 ? 4 : 8;
      const ffn::BlockShape s{T, d, n, (d + c - 1) / c * c, (n + 63) / 64 * 64};
      first_factor("x", f32, T, d, r, 2);
      product("hidden", ffn::hidden_plan(f32, s, true));
      first_factor("z", f32, T, n, r, 1);
      product("down", ffn::token_plan(f32, T, d, n, 1, true));
    } else {
      first_factor("x", f32, T, d, r, 1);
      product("projection", ffn::token_plan(f32, T, n, d, 1, true));
    }
    std::printf("\n");
  }
  return 0;
}
