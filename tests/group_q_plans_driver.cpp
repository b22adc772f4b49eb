// Host check of the tiles of the products with group scales.  Reads lines "xf32 gated group T n_in n_out" and prints for
// each "nt wk u whole ns chunk per_share shares blocks lds", the library's own plan.
#include <cstdio>

#include "ffn_group_q_internal.h"

int main() {
  int xf32, gated, group, T, n_in, n_out;
  while (scanf("%d %d %d %d %d %d", &xf32, &gated, &group, &T, &n_in, &n_out) == 6) {
    const ffn::GqPlan p = ffn::gq_plan(xf32, gated, group, T, n_in, n_out);
    printf("%d %d %d %d %d %d %d %d %d %zu\n", p.nt, p.wk, p.u, (int)p.whole, p.ns, p.chunk, p.per_share, p.shares, p.blocks,
           ffn::gq_lds(xf32, p, T));
  }
  return 0;
}
