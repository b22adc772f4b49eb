// Host check of the norms' launches.  Reads lines "T d" and prints for each "tpr ept blocks" of the forward call and "tpr ept
// groups" of the backward call, the library's own plan.
#include <cstdio>

#include "ffn_norm_internal.h"

int main() {
  int T, d;
  while (scanf("%d %d", &T, &d) == 2) {
    const ffn::NormPlan f = ffn::norm_forward_plan(d), b = ffn::norm_backward_plan(d);
    printf("%d %d %d %d %d %d\n", f.tpr, f.ept, ffn::norm_blocks(T, d), b.tpr, b.ept, ffn::norm_groups(T, d));
  }
  return 0;
}
