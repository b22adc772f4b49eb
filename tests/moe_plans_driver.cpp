// Host check of the experts' launches.  Reads lines "f32 T d d_ff E k" and prints for each "slots ldz pieces part_rows", the
// library's own plan.
#include <cstdio>

#include "ffn_moe_internal.h"

int main() {
  int f32, T, d, d_ff, E, k;
  while (scanf("%d %d %d %d %d %d", &f32, &T, &d, &d_ff, &E, &k) == 6)
    printf("%d %d %d %zu\n", ffn::moe_slots(T, E, k), ffn::moe_ldz(d_ff), ffn::moe_pieces(f32, T, d, d_ff, E, k),
           ffn::moe_part_rows(f32, T, d, d_ff, E, k));
  return 0;
}
