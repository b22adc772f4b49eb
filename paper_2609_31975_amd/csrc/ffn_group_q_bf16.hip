// Products with group scales of bf16 tokens.
#include "ffn_group_q_kernels.h"

namespace ffn {

hipError_t launch_group_q_bf16(bool sf32, bool gated, const GqArgs& a, const GqPlan& p, hipStream_t st) {
  return gated ? launch_form<false, true>(sf32, a, p, st) : launch_form<false, false>(sf32, a, p, st);
}

}  // namespace ffn
