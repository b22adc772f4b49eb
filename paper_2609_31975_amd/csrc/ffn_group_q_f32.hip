// Products with group scales of f32 tokens.
#include "ffn_group_q_kernels.h"

namespace ffn {

hipError_t launch_group_q_f32(bool sf32, bool gated, const GqArgs& a, const GqPlan& p, hipStream_t st) {
  return gated ? launch_form<true, true>(sf32, a, p, st) : launch_form<true, false>(sf32, a, p, st);
}

}  // namespace ffn
