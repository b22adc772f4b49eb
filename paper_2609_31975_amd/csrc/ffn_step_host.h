// Host-side checks shared by the calls around and in place of a block (norms, group-scaled products,
// experts).  Not part of the public ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "ffn_sparse.h"

namespace ffn {
namespace {

constexpr int64_t kMaxElems = (int64_t)1 << 31;

inline bool aligned(const void* p, uintptr_t a = 16) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool known(ffn_dtype_t w) { return w == FFN_F32 || w == FFN_BF16; }
template <class T>
T ceil_div(T a, T b) {  // a up to the type's largest
  return a / b + (a % b != 0);
}

struct Carver {
  char* base;
  size_t off = 0;
  void* take(size_t bytes) {
    void* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  }
};

// Gate activation, threshold and the up side of one call; opt's other fields are for LoPA gating.
struct ActForm {
  int act, silu_up;
  float t;
};
inline int check_act(const ffn_options_t* o, float t, ActForm* f) {
  *f = ActForm{FFN_ACT_RELU, 0, t};
  if (!o) return FFN_OK;
  if (o->act != FFN_ACT_RELU && o->act != FFN_ACT_RSPLUS && o->act != FFN_ACT_SILU) return FFN_ERR_OPTION;
  if (o->silu_up != 0 && o->silu_up != 1) return FFN_ERR_OPTION;
  if (o->g_idx || o->g_sign || o->rms_norm || o->rms_gain) return FFN_ERR_OPTION;
  f->act = o->act;
  f->silu_up = o->silu_up;
  return FFN_OK;
}

}  // namespace
}  // namespace ffn
