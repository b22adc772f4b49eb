// Device-side helpers shared by the calls around and in place of a block.  Not part of the public ABI.
#pragma once

#include "ffn_device.h"
#include "ffn_step_host.h"

namespace ffn {
namespace {

__device__ __forceinline__ float bf_to_f(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ uint16_t f_to_bf(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ uint32_t f_to_bf2(float lo, float hi) {
  typedef float f2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
  const f2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2_t));
}

template <bool F32>
__device__ __forceinline__ void store_as(void* p, size_t i, float v) {
  if constexpr (F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = f_to_bf(v);
}

// A(h - t) U(v) of the gated block (ffn_gated.h): a NaN gate value is not above the border of FFN_ACT_RELU and
// FFN_ACT_RSPLUS.
__device__ __forceinline__ float act_product(const ActForm& f, float h, float v) {
  const float g = h - f.t;
  float a = f.act == FFN_ACT_RELU ? g : g / (1.f + expf(-g));
  if (f.act != FFN_ACT_SILU) a = g > 0.f ? a : 0.f;
  return a * up_value(f.silu_up, v);
}

}  // namespace
}  // namespace ffn
