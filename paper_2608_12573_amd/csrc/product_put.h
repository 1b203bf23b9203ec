// One output of the dense product: bias, activation and residual, whatever they
// are.
#pragma once

#include "product.h"

namespace profk {

namespace {

__device__ __forceinline__ float act_any(float z, int act) {
  if (act == PROFK_ACT_RELU) return act_of<PROFK_ACT_RELU>(z);
  if (act == PROFK_ACT_GELU) return act_of<PROFK_ACT_GELU>(z);
  if (act == PROFK_ACT_SILU) return act_of<PROFK_ACT_SILU>(z);
  return z;
}

__device__ __forceinline__ void put(const ProdArgs& g, uint32_t i, uint32_t j, float z) {
  const size_t at = static_cast<size_t>(i) * g.J + j;
  if (g.bias) z += g.bias[j];
  float y = act_any(z, g.act);
  if (g.residual) {
    const size_t r = i * g.residual_stride + j;
    y += g.out_dtype == PROFK_F32 ? static_cast<const float*>(g.residual)[r]
                                  : static_cast<float>(static_cast<const __bf16*>(g.residual)[r]);
  }
  if (g.out_dtype == PROFK_F32) {
    static_cast<float*>(g.out)[at] = y;
    if (g.pre) static_cast<float*>(g.pre)[at] = z;
  } else {
    static_cast<__bf16*>(g.out)[at] = static_cast<__bf16>(y);
    if (g.pre) static_cast<__bf16*>(g.pre)[at] = static_cast<__bf16>(z);
  }
}

}  // namespace

}  // namespace profk
