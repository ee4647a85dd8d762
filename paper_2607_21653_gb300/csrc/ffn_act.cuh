// The feed-forward block's activations and their derivatives.
#pragma once

#include "ffn.cuh"
#include "ptx.cuh"

namespace molt {

constexpr float kFfnLog2e = 1.4426950408889634f;

// act(g), and with it act'(g)
__device__ __forceinline__ float ffn_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2 sqrt(2 / pi) log2 e, and 0.044715 of it
constexpr float kGeluA = 2.f * 0.7978845608028654f, kGeluB = 0.044715f;
template <bool kGrad>
__device__ __forceinline__ float ffn_activate(int act, float g, float& d) {
  if (act == kActRelu) {
    d = g > 0.f ? 1.f : 0.f;
    return g <= 0.f ? 0.f : g;
  }
  if (act == kActSilu) {
    const float p = ffn_rcp(1.f + ex2_approx(-kFfnLog2e * g));
    if (kGrad) d = fmaf(g * (1.f - p), p, p);
    return g * p;
  }
  // (1 + tanh z) / 2 = 1 / (1 + e^(-2 z)), z = sqrt(2 / pi) (g + 0.044715 g^3)
  const float q = g * g;
  const float p = ffn_rcp(1.f + ex2_approx(-kFfnLog2e * kGeluA * g * fmaf(kGeluB, q, 1.f)));
  if (kGrad) d = fmaf(g * p * (1.f - p), kGeluA * fmaf(3.f * kGeluB, q, 1.f), p);
  return g * p;
}

}  // namespace molt
