// The feed-forward block's activations and their derivatives.
#pragma once

#include <type_traits>

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
template <int kAct, bool kGrad>
__device__ __forceinline__ float ffn_activate(float g, float& d) {
  if constexpr (kAct == kActRelu) {
    d = g > 0.f ? 1.f : 0.f;
    return g <= 0.f ? 0.f : g;
  }
  if constexpr (kAct == kActSilu) {
    const float p = ffn_rcp(1.f + ex2_approx(-kFfnLog2e * g));
    if (kGrad) d = fmaf(g * (1.f - p), p, p);
    return g * p;
  }
  // (1 + tanh z) / 2 = 1 / (1 + e^(-2 z)), z = sqrt(2 / pi) (g + 0.044715 g^3)
  static_assert(kAct == kActRelu || kAct == kActSilu || kAct == kActGelu);
  // (p is 0 or 1 from |g| = 100 on; the derivative's g^2, infinite from 2^64 on, would make 0 times it NaN)
  const float q = fminf(g * g, 1e4f);
  const float p = ffn_rcp(1.f + ex2_approx(-kFfnLog2e * kGeluA * g * fmaf(kGeluB, q, 1.f)));
  if (kGrad) d = fmaf(g * p * (1.f - p), kGeluA * fmaf(3.f * kGeluB, q, 1.f), p);
  return g * p;
}

// f with the activation as a constant: a branch for every element keeps the compiler from
// interleaving their exponentials (the backward's tile of 256 x 256 took 30 us, not 10)
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
  if (act == kActSilu)
    f(std::integral_constant<int, kActSilu>{});
  else if (act == kActGelu)
    f(std::integral_constant<int, kActGelu>{});
  else
    f(std::integral_constant<int, kActRelu>{});
}

}  // namespace molt
