// Activations of the gated product, in fp32, and their derivatives.
#pragma once

#include "cci_block.hpp"
#include "cci_device.hpp"

namespace cci {

// 1 / (1 + exp(-x)), within about 4 + |x| steps of fp32: exp by the hardware's
// exp2 (the product with log2(e) is off by half a step, which grows with |x|)
// and the hardware's reciprocal.  0 and 1 at the ends, where exp overflows.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// Phi(x).  By the complement of the error function: 1 + erf cancels for x < 0,
// 4% off at -5, and the up value that it meets knows no bound.
__device__ __forceinline__ float normal_cdf(float x) { return 0.5f * erfcf(x * -0.70710678f); }

// The activation is uniform over a launch.  The tanh approximation of the GELU
// is x sigmoid(2 z), since (1 + tanh z) / 2 is sigmoid(2 z).
__device__ __forceinline__ float act_value(Act act, float x) {
  switch (act) {
    case Act::RELU: return x > 0.0f ? x : (x != x ? x : 0.0f);
    case Act::SILU: return x * sigmoid(x);
    case Act::GELU: return x * normal_cdf(x);
    case Act::GELU_TANH: return x * sigmoid(1.5957691f * (x + 0.044715f * x * x * x));
    default: return x;
  }
}

// y = act(g) u over eight elements (one branch on the activation).
__device__ __forceinline__ void act_times8(Act act, const float (&g)[8], const float (&u)[8], float (&y)[8]) {
  const auto each = [&](Act a) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = act_value(a, g[e]) * u[e];
  };
  switch (act) {
    case Act::RELU: each(Act::RELU); break;
    case Act::SILU: each(Act::SILU); break;
    case Act::GELU: each(Act::GELU); break;
    case Act::GELU_TANH: each(Act::GELU_TANH); break;
    default: each(Act::NONE);
  }
}

// act(x) and act'(x).
template <Act A>
__device__ __forceinline__ void act_both(float x, float& a, float& d) {
  if constexpr (A == Act::RELU) {
    a = act_value(Act::RELU, x);
    d = x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
  } else if constexpr (A == Act::SILU) {
    const float s = sigmoid(x);
    a = x * s;
    d = s * (1.0f + x * (1.0f - s));
  } else if constexpr (A == Act::GELU) {
    const float c = normal_cdf(x);
    a = x * c;
    d = c + x * 0.39894228f * __expf(-0.5f * x * x);
  } else if constexpr (A == Act::GELU_TANH) {
    const float x2 = x * x;
    const float s = sigmoid(1.5957691f * (x + 0.044715f * x * x2));
    const float e = s * (1.0f - s);  // 0 far out, where x2 may overflow
    a = x * s;
    d = s + (e == 0.0f ? 0.0f : x * e * 1.5957691f * (1.0f + 0.134145f * x2));
  } else {
    a = x;
    d = 1.0f;
  }
}

}  // namespace cci
