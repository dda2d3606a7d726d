// Activations of the gated product, in fp32, and their derivatives.
#pragma once

#include "cci_block.hpp"
#include "cci_device.hpp"

namespace cci {

// exp, erf and tanh are the device library's.  1 / (1 + exp(-x)) tends to 0
// or 1 at either end without overflow into NaN for finite x.
// The activation is uniform over a launch.
__device__ __forceinline__ float act_value(Act act, float x) {
  switch (act) {
    case Act::RELU: return x > 0.0f ? x : (x != x ? x : 0.0f);
    case Act::SILU: return x / (1.0f + expf(-x));
    case Act::GELU: return 0.5f * x * (1.0f + erff(x * 0.70710678f));
    case Act::GELU_TANH: return 0.5f * x * (1.0f + tanhf(0.79788456f * (x + 0.044715f * x * x * x)));
    default: return x;
  }
}

// act(x) and act'(x).
template <Act A>
__device__ __forceinline__ void act_both(float x, float& a, float& d) {
  if constexpr (A == Act::RELU) {
    a = act_value(Act::RELU, x);
    d = x > 0.0f ? 1.0f : (x != x ? x : 0.0f);
  } else if constexpr (A == Act::SILU) {
    const float s = 1.0f / (1.0f + expf(-x));
    a = x * s;
    d = s * (1.0f + x * (1.0f - s));
  } else if constexpr (A == Act::GELU) {
    const float c = 0.5f * (1.0f + erff(x * 0.70710678f));
    a = x * c;
    d = c + x * 0.39894228f * expf(-0.5f * x * x);
  } else if constexpr (A == Act::GELU_TANH) {
    const float x2 = x * x;
    const float t = tanhf(0.79788456f * (x + 0.044715f * x * x2));
    const float e = 1.0f - t * t;  // 0 far out, where x2 may overflow
    a = 0.5f * x * (1.0f + t);
    d = 0.5f * (1.0f + t) + (e == 0.0f ? 0.0f : 0.5f * x * e * 0.79788456f * (1.0f + 0.134145f * x2));
  } else {
    a = x;
    d = 1.0f;
  }
}

}  // namespace cci
