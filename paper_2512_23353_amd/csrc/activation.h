// Activations of the policy's linear layers and their slopes, in fp32.
#pragma once

#include <type_traits>

#include "common.h"

namespace isopo {

enum class Act { kNone, kRelu, kGelu, kSilu };

constexpr float kLog2e = 1.4426950408889634f;

// 1 / (1 + e^-z): one exponential and one reciprocal of the transcendental unit, within 2 ulp; 0 and 1 where e^-z leaves fp32
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * z)); }

constexpr float kGeluA = 0.7978845608028654f, kGeluB = 0.044715f;       // sqrt(2/pi)

// z (1 + tanh u) / 2 = z / (1 + e^-2u) with u = kGeluA (z + kGeluB z^3)
template <Act A>
__device__ __forceinline__ float activate(float z) {
  if constexpr (A == Act::kRelu) return z > 0.f || z != z ? z : 0.f;
  if constexpr (A == Act::kSilu) return z * sigmoid(z);
  if constexpr (A == Act::kGelu) return z * sigmoid(2.f * kGeluA * (z + kGeluB * z * z * z));
  return z;
}

template <Act A>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (A == Act::kRelu) return z > 0.f ? 1.f : 0.f;
  if constexpr (A == Act::kSilu) {
    const float s = sigmoid(z);
    return s + z * s * (1.f - s);
  }
  if constexpr (A == Act::kGelu) {
    const float s = sigmoid(2.f * kGeluA * (z + kGeluB * z * z * z)), t = s * (1.f - s);
    return t == 0.f ? s : s + z * t * (2.f * kGeluA) * (1.f + 3.f * kGeluB * z * z);          // (z^2 may leave fp32 where t is 0)
  }
  return 1.f;
}

// f(std::integral_constant<Act, A>) for the A that `act` names
template <class F>
auto with_act(Act act, F&& f) {
  switch (act) {
    case Act::kRelu: return f(std::integral_constant<Act, Act::kRelu>{});
    case Act::kGelu: return f(std::integral_constant<Act, Act::kGelu>{});
    case Act::kSilu: return f(std::integral_constant<Act, Act::kSilu>{});
    default: return f(std::integral_constant<Act, Act::kNone>{});
  }
}

}  // namespace isopo
