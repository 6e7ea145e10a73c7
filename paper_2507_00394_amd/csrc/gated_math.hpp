// What the gated projections do with an element.
#pragma once
#include "helix_common.hpp"
#include "kernels.hpp"

namespace helix {

// The activation and its derivative.
template <Activation ACT>
__device__ __forceinline__ void activate(float g, float& value, float& slope) {
  if constexpr (ACT == Activation::silu) {   // s = 1 / (1 + e^-g):  g s,  s (1 + g (1 - s))
    const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * g));
    value = g * s;
    slope = s * fmaf(g, 1.f - s, 1.f);
  } else {   // P the normal distribution, P' its density:  g P,  P + g P'
    // P(-|g|) = erfc(|g| / sqrt 2) / 2 by Abramowitz and Stegun 7.1.26, off by 7.5e-8 and its fp32 roundings, 2.6e-7 in all: one exponential for it and the density, and no branch,
    // where the library's erff has one for every element.
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(g), 1.f)), e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * g * g);
    const float poly = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
    const float tail = 0.5f * poly * t * e, P = g < 0.f ? tail : 1.f - tail;
    value = g * P;
    slope = fmaf(g * 0.39894228f, e, P);
  }
}

}  // namespace helix
