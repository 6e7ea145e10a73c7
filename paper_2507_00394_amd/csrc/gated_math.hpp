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
    // P(-|g|) = e^(-g^2 / 2) t Q(t) with t = 1 / (1 + 0.3 |g|): one exponential for it and the density, and no branch, where the library's erff has one for every element.  Q is fitted to
    // e^(g^2 / 2) P(-|g|) / t on 0 <= |g| <= 14 (weighted least squares, the weights moved to where the relative error is largest until it was level), 1.5e-7 off RELATIVE to it, so that the negative
    // tail, where P + g P' and g P are small, is as good as the rest: with the roundings in fp32, P off by 2.2e-7 and g P by 3.8e-7 at most, and g P by 1e-6 of itself down to g = -4, 3e-6 to -8 and
    // 8e-6 to -13 (the rounding of the exponent), behind which it leaves the range of fp32.
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(g), 1.f)), e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * g * g);
    const float poly = fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(0.035674926f, t, -0.15720364f), t, 0.20635436f), t, -0.053684328f), t, 0.12856194f), t, 0.09991341f), t, 0.120753966f), t, 0.1196293f);
    const float tail = poly * t * e, P = g < 0.f ? tail : 1.f - tail;
    value = g * P;
    slope = fmaf(g * 0.39894228f, e, P);
  }
}

}  // namespace helix
