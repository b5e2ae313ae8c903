// The activations of the gated feed-forward block, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include "lobra_mlora.h"

namespace lobra {

// 1 / (1 + exp(-v)): v_exp and v_rcp, each within an ulp or so.  exp(-v) = inf: 0.
__device__ __forceinline__ float logistic(float v)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
}

constexpr float kGeluC = 0.7978845608028654f, kGeluK = 0.044715f;     // sqrt(2 / pi)

// a(g).  gelu: (1 + tanh v) / 2 = 1 / (1 + exp(-2 v))
template <int ACT> __device__ __forceinline__ float activate(float g)
{
    if (ACT == LOBRA_ACT_SILU) return g * logistic(g);
    return g * logistic(2.f * kGeluC * (g + kGeluK * g * g * g));
}

// a(g), and a'(g) in da.  gelu, with p = (1 + tanh v) / 2: (1 - tanh^2 v) / 2 = 2 p (1 - p)
template <int ACT> __device__ __forceinline__ float activate(float g, float& da)
{
    if (ACT == LOBRA_ACT_SILU) {
        const float q = logistic(g);
        da = q * (1.f + g * (1.f - q));
        return g * q;
    }
    const float g2 = g * g, p = logistic(2.f * kGeluC * g * (1.f + kGeluK * g2));
    const float s = 2.f * p * (1.f - p);
    da = s == 0.f ? p : p + g * s * kGeluC * (1.f + 3.f * kGeluK * g2);      // (s = 0: g^2 may be inf)
    return g * p;
}

}  // namespace lobra
