// The activations of the selective operators and of group norm, in fp32.
#pragma once

#include "common.hpp"

namespace sv {

constexpr float kLog2E = 1.44269504088896341f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + exp_of(-x)); }
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }
// silu'(x) with s = sigmoid(x)
__device__ __forceinline__ float silu_slope(float x, float s) { return s * __builtin_fmaf(x, 1.f - s, 1.f); }

// log(1 + exp(x)) = max(x, 0) + log(1 + e) with e = exp(-|x|) <= 1, and log(1 + e) = 2 atanh(s), s = e / (2 + e) <= 1/3: atanh(s) / s = 1 + q r(q) in
// q = s^2 <= 1/9, r of degree 3 through the Chebyshev nodes of that range (off by 1.6e-8 of atanh, a quarter of a rounding).  Small steps keep their
// relative precision.  `slope` receives sigmoid(x), from the same exponential.
__device__ __forceinline__ float softplus(float x, float &slope)
{
    const float e = exp_of(-fabsf(x)), s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float p = 2 * 0.13433776651071558f;
    p = __builtin_fmaf(p, q, 2 * 0.14116977575001344f);
    p = __builtin_fmaf(p, q, 2 * 0.20003835452329463f);
    p = __builtin_fmaf(p, q, 2 * 0.3333331983251299f);
    p = __builtin_fmaf(p, q, 2.f);
    const float r = __builtin_amdgcn_rcpf(1.f + e);
    slope = x < 0.f ? e * r : r;
    return __builtin_fmaf(s, p, fmaxf(x, 0.f));
}
__device__ __forceinline__ float softplus(float x)
{
    float slope;
    return softplus(x, slope);
}

}  // namespace sv
