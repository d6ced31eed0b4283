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

// log(1 + exp(x)) = max(x, 0) + log(1 + e) with e = exp(-|x|) <= 1, and log(1 + e) = 2 atanh(e / (2 + e)): the odd series, whose argument is at most
// 1/3, ends after s^15 / 15 (what follows is below 3^-17 / 17 of s = 4e-10 of the result), so small steps keep their relative precision.
// `slope` receives sigmoid(x), from the same exponential.
__device__ __forceinline__ float softplus(float x, float &slope)
{
    const float e = exp_of(-fabsf(x)), s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
    float p = 1.f / 15;
    p = __builtin_fmaf(p, q, 1.f / 13);
    p = __builtin_fmaf(p, q, 1.f / 11);
    p = __builtin_fmaf(p, q, 1.f / 9);
    p = __builtin_fmaf(p, q, 1.f / 7);
    p = __builtin_fmaf(p, q, 1.f / 5);
    p = __builtin_fmaf(p, q, 1.f / 3);
    p = __builtin_fmaf(p, q, 1.f);
    const float r = __builtin_amdgcn_rcpf(1.f + e);
    slope = x < 0.f ? e * r : r;
    return __builtin_fmaf(2.f * s, p, fmaxf(x, 0.f));
}
__device__ __forceinline__ float softplus(float x)
{
    float slope;
    return softplus(x, slope);
}

}  // namespace sv
