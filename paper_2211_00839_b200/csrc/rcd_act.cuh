// Activations of rcd_linear and their derivatives, in fp32.
#pragma once

#include "rcd_elem.cuh"

namespace rcd {

#ifdef __CUDACC__
constexpr float kRootHalf = 0.70710678118654752f, kRootInv2Pi = 0.39894228040143268f, kTanhScale = 0.79788456080286536f, kTanhCube = 0.044715f;

// One instruction each, results below the normal range as 0: 2^x within 2 units of fp32, 1 / x within one; 1 / infinity is 0.
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float inverse_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2e = 1.44269504088896341f;
// erf by formula 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions (absolute error at most 1.5e-7, three units of
// fp32 next to 1), without branches: many of them side by side in a kernel's epilogue are short.
__device__ __forceinline__ float erf_as(float x)
{
    const float a = fabsf(x), t = inverse_fast(fmaf(0.3275911f, a, 1.0f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return copysignf(fmaf(-poly, exp2_fast(-kLog2e * a * a), 1.0f), x);
}
// tanh(u) = 1 - 2 / (1 + exp(2 u)); an infinite exponential makes the quotient 0.
__device__ __forceinline__ float tanh_exp(float u) { return fmaf(-2.0f, inverse_fast(1.0f + exp2_fast(2.0f * kLog2e * u)), 1.0f); }
__device__ __forceinline__ float logistic(float z) { return inverse_fast(1.0f + exp2_fast(-kLog2e * z)); }

template <int kAct>
__device__ __forceinline__ float activate_as(float z)
{
    if constexpr (kAct == RCD_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;      // (a NaN stays one)
    if constexpr (kAct == RCD_ACT_GELU) return 0.5f * z * (1.0f + erf_as(z * kRootHalf));
    if constexpr (kAct == RCD_ACT_GELU_TANH) return 0.5f * z * (1.0f + tanh_exp(kTanhScale * (z + kTanhCube * z * z * z)));
    if constexpr (kAct == RCD_ACT_SILU) return z * logistic(z);
    return z;
}
template <int kAct>
__device__ __forceinline__ float slope_as(float z)
{
    if constexpr (kAct == RCD_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    if constexpr (kAct == RCD_ACT_GELU) return 0.5f * (1.0f + erf_as(z * kRootHalf)) + z * exp2_fast(-0.5f * kLog2e * z * z) * kRootInv2Pi;
    if constexpr (kAct == RCD_ACT_GELU_TANH) {
        const float t = tanh_exp(kTanhScale * (z + kTanhCube * z * z * z));
        return 0.5f * (1.0f + t) + 0.5f * z * (1.0f - t * t) * kTanhScale * (1.0f + 3.0f * kTanhCube * fminf(z * z, 1e30f));     // (0 times that, not times infinity)
    }
    if constexpr (kAct == RCD_ACT_SILU) {
        const float s = logistic(z);
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}
// z becomes act(z); d becomes d act'(z).  Which one is asked once for all.
template <int N, int kAct>
__device__ __forceinline__ void activate_all(float (&z)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) z[j] = activate_as<kAct>(z[j]);
}
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act)
{
    switch (act) {
    case RCD_ACT_RELU: activate_all<N, RCD_ACT_RELU>(z); break;
    case RCD_ACT_GELU: activate_all<N, RCD_ACT_GELU>(z); break;
    case RCD_ACT_GELU_TANH: activate_all<N, RCD_ACT_GELU_TANH>(z); break;
    case RCD_ACT_SILU: activate_all<N, RCD_ACT_SILU>(z); break;
    default: break;
    }
}
template <int N, int kAct>
__device__ __forceinline__ void slopes_all(float (&d)[N], const float (&z)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) d[j] *= slope_as<kAct>(z[j]);
}
template <int N>
__device__ __forceinline__ void slopes(float (&d)[N], const float (&z)[N], int act)
{
    switch (act) {
    case RCD_ACT_RELU: slopes_all<N, RCD_ACT_RELU>(d, z); break;
    case RCD_ACT_GELU: slopes_all<N, RCD_ACT_GELU>(d, z); break;
    case RCD_ACT_GELU_TANH: slopes_all<N, RCD_ACT_GELU_TANH>(d, z); break;
    case RCD_ACT_SILU: slopes_all<N, RCD_ACT_SILU>(d, z); break;
    default: break;
    }
}
#endif

}  // namespace rcd
