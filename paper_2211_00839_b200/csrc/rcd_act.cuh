// Activations of rcd_linear and their derivatives, in fp32.
#pragma once

#include "rcd_elem.cuh"

namespace rcd {

#ifdef __CUDACC__
constexpr float kRootInv2Pi = 0.39894228040143268f, kTanhScale = 0.79788456080286536f, kTanhCube = 0.044715f;

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
// The normal distribution from -|z| on, and exp(-z^2 / 2): phi = t P(t) exp(-z^2 / 2) with t = 1 / (1 + |z| / sqrt(8)), the form of formula 7.1.26 of
// Abramowitz and Stegun, Handbook of Mathematical Functions.  P is of degree 8, fitted to the relative error up to |z| = 14 (4.3e-8): what
// is left below zero is never a difference of near numbers.  In fp32: some 6 units next to 0, and z^2 units from the exponential's
// argument.  Without branches and two values at a time (each rounded as alone): 301 us for 50 000 x 2048 x 2048 with z kept, 321 one at a time.
__device__ __forceinline__ float2 normal_tails(float2 z, float2 *density)
{
    const Two t = two(inverse_fast(fmaf(0.35355339f, fabsf(z.x), 1.0f)), inverse_fast(fmaf(0.35355339f, fabsf(z.y), 1.0f)));
    auto both = [](float c) { return two(c, c); };
    Two p = fma2(t, both(-0.0295355041f), both(0.142291993f));
    p = fma2(t, p, both(-0.243608341f));
    p = fma2(t, p, both(0.139042139f));
    p = fma2(t, p, both(-0.0133180469f));
    p = fma2(t, p, both(0.101345368f));
    p = fma2(t, p, both(0.121551454f));
    p = fma2(t, p, both(0.141187713f));
    p = fma2(t, p, both(0.141043201f));
    const Two zz = two(z.x, z.y);
    const float2 u = parts(mul2(both(-0.5f * kLog2e), mul2(zz, zz)));
    *density = make_float2(exp2_fast(u.x), exp2_fast(u.y));
    return parts(mul2(mul2(p, t), two(density->x, density->y)));
}
__device__ __forceinline__ float logistic(float z) { return inverse_fast(1.0f + exp2_fast(-kLog2e * z)); }
// The logistic function and its derivative, either of them as small as it is on both sides.
__device__ __forceinline__ float logistic_slope(float z, float *slope)
{
    const float e = exp2_fast(-kLog2e * fabsf(z)), p = inverse_fast(1.0f + e), q = e * p;
    *slope = q * p;
    return z < 0.0f ? q : p;
}
// 0.5 (1 + tanh(u)) is the logistic function of 2 u, which does not end in a difference: this is 2 u.
__device__ __forceinline__ float tanh_argument(float z) { return 2.0f * kTanhScale * (z * fmaf(kTanhCube, z * z, 1.0f)); }

template <int kAct>
__device__ __forceinline__ float activate_as(float z)
{
    if constexpr (kAct == RCD_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;      // (a NaN stays one)
    if constexpr (kAct == RCD_ACT_GELU_TANH) return z * logistic(tanh_argument(z));
    if constexpr (kAct == RCD_ACT_SILU) return z * logistic(z);
    return z;
}
template <int kAct>
__device__ __forceinline__ float slope_as(float z)
{
    if constexpr (kAct == RCD_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    if constexpr (kAct == RCD_ACT_GELU_TANH) {
        float slope;
        const float s = logistic_slope(tanh_argument(z), &slope);
        return fmaf(z * slope, 2.0f * kTanhScale * fmaf(3.0f * kTanhCube, fminf(z * z, 1e30f), 1.0f), s);     // (0 times that, not times infinity)
    }
    if constexpr (kAct == RCD_ACT_SILU) {
        float slope;
        const float s = logistic_slope(z, &slope);
        return fmaf(z, slope, s);
    }
    return 1.0f;
}
// z becomes act(z); d becomes d act'(z).  Which one is asked once for all.
template <int N, int kAct>
__device__ __forceinline__ void activate_all(float (&z)[N])
{
    if constexpr (kAct == RCD_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const float2 x = make_float2(z[j], z[j + 1 < N ? j + 1 : j]);
            float2 density;
            const float2 tail = normal_tails(x, &density);
            z[j] = x.x * (x.x < 0.0f ? tail.x : 1.0f - tail.x);
            if (j + 1 < N) z[j + 1] = x.y * (x.y < 0.0f ? tail.y : 1.0f - tail.y);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) z[j] = activate_as<kAct>(z[j]);
    }
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
    if constexpr (kAct == RCD_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            const float2 x = make_float2(z[j], z[j + 1 < N ? j + 1 : j]);
            float2 density;
            const float2 tail = normal_tails(x, &density);
            d[j] *= fmaf(x.x * density.x, kRootInv2Pi, x.x < 0.0f ? tail.x : 1.0f - tail.x);
            if (j + 1 < N) d[j + 1] *= fmaf(x.y * density.y, kRootInv2Pi, x.y < 0.0f ? tail.y : 1.0f - tail.y);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) d[j] *= slope_as<kAct>(z[j]);
    }
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
