// Activations of rcd_linear and their derivatives, in fp32.
#pragma once

#include "rcd_elem.cuh"

namespace rcd {

#ifdef __CUDACC__
constexpr float kRootHalf = 0.70710678118654752f, kRootInv2Pi = 0.39894228040143268f, kTanhScale = 0.79788456080286536f, kTanhCube = 0.044715f;

__device__ __forceinline__ float activate(float z, int act)
{
    switch (act) {
    case RCD_ACT_RELU: return z > 0.0f ? z : z == z ? 0.0f : z;      // (a NaN stays one)
    case RCD_ACT_GELU: return 0.5f * z * (1.0f + erff(z * kRootHalf));
    case RCD_ACT_GELU_TANH: return 0.5f * z * (1.0f + tanhf(kTanhScale * (z + kTanhCube * z * z * z)));
    case RCD_ACT_SILU: return z / (1.0f + __expf(-z));               // (-z so large that the exponential is infinite: 0)
    default: return z;
    }
}
__device__ __forceinline__ float activation_slope(float z, int act)
{
    switch (act) {
    case RCD_ACT_RELU: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    case RCD_ACT_GELU: return 0.5f * (1.0f + erff(z * kRootHalf)) + z * __expf(-0.5f * z * z) * kRootInv2Pi;
    case RCD_ACT_GELU_TANH: {
        const float t = tanhf(kTanhScale * (z + kTanhCube * z * z * z));
        return 0.5f * (1.0f + t) + 0.5f * z * (1.0f - t * t) * kTanhScale * (1.0f + 3.0f * kTanhCube * z * z);
    }
    case RCD_ACT_SILU: {
        const float s = 1.0f / (1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    default: return 1.0f;
    }
}
#endif

}  // namespace rcd
