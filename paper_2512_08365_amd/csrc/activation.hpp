// activation.hpp -- the block's activations and their slopes, in fp32.
#pragma once

#include "block.hpp"

namespace mag {

__device__ __forceinline__ float logistic(float z) { return 1.0f / (1.0f + __expf(-z)); }

constexpr float GELU_2K = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float GELU_C = 0.044715f;

__device__ __forceinline__ float activation(float z, int act)
{
    switch (act) {
    case MAG_ACT_RELU: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case MAG_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case MAG_ACT_GELU_TANH: return z * logistic(GELU_2K * (z + GELU_C * z * z * z));
    case MAG_ACT_SILU: return z * logistic(z);
    default: return z;
    }
}

__device__ __forceinline__ float slope(float z, int act)
{
    switch (act) {
    case MAG_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case MAG_ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) +
               z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    case MAG_ACT_GELU_TANH: {
        const float s = logistic(GELU_2K * (z + GELU_C * z * z * z));
        return s + z * s * (1.0f - s) * GELU_2K * (1.0f + 3.0f * GELU_C * z * z);
    }
    case MAG_ACT_SILU: {
        const float s = logistic(z);
        return s + z * s * (1.0f - s);
    }
    default: return 1.0f;
    }
}

}  // namespace mag
