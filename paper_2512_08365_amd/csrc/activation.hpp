// activation.hpp -- the block's activations and their slopes, in fp32.
#pragma once

#include "block.hpp"

namespace mag {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float GELU_2K = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float GELU_C = 0.044715f;

// 1 / (1 + 2^y), the logistic function of -y ln 2 (the hardware's exponential
// and reciprocal, off by a unit of the last place each; 1 / inf = 0)
__device__ __forceinline__ float logistic2(float y)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y));
}
__device__ __forceinline__ float logistic(float z) { return logistic2(-LOG2E * z); }
// of 2 sqrt(2/pi) (z + 0.044715 z^3)
__device__ __forceinline__ float gelu_logistic(float z)
{
    return logistic2(z * fmaf(-LOG2E * GELU_2K * GELU_C * z, z, -LOG2E * GELU_2K));
}

// The normal distribution's Phi(z) and, times sqrt(2 pi), its density: Abramowitz
// and Stegun's formula 7.1.26 for the error function (off by 1.5e-7 at most), as
// the tail below 0, so that small tails keep their size.
__device__ __forceinline__ float normal(float z, float& density)
{
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    density = __expf(-0.5f * z * z);
    float q = fmaf(1.061405429f, t, -1.453152027f);
    q = fmaf(q, t, 1.421413741f);
    q = fmaf(q, t, -0.284496736f);
    q = fmaf(q, t, 0.254829592f);
    const float tail = 0.5f * q * t * density;
    return z > 0.0f ? 1.0f - tail : tail;
}

// one activation or slope of N values: the kind is looked at once
template <int N, class F>
__device__ __forceinline__ void each(float* z, F f)
{
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = f(z[i]);
}

template <int N>
__device__ __forceinline__ void activate(float* z, int act)
{
    switch (act) {
    case MAG_ACT_RELU: return each<N>(z, [](float v) { return v > 0.0f ? v : (v != v ? v : 0.0f); });
    case MAG_ACT_GELU:
        return each<N>(z, [](float v) {
            float density;
            return v * normal(v, density);
        });
    case MAG_ACT_GELU_TANH:
        return each<N>(z, [](float v) { return v * gelu_logistic(v); });
    case MAG_ACT_SILU: return each<N>(z, [](float v) { return v * logistic(v); });
    default: return;
    }
}

// z -> the activation's slope at z
template <int N>
__device__ __forceinline__ void slopes(float* z, int act)
{
    switch (act) {
    case MAG_ACT_RELU: return each<N>(z, [](float v) { return v > 0.0f ? 1.0f : 0.0f; });
    case MAG_ACT_GELU:
        return each<N>(z, [](float v) {
            float density;
            const float phi = normal(v, density);
            return fmaf(v * density, 0.39894228040143268f, phi);
        });
    case MAG_ACT_GELU_TANH:
        return each<N>(z, [](float v) {
            // (s (1 - s) is zero from 16 on, and v v, which would pass the range, counts no more)
            const float s = gelu_logistic(v), u = __builtin_amdgcn_fmed3f(v, -16.0f, 16.0f);
            return s + u * s * (1.0f - s) * GELU_2K * (1.0f + 3.0f * GELU_C * u * u);
        });
    case MAG_ACT_SILU:
        return each<N>(z, [](float v) {
            const float s = logistic(v);
            return s + v * s * (1.0f - s);
        });
    default: return each<N>(z, [](float) { return 1.0f; });
    }
}

}  // namespace mag
