// activation.hpp -- the block's activations and their slopes, in fp32.
#pragma once

#include "block.hpp"

namespace mag {

constexpr float LN2 = 0.69314718055994531f;
constexpr float LOG2E = 1.4426950408889634f, LOG2E_REST = 1.92596299e-8f;     // the float nearest, what is left
constexpr float GELU_2K = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float GELU_C = 0.044715f, GELU_C_REST = 1.54614448e-9f;
constexpr float GELU_2K_LOG2E = 2.3022081981443252f, GELU_2K_LOG2E_REST = 1.29484024e-8f;

// FINE: for results of fp32.  An argument of an exponential is then held in two
// floats, `rest` what rounding took from y: an error of half its last place would
// otherwise be |y| ln 2 times as large in the result.  Two-byte results round
// a thousand times as much away.

// 2^(y + rest) (the hardware's exponential, off by a unit of the last place)
template <bool FINE>
__device__ __forceinline__ float power2(float y, float rest)
{
    const float e = __builtin_amdgcn_exp2f(y);
    return FINE ? e * (1.0f + (fabsf(y) < 150.0f ? LN2 * rest : 0.0f)) : e;
}

// s = 1 / (1 + 2^y), the logistic function of -y ln 2, and c = 1 - s (the hardware's
// reciprocal, off by a unit of the last place; 1 / inf = 0)
struct Logistic {
    float s, c;
};
template <bool FINE>
__device__ __forceinline__ Logistic logistic2(float y, float rest)
{
    const float e = power2<FINE>(y, rest);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    return {s, FINE && y < 0.0f ? e * s : 1.0f - s};
}
template <bool FINE>
__device__ __forceinline__ Logistic logistic(float z)
{
    const float y = -LOG2E * z;
    return logistic2<FINE>(y, FINE ? fmaf(-LOG2E, z, -y) - LOG2E_REST * z : 0.0f);
}
// of 2 sqrt(2/pi) (z + 0.044715 z^3)
template <bool FINE>
__device__ __forceinline__ Logistic gelu_logistic(float z)
{
#pragma clang fp contract(off)   // (w - b below is of the rounded product)
    if constexpr (!FINE)
        return logistic2<false>(z * fmaf(-GELU_2K_LOG2E * GELU_C * z, z, -GELU_2K_LOG2E), 0.0f);
    const float s = z * z, s_rest = fmaf(z, z, -s);
    const float w = GELU_C * s, w_rest = fmaf(GELU_C, s, -w) + fmaf(GELU_C, s_rest, GELU_C_REST * s);
    const float q = 1.0f + w, b = q - 1.0f, q_rest = (1.0f - (q - b)) + (w - b) + w_rest;
    const float m = -GELU_2K_LOG2E * z, m_rest = fmaf(-GELU_2K_LOG2E, z, -m) - GELU_2K_LOG2E_REST * z;
    const float y = m * q;
    return logistic2<true>(y, fmaf(m, q, -y) + fmaf(m, q_rest, m_rest * q));
}

// The normal distribution's Phi(z) and, times sqrt(2 pi), its density.  The tail
// below 0 is the density times a polynomial in t = 1 / (1 + p |z|) without a
// constant term, fitted to the smallest relative error down to where fp32 ends:
// 1.2e-8 by nine terms, 4.2e-6 by six (a two-byte result's rounding is a hundred
// times that).  So small tails keep their digits.
template <bool FINE>
__device__ __forceinline__ float normal(float z, float& density)
{
    const float x = FINE ? __builtin_amdgcn_fmed3f(z, -20.0f, 20.0f) : z;   // (its square's rest is finite)
    const float s = x * x, y = -0.5f * LOG2E * s;
    density = power2<FINE>(y, FINE ? fmaf(-0.5f * LOG2E, s, -y) -
                                         fmaf(0.5f * LOG2E_REST, s, 0.5f * LOG2E * fmaf(x, x, -s))
                                   : 0.0f);
    const float t = __builtin_amdgcn_rcpf(fmaf(FINE ? 0.265165031f : 0.307591438f, fabsf(z), 1.0f));
    float q;
    if constexpr (FINE) {
        q = fmaf(0.030769188f, t, -0.143664613f);
        q = fmaf(q, t, 0.216198519f);
        q = fmaf(q, t, -0.114705838f);
        q = fmaf(q, t, 0.136861816f);
        q = fmaf(q, t, 0.0607526787f);
        q = fmaf(q, t, 0.102656692f);
        q = fmaf(q, t, 0.105324827f);
        q = fmaf(q, t, 0.105806731f);
    } else {
        q = fmaf(-0.0754296258f, t, 0.190648258f);
        q = fmaf(q, t, 0.00642877724f);
        q = fmaf(q, t, 0.136722073f);
        q = fmaf(q, t, 0.118667327f);
        q = fmaf(q, t, 0.122962758f);
    }
    const float tail = q * t * density;
    return z > 0.0f ? 1.0f - tail : tail;
}

// one activation or slope of N values: the kind is looked at once
template <int N, class F>
__device__ __forceinline__ void each(float* z, F f)
{
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = f(z[i]);
}

// z -> the activation of z, for results of type T
template <class T, int N>
__device__ __forceinline__ void activate(float* z, int act)
{
    constexpr bool FINE = sizeof(T) == 4;
    switch (act) {
    case MAG_ACT_RELU: return each<N>(z, [](float v) { return v > 0.0f ? v : (v != v ? v : 0.0f); });
    case MAG_ACT_GELU:
        return each<N>(z, [](float v) {
            float density;
            return v * normal<FINE>(v, density);
        });
    case MAG_ACT_GELU_TANH:
        return each<N>(z, [](float v) { return v * gelu_logistic<FINE>(v).s; });
    case MAG_ACT_SILU: return each<N>(z, [](float v) { return v * logistic<FINE>(v).s; });
    default: return;
    }
}

// z -> the activation's slope at z
template <class T, int N>
__device__ __forceinline__ void slopes(float* z, int act)
{
    constexpr bool FINE = sizeof(T) == 4;
    switch (act) {
    case MAG_ACT_RELU: return each<N>(z, [](float v) { return v > 0.0f ? 1.0f : 0.0f; });
    case MAG_ACT_GELU:
        return each<N>(z, [](float v) {
            float density;
            const float phi = normal<FINE>(v, density);
            return fmaf(v * density, 0.39894228040143268f, phi);
        });
    case MAG_ACT_GELU_TANH:
        return each<N>(z, [](float v) {
            // (s c is zero from 16 on, and v v, which would pass the range, counts no more)
            const Logistic l = gelu_logistic<FINE>(v);
            const float u = __builtin_amdgcn_fmed3f(v, -16.0f, 16.0f);
            return l.s + u * l.s * l.c * GELU_2K * (1.0f + 3.0f * GELU_C * u * u);
        });
    case MAG_ACT_SILU:
        return each<N>(z, [](float v) {
            const Logistic l = logistic<FINE>(v);
            return l.s + v * l.s * l.c;
        });
    default: return each<N>(z, [](float) { return 1.0f; });
    }
}

}  // namespace mag
