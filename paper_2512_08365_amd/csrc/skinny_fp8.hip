// skinny_fp8.hip -- 8-bit linear layers of few rows: decode steps.
//
// The weight is read once and bounds the call; everything is one launch.  Each
// workgroup has 16 outputs of every row, its waves share the blocks of the
// reduction and their sums meet in LDS.  The weight is the left operand, straight
// from registers; a wave asks for several blocks before it multiplies the first.
// Rows may lie at any byte.

#include <algorithm>

#include "mm_fp8.hpp"
#include "rows.hpp"

namespace mag {
namespace {

// what a lane has of a block of a row: 16 bytes from 16 (lane / 16) on, and from 64 further on
struct Piece {
    i32x4 lo, hi;
};

__device__ __forceinline__ i32x4 sixteen(const uint8_t* p)
{
    i32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// What is loaded for the bytes from k on at a row's end, its last 16, moved down to its
// place, zeros behind (byte by byte each would be waited for: 29 x 1,021 x 4,099 9.1 us,
// so 6.5 us)
__device__ __forceinline__ i32x4 in_place(i32x4 v, int k, int K)
{
    const int by = k - (K - 16);
    uint32_t w[4];
    __builtin_memcpy(w, &v, 16);
    move_down<1, 4>(w, by <= 0 ? 0 : min(by, 16));
    __builtin_memcpy(&v, w, 16);
    return v;
}

template <int FA, int FB, bool BY_ROW, int MF, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_skinny8(Mm8 p, int32_t half)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int AHEAD = MF == 1 ? 4 : 2;
    __shared__ f32x4 lds[WAVES * MF * 64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int at = lane / 16 * 16;
    const uint8_t* w = p.b + min(n0 + lane % 16, p.S - 1) * p.ldb;
    const uint8_t* x[MF];
    const float* sx[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t m = min((int64_t)f * 16 + lane % 16, p.R - 1);
        x[f] = p.a + m * p.lda;
        sx[f] = p.sa.p + m * p.sa.rs;
    }
    // the scales of the outputs that this lane gets sums of
    const float* sw[BY_ROW ? 4 : 1];
    if constexpr (BY_ROW)
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[e] = p.sb.p + min(n0 + lane / 16 * 4 + e, p.S - 1) * p.sb.rs;
    else
        sw[0] = p.sb.p + n0 / FP8_BLOCK * p.sb.rs;
    f32x4 acc[MF] = {};
    Piece fw[AHEAD], fx[AHEAD][MF];
    float vx[AHEAD][MF], vw[AHEAD][BY_ROW ? 4 : 1];
    auto load = [&](int a, int64_t b) __attribute__((always_inline)) {
        const int k = (int)b * FP8_BLOCK + at, K = (int)p.K;
        // (whole blocks: one address and distances from it)
        if ((int)(b + 1) * FP8_BLOCK <= K) {
            fw[a] = Piece{sixteen(w + k), sixteen(w + k + 64)};
#pragma unroll
            for (int f = 0; f < MF; ++f) fx[a][f] = Piece{sixteen(x[f] + k), sixteen(x[f] + k + 64)};
        } else {
            const int k0 = min(k, K - 16), k1 = min(k + 64, K - 16);
            fw[a] = Piece{sixteen(w + k0), sixteen(w + k1)};
#pragma unroll
            for (int f = 0; f < MF; ++f) fx[a][f] = Piece{sixteen(x[f] + k0), sixteen(x[f] + k1)};
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            vx[a][f] = sx[f][b * p.sa.cs];
        }
#pragma unroll
        for (int e = 0; e < (BY_ROW ? 4 : 1); ++e) vw[a][e] = sw[e][b * p.sb.cs];
    };
    auto whole = [](const Piece& v) { return __builtin_shufflevector(v.lo, v.hi, 0, 1, 2, 3, 4, 5, 6, 7); };
    const int64_t blocks = (p.K + FP8_BLOCK - 1) / FP8_BLOCK;
    for (int64_t b = wave; b < blocks; b += WAVES * AHEAD) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if (b + a * WAVES < blocks) load(a, b + a * WAVES);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int k = (int)(b + a * WAVES) * FP8_BLOCK + at, K = (int)p.K;
            if ((b + a * WAVES + 1) * FP8_BLOCK > K && b + a * WAVES < blocks) {
                fw[a] = Piece{in_place(fw[a].lo, k, K), in_place(fw[a].hi, k + 64, K)};
#pragma unroll
                for (int f = 0; f < MF; ++f)
                    fx[a][f] = Piece{in_place(fx[a][f].lo, k, K), in_place(fx[a][f].hi, k + 64, K)};
            }
            if (b + a * WAVES < blocks)
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    const f32x4 t = mfma8<FB, FA>(whole(fw[a]), whole(fx[a][f]));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[f][e] = fmaf(t[e], vx[a][f] * vw[a][BY_ROW ? e : 0], acc[f][e]);
                }
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f) lds[(wave * MF + f) * 64 + lane] = acc[f];
    __syncthreads();
    for (int i = threadIdx.x; i < MF * 64; i += WAVES * 64) {
        const int f = i / 64, l = i % 64;
        const int64_t m = f * 16 + l % 16, n = n0 + l / 16 * 4;
        if (m >= p.R || n >= p.S) continue;
        f32x4 s = lds[i];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) s += lds[v * MF * 64 + i];
        const Epilogue& e = p.e;
        auto store = [&](auto type) __attribute__((always_inline)) {
            using T = typename decltype(type)::Type;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (n + j >= p.S) break;
                float z = s[j];
                if (e.bias) z += (float)static_cast<const T*>(e.bias)[n + j];
                if (e.pre) static_cast<T*>(e.pre)[m * e.pre_ld + n + j] = (T)z;
                activate<T, 1>(&z, e.act);
                if (e.res) z += (float)static_cast<const T*>(e.res)[m * e.res_rs + (n + j) * e.res_cs];
                static_cast<T*>(e.y)[m * e.y_ld + n + j] = (T)z;
            }
        };
        if (half)
            store(Result<f16>{});
        else
            store(Result<bf16>{});
    }
#endif
}

template <int FA, int FB, bool BY_ROW>
hipError_t launch(const Mm8& p, int dtype, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.S + 15) / 16)), block(512);
    const int32_t half = dtype == MAG_F16;
    if (p.R <= 16)
        hipLaunchKernelGGL((k_skinny8<FA, FB, BY_ROW, 1, 8>), grid, block, 0, stream, p, half);
    else
        hipLaunchKernelGGL((k_skinny8<FA, FB, BY_ROW, 2, 8>), grid, block, 0, stream, p, half);
    return hipGetLastError();
}

template <int FA, int FB>
hipError_t launch(const Mm8& p, int dtype, hipStream_t stream)
{
    return p.by_row ? launch<FA, FB, true>(p, dtype, stream) : launch<FA, FB, false>(p, dtype, stream);
}

}  // namespace

hipError_t launch_skinny8(const Mm8& p, int dtype, hipStream_t stream)
{
    if (p.fa == MAG_E4M3)
        return p.fb == MAG_E4M3 ? launch<MAG_E4M3, MAG_E4M3>(p, dtype, stream)
                                : launch<MAG_E4M3, MAG_E5M2>(p, dtype, stream);
    return p.fb == MAG_E4M3 ? launch<MAG_E5M2, MAG_E4M3>(p, dtype, stream)
                            : launch<MAG_E5M2, MAG_E5M2>(p, dtype, stream);
}

}  // namespace mag
