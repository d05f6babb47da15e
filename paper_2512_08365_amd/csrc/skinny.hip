// skinny.hip -- linear layers of few rows: decode steps.
//
// The weight is read once and bounds the call; everything is one launch, since a
// second one would cost as much as a small weight.  Each workgroup has 16 or 32
// outputs of every row and its waves share the reduction, so that a 4096 x 4096
// weight is read by 2,048 waves, each with half of its loads in flight at once (two
// rounds of four lines); their sums meet in LDS.  The products run on the matrix cores with the weight as the left
// operand, straight from registers where it lies along the reduction, and
// through a transposing LDS read where it is stored input by output.  Rows of
// any alignment: vector loads at any element.  fp32 takes the fp32 matrix
// instruction, whose rate (a sixteenth of bfloat16's) a few rows do not reach.
//
// One row by 4096 x 4096 bfloat16: 9.1 us (3.7 TB/s), by 4096 x 16,384 24 us (5.5);
// 29 rows by 1,021 x 4,099 half stored input by output 8.7 us.  Rows that start
// off a multiple of 4 bytes take up to twice as long (one row by 4,407 x 85: 14.5
// us, by 4096 x 80: 7.5 us).

#include <algorithm>

#include "mm.hpp"

namespace mag {
namespace {

// What a lane has of a fragment: 16 bytes, of row lane % 16 from k = KL (lane / 16)
// on; KL = 8 or, of fp32, 4 elements
template <class T>
struct Frag {
    static constexpr int KL = 16 / (int)sizeof(T), STEP = 4 * KL;
    T v[KL];
};

template <class T>
__device__ __forceinline__ void multiply(const Frag<T>& a, const Frag<T>& b, f32x4& c)
{
    if constexpr (sizeof(T) == 4) {
        // (four k of the 16 a step has, whichever: both operands alike)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
    } else {
        s16x8 x, y;
        __builtin_memcpy(&x, a.v, 16);
        __builtin_memcpy(&y, b.v, 16);
        c = mfma<T>(x, y, c);
    }
}

// elements k .. k + KL - 1 of a row of K neighbours (zeros behind)
template <class T>
__device__ __forceinline__ Frag<T> fetch(const T* row, int64_t k, int64_t K)
{
    Frag<T> f;
    if (k + Frag<T>::KL <= K) {
        __builtin_memcpy(f.v, row + k, 16);
    } else {
#pragma unroll
        for (int i = 0; i < Frag<T>::KL; ++i) f.v[i] = k + i < K ? row[k + i] : (T)0.0f;
    }
    return f;
}

// fragments that end inside the row
template <class T>
__device__ __forceinline__ Frag<T> fetch_inside(const T* row, int64_t k)
{
    Frag<T> f;
    __builtin_memcpy(f.v, row + k, 16);
    return f;
}

// any fragments: their elements asked for before any is looked at
template <class T>
__device__ __forceinline__ Frag<T> fetch_last(const T* row, int64_t k, int64_t K)
{
    Frag<T> f;
#pragma unroll
    for (int i = 0; i < Frag<T>::KL; ++i) f.v[i] = row[min(k + i, K - 1)];
#pragma unroll
    for (int i = 0; i < Frag<T>::KL; ++i) f.v[i] = k + i < K ? f.v[i] : (T)0.0f;
    return f;
}

// the sums of the waves added up and stored: G x 16 outputs of MF x 16 rows
template <class T, int G, int MF, int WAVES>
__device__ __forceinline__ void finish(const SkinnyParams& p, f32x4 (&acc)[G][MF], f32x4* lds, int64_t n0)
{
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int f = 0; f < MF; ++f) lds[(wave * G * MF + g * MF + f) * 64 + lane] = acc[g][f];
    __syncthreads();
    for (int i = threadIdx.x; i < G * MF * 64; i += WAVES * 64) {
        const int g = i / 64 / MF, f = i / 64 % MF, l = i % 64;
        const int64_t m = f * 16 + l % 16, n = n0 + g * 16 + l / 16 * 4;
        if (m >= p.M || n >= p.N) continue;
        f32x4 s = lds[i];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += lds[w * G * MF * 64 + i];
        const Epilogue& e = p.e;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (n + j >= p.N) break;
            float z = s[j];
            if (e.bias) z += (float)static_cast<const T*>(e.bias)[n + j];
            if (e.pre) static_cast<T*>(e.pre)[m * e.pre_ld + n + j] = (T)z;
            activate<T, 1>(&z, e.act);
            if (e.res) z += (float)static_cast<const T*>(e.res)[m * e.res_rs + (n + j) * e.res_cs];
            static_cast<T*>(e.y)[m * e.y_ld + n + j] = (T)z;
        }
    }
}

// The weight along the reduction: element (n, k) at n * w_ld + k.  The waves take
// pieces of two steps (a 128-byte line of each row) in turn, AHEAD pieces at once.
template <class T, int G, int MF, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_skinny_along(SkinnyParams p)
{
    constexpr int STEP = Frag<T>::STEP, PIECE = 2 * STEP, AHEAD = G * MF == 1 ? 4 : 2;
    __shared__ f32x4 lds[WAVES * G * MF * 64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * G);
    const int64_t kl = lane / 16 * Frag<T>::KL;
    const T *w[G], *x[MF];
#pragma unroll
    for (int g = 0; g < G; ++g)
        w[g] = static_cast<const T*>(p.w) + min(n0 + g * 16 + lane % 16, p.N - 1) * p.w_ld;
#pragma unroll
    for (int f = 0; f < MF; ++f)
        x[f] = static_cast<const T*>(p.x) + min((int64_t)f * 16 + lane % 16, p.M - 1) * p.x_ld;
    f32x4 acc[G][MF] = {};
    Frag<T> fw[AHEAD][2][G], fx[AHEAD][2][MF];
    auto load = [&](int a, int64_t k0, auto get) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int g = 0; g < G; ++g) fw[a][s][g] = get(w[g], k0 + s * STEP + kl);
#pragma unroll
            for (int f = 0; f < MF; ++f) fx[a][s][f] = get(x[f], k0 + s * STEP + kl);
        }
    };
    auto add = [&](int a) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int f = 0; f < MF; ++f) multiply(fw[a][s][g], fx[a][s][f], acc[g][f]);
    };
    // the whole pieces (which ones a wave has is the same for all of its lanes) ...
    const int whole = (int)(p.K / PIECE);
    for (int i = wave; i < whole; i += WAVES * AHEAD) {
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if (i + a * WAVES < whole)
                load(a, (int64_t)(i + a * WAVES) * PIECE, [](const T* row, int64_t k) { return fetch_inside(row, k); });
            else
                load(a, 0, [](const T*, int64_t) { return Frag<T>{}; });
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) add(a);
    }
    // ... and what is left, whose turn it is
    if (p.K % PIECE && wave == whole % WAVES) {
        load(0, (int64_t)whole * PIECE, [&](const T* row, int64_t k) { return fetch_last(row, k, p.K); });
        add(0);
    }
    finish<T, G, MF, WAVES>(p, acc, lds, n0);
}

// The weight input by output: element (n, k) at k * w_ld + n.  A wave loads a step
// of 32 outputs into LDS of its own (rows padded against bank conflicts) and
// reads it transposed.
template <class T, int MF, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_skinny_across(SkinnyParams p)
{
    constexpr int G = 2, STEP = Frag<T>::STEP, KL = Frag<T>::KL;
    constexpr int ROW = 32 * sizeof(T) + (sizeof(T) == 2 ? 16 : 32);  // bytes
    constexpr int LOADS = STEP * 32 / KL / 64, PER_ROW = 32 / KL;     // 16-byte pieces
    constexpr int TILE = STEP * ROW;
    constexpr int SUMS = WAVES * G * MF * 64 * 16;
    __shared__ __attribute__((aligned(16))) char lds[SUMS > WAVES * TILE ? SUMS : WAVES * TILE];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;
    char* mine = lds + wave * TILE;
    const int64_t n0 = (int64_t)blockIdx.x * 32;
    const T* w = static_cast<const T*>(p.w);
    const T* x[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
        x[f] = static_cast<const T*>(p.x) + min((int64_t)f * 16 + lane % 16, p.M - 1) * p.x_ld;
    f32x4 acc[G][MF] = {};
    Frag<T> fw[LOADS], fx[MF];
    auto load = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int c = i * 64 + lane;
            const int64_t k = k0 + c / PER_ROW, n = n0 + c % PER_ROW * KL;
            fw[i] = k < p.K ? fetch(w + k * p.w_ld, n, p.N) : Frag<T>{};
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) fx[f] = fetch(x[f], k0 + lane / 16 * KL, p.K);
    };
    load((int64_t)wave * STEP);
    for (int64_t k0 = (int64_t)wave * STEP; k0 < p.K; k0 += (int64_t)WAVES * STEP) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int c = i * 64 + lane;
            s16x8 v;
            __builtin_memcpy(&v, fw[i].v, 16);
            *(s16x8*)(mine + c / PER_ROW * ROW + c % PER_ROW * 16) = v;
        }
        Frag<T> now[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) now[f] = fx[f];
        load(k0 + (int64_t)WAVES * STEP);  // (behind the end: zeros)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            Frag<T> a;
            if constexpr (sizeof(T) == 2) {
                const int q = lane % 16, k = lane / 16 * 8 + q / 4;
                const char* at = mine + k * ROW + g * 32 + q % 4 * 8;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(at + 4 * ROW));
                __builtin_memcpy(a.v, &lo, 8);
                __builtin_memcpy(a.v + 4, &hi, 8);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    a.v[i] = *(const T*)(mine + (lane / 16 * 4 + i) * ROW + (g * 16 + lane % 16) * 4);
            }
#pragma unroll
            for (int f = 0; f < MF; ++f) multiply(a, now[f], acc[g][f]);
        }
    }
    __syncthreads();
    finish<T, G, MF, WAVES>(p, acc, reinterpret_cast<f32x4*>(lds), n0);
}

template <class T, int MF>
hipError_t launch(const SkinnyParams& p, hipStream_t stream)
{
    if (p.across) {
        const dim3 grid((unsigned)((p.N + 31) / 32));
        // (few outputs: more waves share the reduction)
        if (grid.x < 128 && p.K > 1024)
            hipLaunchKernelGGL((k_skinny_across<T, MF, 16>), grid, dim3(1024), 0, stream, p);
        else
            hipLaunchKernelGGL((k_skinny_across<T, MF, 8>), grid, dim3(512), 0, stream, p);
        return hipGetLastError();
    }
    // Two groups of outputs where that leaves enough workgroups: the rows' own
    // fragments, which come from L2, are then used twice (4096 inputs: 32 rows by
    // 8,192 outputs 20 us, one group 25 us; by 4,096 18 and 14 us; 16 rows by 16,384
    // 32 and 35 us).  Of few rows these are nearly the same lines for all lanes (1
    // row by 16,384: 33 and 24 us).
    const bool two = MF == 2 ? p.N >= 8192 : p.M > 8 && p.N >= 16384;
    const dim3 grid((unsigned)((p.N + (two ? 31 : 15)) / (two ? 32 : 16)));
    if (two)
        hipLaunchKernelGGL((k_skinny_along<T, 2, MF, 8>), grid, dim3(512), 0, stream, p);
    else if (grid.x < 128 && p.K > 1024)
        hipLaunchKernelGGL((k_skinny_along<T, 1, MF, 16>), grid, dim3(1024), 0, stream, p);
    else
        hipLaunchKernelGGL((k_skinny_along<T, 1, MF, 8>), grid, dim3(512), 0, stream, p);
    return hipGetLastError();
}

template <class T>
hipError_t launch_rows(const SkinnyParams& p, hipStream_t stream)
{
    return p.M <= 16 ? launch<T, 1>(p, stream) : launch<T, 2>(p, stream);
}

}  // namespace

hipError_t launch_skinny(const SkinnyParams& p, int dtype, hipStream_t stream)
{
    if (dtype == MAG_F32) return launch_rows<float>(p, stream);
    if (dtype == MAG_F16) return launch_rows<f16>(p, stream);
    return launch_rows<bf16>(p, stream);
}

}  // namespace mag
