// gemm.hip -- what surrounds the products of the feed-forward block: operands
// laid out for them, the gradient through the activation, split sums joined.

#include <algorithm>

#include "mm.hpp"

namespace mag {
namespace {

typedef __attribute__((ext_vector_type(8))) short h8;

__device__ __forceinline__ short bits(bf16 v) { return __builtin_bit_cast(short, v); }

// An fp32 number as three bfloat16 parts that add up to it exactly: 8 bits of
// it, 8 of the rest, what is left.  Rounding to nearest keeps every part's
// remainder small; the largest numbers, which it would take to infinity, are
// cut instead.  Infinities and NaN have the first part alone.
__device__ __forceinline__ void three_parts(float v, short& a, short& b, short& c)
{
    bf16 h = (bf16)v;
    if (!(fabsf(v) < __builtin_inff())) {
        a = bits(h);
        b = c = 0;
        return;
    }
    if (!(fabsf((float)h) < __builtin_inff()))
        h = __builtin_bit_cast(bf16, (short)(__builtin_bit_cast(uint32_t, v) >> 16));
    const float r = v - (float)h;
    const bf16 m = (bf16)r;
    a = bits(h);
    b = bits(m);
    c = bits((bf16)(r - (float)m));
}

// eight neighbours of a row, from element j of it, into an operand's row
template <class T>
__device__ __forceinline__ void put8(const float* v, short* row, int64_t j)
{
    h8 o;
    if constexpr (sizeof(T) == 4) {
        h8 m, l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            short a, b, c;
            three_parts(v[i], a, b, c);
            o[i] = a;
            m[i] = b;
            l[i] = c;
        }
        short* d = row + place<3>(j);
        *(h8*)d = o;
        *(h8*)(d + 32) = m;
        *(h8*)(d + 64) = l;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = __builtin_bit_cast(short, (T)v[i]);
        *(h8*)(row + j) = o;
    }
}

// elements of an operand's row of n, without the parts
template <class T>
__host__ __device__ int64_t width_of(int64_t n)
{
    return sizeof(T) == 4 ? (n + 31) / 32 * 32 : (n + 7) / 8 * 8;
}

// Bandwidth bound: each thread moves 8 neighbours of a row.
template <class T>
__global__ __launch_bounds__(256) void k_pack(PackParams p)
{
    const int64_t per_row = width_of<T>(p.cols) / 8, n = p.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per_row, j = i % per_row * 8;
        float v[8];
        get8(static_cast<const T*>(p.src) + r * p.rs, p.cs, j, p.cols, v);
        put8<T>(v, static_cast<short*>(p.dst) + r * p.ld, j);
    }
}

constexpr int SLOPE_COLS = 512;  // columns of a workgroup: 64 lanes of 8

// dz and the column sums of one chunk of rows: four waves take its rows in
// turn, 8 columns a lane, and add their sums up in LDS at the end.
template <class T>
__global__ __launch_bounds__(256) void k_slope(SlopeParams p, int64_t chunk)
{
    __shared__ float sums[4][SLOPE_COLS + 4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t j = (int64_t)blockIdx.x * SLOPE_COLS + lane * 8;
    const int64_t i0 = (int64_t)blockIdx.y * chunk, i1 = min(i0 + chunk, p.M);
    float sum[8] = {};
    if (j < width_of<T>(p.N))
        for (int64_t i = i0 + wave; i < i1; i += 4) {
            float d[8];
            get8(static_cast<const T*>(p.dy) + i * p.dy_rs, p.dy_cs, j, p.N, d);
            if (p.act != MAG_ACT_NONE) {
                float z[8];
                get8(static_cast<const T*>(p.pre) + i * p.pre_rs, p.pre_cs, j, p.N, z);
                slopes<8>(z, p.act);
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] *= z[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += d[e];
            if (p.dz) put8<T>(d, static_cast<short*>(p.dz) + i * p.ldz, j);
        }
    if (!p.dbias) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][lane * 8 + e] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < SLOPE_COLS; c += 256) {
        const int64_t col = (int64_t)blockIdx.x * SLOPE_COLS + c;
        if (col < p.N)
            p.part[(int64_t)blockIdx.y * p.N + col] =
                (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
    }
}

// column sums of the chunks' sums: 4 waves a workgroup of 64 columns
template <class T>
__global__ __launch_bounds__(256) void k_column_sums(const float* part, int64_t chunks, int64_t N,
                                                     T* out)
{
    __shared__ float sums[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t j = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (j < N)
        for (int64_t c = wave; c < chunks; c += 4) s += part[c * N + j];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && j < N) out[j] = (T)((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

template <class TO>
__global__ __launch_bounds__(256) void k_mm_join(Mm p)
{
    const int64_t per_row = p.partial_ld / 8, n = p.R * per_row;
    const int64_t plane = p.R * p.partial_ld;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per_row, s = i % per_row * 8;
        const float* q = p.partial + r * p.partial_ld + s;
        float v[8], w[8];
        load8(q, v);
        for (int k = 1; k < p.splits; ++k) {
            load8(q + k * plane, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
        const int m = (int)min((int64_t)8, p.S - s);
        if constexpr (sizeof(TO) == 4)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < m && !(fabsf(v[e]) < __builtin_inff())) v[e] = whole_sum(p, 0, r, s + e);
        store_linear<TO>(p.e, r, s, m, v);
    }
}

unsigned blocks_for(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16); }

}  // namespace

hipError_t launch_pack(const PackParams& p, int dtype, hipStream_t stream)
{
    const int64_t n = p.rows * ((p.cols + 7) / 8);
    if (n == 0) return hipSuccess;
    const dim3 grid(blocks_for(n)), block(256);
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_pack<float>, grid, block, 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_pack<f16>, grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL(k_pack<bf16>, grid, block, 0, stream, p);
    return hipGetLastError();
}

// chunks of rows of the column sums: enough workgroups to fill the device
int64_t slope_chunks(int64_t M, int64_t N)
{
    const int64_t across = (N + SLOPE_COLS - 1) / SLOPE_COLS;
    const int64_t want = std::max<int64_t>(1, 2048 / std::max<int64_t>(across, 1));
    return std::max<int64_t>(1, std::min<int64_t>(want, (M + 15) / 16));
}

hipError_t launch_slope(const SlopeParams& p, int dtype, hipStream_t stream)
{
    if (p.N == 0) return hipSuccess;
    const int64_t chunks = slope_chunks(p.M, p.N), chunk = (p.M + chunks - 1) / chunks;
    const dim3 grid((unsigned)((p.N + SLOPE_COLS - 1) / SLOPE_COLS), (unsigned)chunks), block(256);
    const dim3 sums((unsigned)((p.N + 63) / 64));
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_slope<float>, grid, block, 0, stream, p, chunk);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_slope<f16>, grid, block, 0, stream, p, chunk);
    else
        hipLaunchKernelGGL(k_slope<bf16>, grid, block, 0, stream, p, chunk);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.dbias) return e;
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_column_sums<float>, sums, block, 0, stream, p.part, chunks, p.N,
                           static_cast<float*>(p.dbias));
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_column_sums<f16>, sums, block, 0, stream, p.part, chunks, p.N,
                           static_cast<f16*>(p.dbias));
    else
        hipLaunchKernelGGL(k_column_sums<bf16>, sums, block, 0, stream, p.part, chunks, p.N,
                           static_cast<bf16*>(p.dbias));
    return hipGetLastError();
}

hipError_t launch_mm_join(const Mm& p, int dtype, hipStream_t stream)
{
    const dim3 grid(blocks_for(p.R * (p.partial_ld / 8))), block(256);
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_mm_join<float>, grid, block, 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_mm_join<f16>, grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL(k_mm_join<bf16>, grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
