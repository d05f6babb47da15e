// ortho.hip -- the beginning of an orthogonalised update: norms and scaling.

#include <algorithm>

#include "mm.hpp"

namespace mag {
namespace {

// sums of squares of one of a matrix's `chunks` runs of rows, in fp64 (the
// squares of fp32 numbers pass its range); bound by memory and a launch's latency
// (2,048 x 8,192 bfloat16: 10 us, 3.4 TB/s)
template <class T>
__global__ __launch_bounds__(256) void k_orth_norm(OrthParams p)
{
    __shared__ double part[4];
    const int64_t bt = blockIdx.y;
    const T* g = static_cast<const T*>(p.g) + bt * p.g_batch;
    const int64_t per_row = (p.cols + 7) / 8, n = p.rows * per_row;
    const int64_t i0 = n * blockIdx.x / p.chunks, i1 = n * (blockIdx.x + 1) / p.chunks;
    double s = 0.0;
    for (int64_t i = i0 + threadIdx.x; i < i1; i += 256) {
        float v[8];
        const int64_t r = quotient(i, per_row);
        get8(g + r * p.g_rs, p.g_cs, (i - r * per_row) * 8, p.cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
    }
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x == 0)
        p.part[bt * p.chunks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// scale g / (|g| + eps), 8 neighbours of a row a thread; bound by memory (2,048 x
// 8,192 bfloat16: 100 MB in 27 us)
template <class T>
__global__ __launch_bounds__(256) void k_orth_scale(OrthParams p)
{
    typedef __attribute__((ext_vector_type(8))) f16 h8;
    const int64_t bt = blockIdx.y;
    double s = 0.0;
    for (int c = (int)threadIdx.x % 64; c < p.chunks; c += 64) s += p.part[bt * p.chunks + c];
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    const double scale = (double)p.scale / (sqrt(s) + p.eps);
    const T* g = static_cast<const T*>(p.g) + bt * p.g_batch;
    const int64_t per_row = (p.cols + 31) / 32 * 4, n = p.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = quotient(i, per_row), j = (i - r * per_row) * 8;
        h8 hi, lo;
        float x[8];
        get8(g + r * p.g_rs, p.g_cs, j, p.cols, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (0 / 0 of a zero matrix without eps: NaN, as the formula says)
            const float v = j + e < p.cols ? (float)((double)x[e] * scale) : 0.0f;
            f16 h, l;
            two_halves(v, h, l);
            hi[e] = h;
            lo[e] = l;
            if (p.out && j + e < p.cols) static_cast<T*>(p.out)[bt * p.out_batch + r * p.out_ld + j + e] = (T)v;
        }
        if (p.z) {
            f16* z = p.z + bt * p.z_batch + r * p.z_ld + place<2>(j);
            *(h8*)z = hi;
            *(h8*)(z + 32) = lo;
        }
    }
}

template <class T>
hipError_t begin(const OrthParams& p, hipStream_t stream)
{
    hipLaunchKernelGGL(k_orth_norm<T>, dim3((unsigned)p.chunks, (unsigned)p.batch), dim3(256), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t n = p.rows * ((p.cols + 31) / 32 * 4);
    hipLaunchKernelGGL(k_orth_scale<T>,
                       dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096), (unsigned)p.batch),
                       dim3(256), 0, stream, p);
    return hipGetLastError();
}

// The sums of a split product added up: one 64 x 64 block a workgroup (of a
// symmetric product those on and above the diagonal, and their transposes
// through LDS).
__global__ __launch_bounds__(256) void k_orth_join(Mm p)
{
    __shared__ float block[64][65];
    const uint32_t ts = (uint32_t)((p.S + 63) / 64);
    uint32_t bi = blockIdx.x / ts, bj = blockIdx.x % ts;
    if (p.symmetric) tile_above(blockIdx.x, ts, bi, bj);
    const int64_t r0 = (int64_t)bi * 64, s0 = (int64_t)bj * 64, bt = blockIdx.y;
    const bool mirror = p.symmetric && bi != bj;
    const int64_t across = p.o.z ? p.o.z_ld / 2 : p.S;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int64_t r = r0 + i / 8, s = s0 + i % 8 * 8;
        if (r >= p.R || s >= across) continue;
        const int n = (int)max((int64_t)0, min((int64_t)8, p.S - s));
        float v[8] = {};
        if (n > 0)
            add_parts(p.partial + ((int64_t)bt * p.splits * p.R + r) * p.partial_ld + s, p.R * p.partial_ld,
                      p.splits, v);
        if (mirror)
#pragma unroll
            for (int e = 0; e < 8; ++e) block[i / 8][i % 8 * 8 + e] = v[e];
        store_orth(p, bt, r, s, n, v);
    }
    if (!mirror) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int64_t r = s0 + i / 8, s = r0 + i % 8 * 8;
        if (r >= p.S || s >= p.R) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = block[i % 8 * 8 + e][i / 8];
        store_orth(p, bt, r, s, (int)min((int64_t)8, p.R - s), v);
    }
}

}  // namespace

hipError_t launch_orth_join(const Mm& p, hipStream_t stream)
{
    const int64_t tr = (p.R + 63) / 64, ts = (p.S + 63) / 64;
    const dim3 grid((unsigned)(p.symmetric ? tr * (tr + 1) / 2 : tr * ts), (unsigned)p.batch);
    hipLaunchKernelGGL(k_orth_join, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_orth_begin(const OrthParams& p, int dtype, hipStream_t stream)
{
    if (dtype == MAG_F32) return begin<float>(p, stream);
    if (dtype == MAG_F16) return begin<f16>(p, stream);
    return begin<bf16>(p, stream);
}

}  // namespace mag
