// ortho.hip -- the ends of the orthogonalised update: norm, scaling, result.

#include "block.hpp"

namespace mag {
namespace {

template <class T>
__global__ __launch_bounds__(1024) void k_orth_begin(OrthParams p)
{
    __shared__ double part[16];
    const int64_t bt = blockIdx.x, n = p.m * p.n;
    const T* g = static_cast<const T*>(p.g) + bt * p.g_batch;
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) {
        const double v = (double)(float)g[i / p.n * p.g_rs + i % p.n * p.g_cs];
        s += v * v;
    }
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += part[w];
    const double scale = 1.0 / (sqrt(s) + p.eps);
    for (int64_t i = threadIdx.x; i < n; i += 1024)
        p.X[bt * n + i] = (float)((double)(float)g[i / p.n * p.g_rs + i % p.n * p.g_cs] * scale);
}

template <class T>
__global__ __launch_bounds__(256) void k_orth_end(OrthParams p)
{
    const int64_t n = p.m * p.n;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * p.batch;
         i += (int64_t)gridDim.x * 256) {
        const int64_t bt = i / n, e = i % n;
        static_cast<T*>(p.out)[bt * p.out_batch + e / p.n * p.out_rs + e % p.n * p.out_cs] =
            (T)p.X[i];
    }
}

}  // namespace

hipError_t launch_orth_begin(const OrthParams& p, int dtype, hipStream_t stream)
{
    const dim3 grid((unsigned)p.batch);
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_orth_begin<float>, grid, dim3(1024), 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_orth_begin<f16>, grid, dim3(1024), 0, stream, p);
    else
        hipLaunchKernelGGL(k_orth_begin<bf16>, grid, dim3(1024), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_orth_end(const OrthParams& p, int dtype, hipStream_t stream)
{
    const dim3 grid(2048);
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_orth_end<float>, grid, dim3(256), 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_orth_end<f16>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(k_orth_end<bf16>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
