// norm.hip -- layer norm, forward and backward.

#include "block.hpp"

namespace mag {
namespace {

__device__ float block_sum(float v, float* lds)
{
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

template <class T, class W>
__global__ __launch_bounds__(256) void k_norm(NormParams p)
{
    __shared__ float lds[4];
    const int64_t i = blockIdx.x;
    const T* x = static_cast<const T*>(p.x) + i * p.x_rs;
    float s = 0.0f;
    for (int64_t j = threadIdx.x; j < p.N; j += 256) s += (float)x[j * p.x_cs];
    const float mean = block_sum(s, lds) / (float)p.N;
    s = 0.0f;
    for (int64_t j = threadIdx.x; j < p.N; j += 256) {
        const float d = (float)x[j * p.x_cs] - mean;
        s = fmaf(d, d, s);
    }
    const float rstd = 1.0f / sqrtf(block_sum(s, lds) / (float)p.N + p.eps);
    for (int64_t j = threadIdx.x; j < p.N; j += 256) {
        float y = ((float)x[j * p.x_cs] - mean) * rstd;
        if (p.weight) y *= (float)static_cast<const W*>(p.weight)[j];
        if (p.bias) y += (float)static_cast<const W*>(p.bias)[j];
        static_cast<T*>(p.y)[i * p.y_ld + j] = (T)y;
    }
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[i] = mean;
        if (p.rstd) p.rstd[i] = rstd;
    }
}

template <class T, class W>
__global__ __launch_bounds__(256) void k_norm_weights(NormParams p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.N) return;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t i = 0; i < p.M; ++i) {
        const float d = (float)static_cast<const T*>(p.dy)[i * p.dy_rs + j * p.dy_cs];
        const float xh = ((float)static_cast<const T*>(p.x)[i * p.x_rs + j * p.x_cs] - p.mean[i]) *
                         p.rstd[i];
        sw = fmaf(d, xh, sw);
        sb += d;
    }
    if (p.dweight) static_cast<W*>(p.dweight)[j] = (W)sw;
    if (p.dbias) static_cast<W*>(p.dbias)[j] = (W)sb;
}

template <class T, class W>
__global__ __launch_bounds__(256) void k_norm_dx(NormParams p)
{
    __shared__ float lds[4];
    const int64_t i = blockIdx.x;
    const T* x = static_cast<const T*>(p.x) + i * p.x_rs;
    const T* dy = static_cast<const T*>(p.dy) + i * p.dy_rs;
    const float mean = p.mean[i], rstd = p.rstd[i];
    const W* w = static_cast<const W*>(p.weight);
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < p.N; j += 256) {
        const float h = (float)dy[j * p.dy_cs] * (w ? (float)w[j] : 1.0f);
        s1 += h;
        s2 = fmaf(h, ((float)x[j * p.x_cs] - mean) * rstd, s2);
    }
    s1 = block_sum(s1, lds) / (float)p.N;
    s2 = block_sum(s2, lds) / (float)p.N;
    for (int64_t j = threadIdx.x; j < p.N; j += 256) {
        const float h = (float)dy[j * p.dy_cs] * (w ? (float)w[j] : 1.0f);
        const float xh = ((float)x[j * p.x_cs] - mean) * rstd;
        static_cast<T*>(p.y)[i * p.y_ld + j] = (T)(rstd * (h - s1 - xh * s2));
    }
}

template <class T, class W>
hipError_t forward(const NormParams& p, hipStream_t stream)
{
    hipLaunchKernelGGL((k_norm<T, W>), dim3((unsigned)p.M), dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <class T, class W>
hipError_t backward(const NormParams& p, hipStream_t stream)
{
    if (p.dweight || p.dbias) {
        hipLaunchKernelGGL((k_norm_weights<T, W>), dim3((unsigned)((p.N + 255) / 256)), dim3(256),
                           0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.M > 0 && p.y)
        hipLaunchKernelGGL((k_norm_dx<T, W>), dim3((unsigned)p.M), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormParams& p, int dtype, int weight_dtype, hipStream_t stream)
{
    if (p.M == 0) return hipSuccess;
    const bool wide = weight_dtype == MAG_F32;
    if (dtype == MAG_F32) return forward<float, float>(p, stream);
    if (dtype == MAG_F16)
        return wide ? forward<f16, float>(p, stream) : forward<f16, f16>(p, stream);
    return wide ? forward<bf16, float>(p, stream) : forward<bf16, bf16>(p, stream);
}

hipError_t launch_norm_backward(const NormParams& p, int dtype, int weight_dtype,
                                hipStream_t stream)
{
    const bool wide = weight_dtype == MAG_F32;
    if (dtype == MAG_F32) return backward<float, float>(p, stream);
    if (dtype == MAG_F16)
        return wide ? backward<f16, float>(p, stream) : backward<f16, f16>(p, stream);
    return wide ? backward<bf16, float>(p, stream) : backward<bf16, bf16>(p, stream);
}

}  // namespace mag
