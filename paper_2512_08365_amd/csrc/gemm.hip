// gemm.hip -- products of the feed-forward block's operators.

#include <algorithm>

#include "activation.hpp"
#include "block.hpp"

namespace mag {
namespace {

constexpr int TS = 64, TK = 16;

// One 64 x 64 tile of the output per workgroup of 256 threads, 4 x 4 elements
// each, operands of any strides through LDS in fp32.
template <class T>
__global__ __launch_bounds__(256) void k_product(Product p)
{
    __shared__ float la[TK][TS + 1], lb[TK][TS + 1];
    const int tid = threadIdx.x, ti = tid / 16, tj = tid % 16;
    const int64_t tiles_s = (p.S + TS - 1) / TS, tiles_r = (p.R + TS - 1) / TS;
    const int64_t g = blockIdx.x % (tiles_s * tiles_r), bt = blockIdx.x / (tiles_s * tiles_r);
    const int64_t r0 = g / tiles_s * TS, s0 = g % tiles_s * TS;
    const T* A = static_cast<const T*>(p.a) + bt * p.a_batch;
    const T* B = static_cast<const T*>(p.b) + bt * p.b_batch;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < p.K; k0 += TK) {
        for (int i = tid; i < TS * TK; i += 256) {
            const int kk = i % TK, rr = i / TK;
            const int64_t k = k0 + kk;
            la[kk][rr] = r0 + rr < p.R && k < p.K ? (float)A[(r0 + rr) * p.a_rs + k * p.a_ks] : 0.0f;
            lb[kk][rr] = s0 + rr < p.S && k < p.K ? (float)B[(s0 + rr) * p.b_ss + k * p.b_ks] : 0.0f;
        }
        __syncthreads();
        const int kn = (int)min((int64_t)TK, p.K - k0);
        for (int kk = 0; kk < kn; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(la[kk][ti * 4 + i], lb[kk][tj * 4 + j], acc[i][j]);
        __syncthreads();
    }
    const Epilogue& e = p.e;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + ti * 4 + i, s = s0 + tj * 4 + j;
            if (r >= p.R || s >= p.S) continue;
            float z = e.scale * acc[i][j];
            if (e.mixed) z += e.mix * e.mixed[bt * p.mixed_batch + r * e.mixed_ld + s];
            if (e.bias) z += (float)static_cast<const T*>(e.bias)[s];
            if (e.pre) static_cast<T*>(e.pre)[r * e.pre_ld + s] = (T)z;
            float y = activation(z, e.act);
            if (e.res) y += (float)static_cast<const T*>(e.res)[r * e.res_rs + s * e.res_cs];
            static_cast<T*>(e.y)[bt * p.y_batch + r * e.y_ld + s] = (T)y;
        }
}

template <class T>
__global__ __launch_bounds__(256) void k_slope(SlopeParams p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.N) return;
    float sum = 0.0f;
    for (int64_t i = 0; i < p.M; ++i) {
        float d = (float)static_cast<const T*>(p.dy)[i * p.dy_rs + j * p.dy_cs];
        if (p.act != MAG_ACT_NONE)
            d *= slope((float)static_cast<const T*>(p.pre)[i * p.pre_rs + j * p.pre_cs], p.act);
        sum += d;
        if (p.dz) static_cast<T*>(p.dz)[i * p.ldz + j] = (T)d;
    }
    if (p.dbias) static_cast<T*>(p.dbias)[j] = (T)sum;
}

}  // namespace

hipError_t launch_product(const Product& p, int dtype, hipStream_t stream)
{
    const int64_t tiles = (p.R + TS - 1) / TS * ((p.S + TS - 1) / TS) * p.batch;
    if (tiles == 0) return hipSuccess;
    if (tiles > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)tiles);
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_product<float>, grid, dim3(256), 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_product<f16>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(k_product<bf16>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_slope(const SlopeParams& p, int dtype, hipStream_t stream)
{
    if (p.N == 0) return hipSuccess;
    const dim3 grid((unsigned)((p.N + 255) / 256));
    if (dtype == MAG_F32)
        hipLaunchKernelGGL(k_slope<float>, grid, dim3(256), 0, stream, p);
    else if (dtype == MAG_F16)
        hipLaunchKernelGGL(k_slope<f16>, grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL(k_slope<bf16>, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
