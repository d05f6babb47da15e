// block.hpp -- shared definitions of the feed-forward block's operators (linear
// layers, layer norms, orthogonalised updates; not part of the public ABI).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "magneton.h"

namespace mag {

using bf16 = __bf16;
using f16 = _Float16;

// what is stored of a product's sums (Product::acc) for element (r, s)
struct Epilogue {
    float scale;          // z = scale * sum (+ bias[s]) (+ mix * mixed[r][s])
    float mix;
    const float* mixed;
    int64_t mixed_ld;
    const void* bias;     // T, or NULL
    int32_t act;
    const void* res;      // T, or NULL: y = act(z) + res
    int64_t res_rs, res_cs;
    void* pre;            // T, or NULL: z
    int64_t pre_ld;
    void* y;              // T
    int64_t y_ld;
};

// out[r][s] = sum over k of a[r][k] b[s][k], any strides
struct Product {
    const void* a;
    const void* b;
    int64_t R, S, K;
    int64_t a_rs, a_ks, b_ss, b_ks;
    int64_t batch, a_batch, b_batch, y_batch, mixed_batch;
    Epilogue e;
};

// dtype: of a, b, bias, res, pre and y (MAG_F32 ...)
hipError_t launch_product(const Product& p, int dtype, hipStream_t stream);

// dz = dy act'(pre) (T, row stride ldz), and dbias = the column sums of dz
struct SlopeParams {
    const void* dy;
    int64_t dy_rs, dy_cs;
    const void* pre;
    int64_t pre_rs, pre_cs;
    int64_t M, N;
    int32_t act;
    void* dz;        // NULL: not wanted
    int64_t ldz;
    void* dbias;     // NULL: not wanted
};
hipError_t launch_slope(const SlopeParams& p, int dtype, hipStream_t stream);

struct NormParams {
    const void* x;
    int64_t x_rs, x_cs;
    const void* dy;
    int64_t dy_rs, dy_cs;
    void* y;         // y, or dx
    int64_t y_ld;
    int64_t M, N;
    const void* weight;
    const void* bias;
    float* mean;
    float* rstd;
    void* dweight;
    void* dbias;
    float eps;
};
hipError_t launch_norm(const NormParams& p, int dtype, int weight_dtype, hipStream_t stream);
hipError_t launch_norm_backward(const NormParams& p, int dtype, int weight_dtype,
                                hipStream_t stream);

// one update of `batch` matrices seen as m x n, m <= n
struct OrthParams {
    const void* g;
    int64_t g_batch, g_rs, g_cs;
    void* out;
    int64_t out_batch, out_rs, out_cs;
    int64_t batch, m, n;
    double eps;
    float* X;  // [batch][m][n]
};
hipError_t launch_orth_begin(const OrthParams& p, int dtype, hipStream_t stream);
hipError_t launch_orth_end(const OrthParams& p, int dtype, hipStream_t stream);

// the host's error record (api.hip)
int set_error(int code, const char* msg);
int set_hip_error(hipError_t e, const char* where);
void clear_error();

}  // namespace mag
