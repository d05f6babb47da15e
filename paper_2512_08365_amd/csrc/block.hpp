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

// An operand of a product: element (row, k) at row * ld + k, or with mc at k *
// ld + row (data and rows at multiples of 16 bytes, and the run that is
// contiguous a multiple of 16 bytes or zero-padded to one).  In P = 2 or
// 3 parts, that run has 32 elements' first parts, then their second ones, and so
// on, zero-padded to whole 32s, and ld counts all of them.
struct MmOperand {
    const void* p;
    int64_t ld;
    int64_t batch;  // elements from one matrix of a batch to the next
    int32_t mc;
};

// z = sum + bias, pre = z, y = act(z) + res
struct Epilogue {
    const void* bias;     // or NULL
    const void* res;      // or NULL
    int64_t res_rs, res_cs;
    void* pre;            // or NULL
    int64_t pre_ld;
    void* y;
    int64_t y_ld;
    int32_t act;
    int32_t vec;          // neighbours of a row are neighbours in memory everywhere
};

// z = scale sum + mix M + diagonal I, as two halves or, for the result, one number
struct OrthStore {
    float scale, mix, diagonal;
    const f16* m;         // or NULL: two parts, as an operand's
    int64_t m_ld, m_batch;
    f16* z;               // two parts, as an operand's, or NULL
    int64_t z_ld, z_batch;
    void* out;            // the result (z NULL)
    int64_t out_ld, out_batch;
    int32_t dtype;        // of out
};

// out[r][s] = sum over k of a(r, k) b(s, k)
struct Mm {
    MmOperand a, b;
    int64_t R, S, K;
    int32_t batch;
    int32_t splits;       // of the reduction, each with its own sums in `partial`
    int32_t in_parts;     // fp32 operands in three parts: sums that are not finite are retaken
    int32_t symmetric;    // tiles on and above the diagonal only, mirrored (R = S)
    float* partial;       // [batch][splits][R][partial_ld]
    int64_t partial_ld;
    Epilogue e;
    OrthStore o;
};
enum { MM_LINEAR, MM_PARTIAL, MM_ORTH };
enum { TILE_64, TILE_128, TILE_256, TILES };
constexpr int64_t TILE_SIDE[TILES] = {64, 128, 256};
// what a product is made of: operands and result of bfloat16, half or fp32; fp32
// operands in three bfloat16 parts; an update's in two half parts
enum { MM_BF16, MM_F16, MM_F32, MM_F32_PARTS, MM_HALVES, MM_KINDS };
// tile: TILE_*
hipError_t launch_mm_bf16(const Mm& p, int tile, hipStream_t stream);
hipError_t launch_mm_f16(const Mm& p, int tile, hipStream_t stream);
hipError_t launch_mm_f32(const Mm& p, hipStream_t stream);                   // (64 alone)
hipError_t launch_mm_f32_parts(const Mm& p, int tile, hipStream_t stream);   // (no 256 tile)
// kind: MM_BF16 ... (tiles as above, no 256)
hipError_t launch_mm_partial(const Mm& p, int kind, int tile, hipStream_t stream);
hipError_t launch_mm_orth(const Mm& p, int tile, hipStream_t stream);
// two unsplit products in 64 tiles, dx's a along the reduction, the other operands
// across it; kind: not MM_HALVES
hipError_t launch_mm_two(const Mm& dx, const Mm& dw, int kind, int wgs_dx, int wgs_dw, hipStream_t stream);
// the partial sums of a split product added up and stored (dtype: of y)
hipError_t launch_mm_join(const Mm& p, int dtype, hipStream_t stream);
hipError_t launch_orth_join(const Mm& p, hipStream_t stream);

// y of at most SKINNY_ROWS rows, operands as they lie: x row by row, weight along
// the reduction or (across) input by output
constexpr int64_t SKINNY_ROWS = 32;
struct SkinnyParams {
    const void* x;
    int64_t x_ld;
    const void* w;
    int64_t w_ld;
    int32_t across;
    int64_t M, N, K;
    Epilogue e;
};
hipError_t launch_skinny(const SkinnyParams& p, int dtype, hipStream_t stream);

// rows x cols values of any strides as an operand's rows of ld elements: as they
// are, or fp32 in three bfloat16 parts
struct PackParams {
    const void* src;
    int64_t rs, cs;
    int64_t rows, cols;
    void* dst;
    int64_t ld;
};
// column sums of `chunks` rows of sums
struct ColumnSums {
    const float* part;
    int64_t chunks, N;
    void* out;
};
// two matrices packed and column sums finished, any of them NULL: one launch
// (kind: MM_*, of the products that follow)
hipError_t launch_prepare(const PackParams* a, const PackParams* b, const ColumnSums* c, int kind,
                          hipStream_t stream);

// dz = dy act'(pre), and with dbias the column sums of dz by chunks of rows
struct SlopeParams {
    const void* dy;
    int64_t dy_rs, dy_cs;
    const void* pre;
    int64_t pre_rs, pre_cs;
    int64_t M, N;
    int32_t act;
    void* dz;        // NULL: not wanted; an operand's rows
    int64_t ldz;
    void* dbias;     // NULL: not wanted
    float* part;     // [slope_chunks(M)][N] column sums of the chunks of rows
};
int64_t slope_chunks(int64_t M, int64_t N);
hipError_t launch_slope(const SlopeParams& p, int kind, hipStream_t stream);

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
    float* part;     // backward: [norm_parts(...)][2][N] sums over rows
    float eps;
};
int norm_parts(int64_t M, int64_t N, int dtype);
hipError_t launch_norm(const NormParams& p, int dtype, int weight_dtype, hipStream_t stream);
hipError_t launch_norm_backward(const NormParams& p, int dtype, int weight_dtype,
                                hipStream_t stream);

// `batch` updates of rows x cols: their norms (part: [batch][chunks] sums of
// squares), and scale g / (|g| + eps) as an operand of two halves or, with out,
// as the result
struct OrthParams {
    const void* g;
    int64_t g_batch, g_rs, g_cs;
    int64_t batch, rows, cols;
    double eps;
    double* part;
    int32_t chunks;
    float scale;
    f16* z;
    int64_t z_ld, z_batch;
    void* out;
    int64_t out_ld, out_batch;
};
hipError_t launch_orth_begin(const OrthParams& p, int dtype, hipStream_t stream);

// the host's error record (api.hip)
int set_error(int code, const char* msg);
int device_cu_count();
int set_hip_error(hipError_t e, const char* where);
void clear_error();

}  // namespace mag
