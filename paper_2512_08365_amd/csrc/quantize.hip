// quantize.hip -- numbers cut to 8 bits with a scale for each block.
//
// Bound by memory: x is read once, q and qt are written once.  A block of a row is 16
// lanes of 8 neighbours, its largest magnitude a reduction within them.  For the
// transpose (and blocks of 128 x 128) a workgroup holds a tile of 128 x 128 in
// registers, 8 x 8 a thread, takes the largest of rows and columns from there and
// turns the transpose's bytes in LDS, 8 neighbours of a column at a time.

#include <algorithm>

#include "fp8.hpp"
#include "mm.hpp"
#include "rows.hpp"

namespace mag {
namespace {

// How a block's numbers x become x / scale, scale = max(most / LARGEST, 2^-126).  The
// largest numbers of both formats are 0.875 times a power of two, 2^9 and 2^16: x /
// scale = 0.875 x / (most 2^-9), whose parts are exact for two-byte x, and whose
// quotient, a reciprocal and one correction, is right to the last place: ties
// between two numbers of the format are then seen as such (by a product with the
// reciprocal of a rounded scale, of 8,192 x 4,096 one number in 10,000 went the
// other way).
template <int FORMAT>
struct Cut {
    static constexpr float LARGEST = FORMAT == MAG_E4M3 ? 448.0f : 57344.0f;
    static constexpr float DOWN = FORMAT == MAG_E4M3 ? 0x1p-9f : 0x1p-16f;
    static constexpr float ONE = 1.0f / LARGEST;
    float d, inverse;

    __device__ __forceinline__ explicit Cut(float most)
    {
        d = fmaxf(most * DOWN, 0.875f * 0x1p-126f);
        // (d and 1 / d lie between 2^-127 and 2^127: neither argument nor result of the
        // hardware's reciprocal, off by a unit of the last place, is a small number)
        inverse = __builtin_amdgcn_rcpf(d * 16.0f) * 16.0f;
        // (an infinite one: finite numbers become 0, infinite ones NaN)
        if (most == __builtin_inff()) d = 1.0f, inverse = 0.0f;
    }
    static __device__ __forceinline__ float scale(float most)
    {
        // (most / LARGEST, to the last place by a correction; an infinite one stays it)
        const float q = most * ONE, s = fmaf(fmaf(-q, LARGEST, most), ONE, q);
        return fmaxf(most == __builtin_inff() ? most : s, (float)MAG_FP8_LEAST_SCALE);
    }
    __device__ __forceinline__ float operator()(float x) const
    {
        const float n = 0.875f * x, q = n * inverse;
        return fmaf(fmaf(-q, d, n), inverse, q);
    }
    // four neighbours
    __device__ __forceinline__ uint32_t four(float a, float b, float c, float e) const
    {
        int v = 0;
        if constexpr (FORMAT == MAG_E4M3) {
            v = __builtin_amdgcn_cvt_pk_fp8_f32((*this)(a), (*this)(b), v, false);
            v = __builtin_amdgcn_cvt_pk_fp8_f32((*this)(c), (*this)(e), v, true);
        } else {
            v = __builtin_amdgcn_cvt_pk_bf8_f32((*this)(a), (*this)(b), v, false);
            v = __builtin_amdgcn_cvt_pk_bf8_f32((*this)(c), (*this)(e), v, true);
        }
        return (uint32_t)v;
    }
};

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// eight bytes from column j of a row on (n of them)
__device__ __forceinline__ void put8(uint8_t* p, u32x2 v, int n)
{
    typedef u32x2 Any __attribute__((aligned(1)));
    if (n >= 8) {
        *(Any*)p = v;
    } else {
        for (int i = 0; i < n; ++i) p[i] = (uint8_t)(v[i / 4] >> (i % 4 * 8));
    }
}

// v of another lane of a group of 16 (CONTROL: the data-parallel one of the instruction)
template <int CONTROL>
__device__ __forceinline__ float moved(float v)
{
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CONTROL, 0xf, 0xf, true));
}

// the largest of 16 neighbouring lanes
__device__ __forceinline__ float most_of_16(float v)
{
    v = fmaxf(v, moved<0xb1>(v));    // lane ^ 1
    v = fmaxf(v, moved<0x4e>(v));    // lane ^ 2
    v = fmaxf(v, moved<0x141>(v));   // 7 - lane % 8
    return fmaxf(v, moved<0x140>(v));   // 15 - lane % 16
}

// the largest of the four lanes 16 apart
__device__ __forceinline__ float most_of_rows(float v)
{
    const unsigned a = __builtin_bit_cast(unsigned, v);
    const auto x = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const unsigned x0 = x[0], x1 = x[1];
    v = fmaxf(__builtin_bit_cast(float, x0), __builtin_bit_cast(float, x1));
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto y = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const unsigned y0 = y[0], y1 = y[1];
    return fmaxf(__builtin_bit_cast(float, y0), __builtin_bit_cast(float, y1));
}

// Eight neighbours from column j on, whose places and values settled() gives: zeros from
// column `cols` on.  WHOLE: neighbours in memory, in rows of whole blocks.
template <bool WHOLE, class T>
__device__ __forceinline__ void eight(Held<T, 8>& h, const T* row, int64_t cs, int64_t j, int64_t cols)
{
    if (WHOLE)
        get<1, 8, false>(h, row + j, 0, 8);
    else if (cs == 1 && cols >= 8)
        fetch<1, 8, true>(h, row, (int)(j / 8), (int)cols);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) h.v[i] = row[min(j + i, cols - 1) * cs];
}
template <bool WHOLE, class T>
__device__ __forceinline__ void settled(Held<T, 8>& h, int64_t cs, int64_t j, int64_t cols, float* v)
{
    if (!WHOLE && cs == 1 && cols >= 8) settle<1, 8, true>(h, (int)(j / 8), (int)cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = WHOLE || j + i < cols ? (float)h.v[i] : 0.0f;
}

constexpr int BLOCKS = 4;   // of a row, by each 16 lanes

// blocks of rows whose elements are neighbours: 16 rows by 4 blocks a workgroup (16
// rows' scales are then neighbours where they lie by columns)
template <class T, int FORMAT, bool WHOLE>
__device__ __forceinline__ void quantize_rows(const QuantizeParams& p, uint32_t across)
{
    const int64_t r = (int64_t)(blockIdx.x / across) * 16 + threadIdx.x / 16;
    const int64_t b0 = (int64_t)(blockIdx.x % across) * BLOCKS;
    const int c = threadIdx.x % 16 * 8;
    if (r >= p.rows) return;   // (16 lanes together)
    const T* x = static_cast<const T*>(p.x) + r * p.rs;
    Held<T, 8> h[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i)
        if (!WHOLE || (b0 + i) * FP8_BLOCK < p.cols) eight<WHOLE>(h[i], x, 1, (b0 + i) * FP8_BLOCK + c, p.cols);
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        const int64_t j = (b0 + i) * FP8_BLOCK + c;
        if ((b0 + i) * FP8_BLOCK >= p.cols) break;
        float v[8];
        settled<WHOLE>(h[i], 1, j, p.cols, v);
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[e]));
        most = most_of_16(most);
        const Cut<FORMAT> cut(most);
        put8(p.q + r * p.q_ld + j, u32x2{cut.four(v[0], v[1], v[2], v[3]),
                                         cut.four(v[4], v[5], v[6], v[7])},
             (int)max((int64_t)0, min((int64_t)8, p.cols - j)));
        if (c == 0) p.scale.p[r * p.scale.rs + (b0 + i) * p.scale.cs] = Cut<FORMAT>::scale(most);
    }
}

// tiles of 128 x 128, of any strides
constexpr int PITCH = FP8_BLOCK + 8;
template <class T, int FORMAT, bool SQUARE, bool WHOLE>
__device__ __forceinline__ void quantize_tile(const QuantizeParams& p, uint32_t across,
                                              float (&most_lds)[4][FP8_BLOCK], uint8_t* turned)
{
    const int64_t bi = blockIdx.x / across, bj = blockIdx.x % across;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int rg = threadIdx.x / 16 * 8, cg = threadIdx.x % 16 * 8;   // first of this thread's rows and columns
    const int64_t r0 = bi * FP8_BLOCK, c0 = bj * FP8_BLOCK;
    float v[8][8];
    {
        // (behind the last row: it once more, which no largest number changes with)
        Held<T, 8> h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            eight<WHOLE>(h[i], static_cast<const T*>(p.x) + min(r0 + rg + i, p.rows - 1) * p.rs, p.cs, c0 + cg, p.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) settled<WHOLE>(h[i], p.cs, c0 + cg, p.cols, v[i]);
    }
    float row[8], col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) row[i] = col[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(v[i][e]);
            row[i] = fmaxf(row[i], a);
            col[e] = fmaxf(col[e], a);
        }
    if constexpr (SQUARE) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, row[i]);
        most = most_of_rows(most_of_16(most));
        if (lane == 0) most_lds[wave][0] = most;
        __syncthreads();
        most = fmaxf(fmaxf(most_lds[0][0], most_lds[1][0]), fmaxf(most_lds[2][0], most_lds[3][0]));
#pragma unroll
        for (int i = 0; i < 8; ++i) row[i] = col[i] = most;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) row[i] = most_of_16(row[i]);
        if (p.qt) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                col[e] = most_of_rows(col[e]);
                if (lane < 16) most_lds[wave][cg + e] = col[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                col[e] = fmaxf(fmaxf(most_lds[0][cg + e], most_lds[1][cg + e]),
                               fmaxf(most_lds[2][cg + e], most_lds[3][cg + e]));
        }
    }
    if (p.q) {
        const int n = (int)max((int64_t)0, min((int64_t)8, p.cols - c0 - cg));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = r0 + rg + i;
            if (r >= p.rows) break;
            __builtin_amdgcn_sched_barrier(0);   // (a row at a time: registers)
            const Cut<FORMAT> cut(row[i]);
            put8(p.q + r * p.q_ld + c0 + cg, u32x2{cut.four(v[i][0], v[i][1], v[i][2], v[i][3]),
                                                   cut.four(v[i][4], v[i][5], v[i][6], v[i][7])}, n);
            if (!SQUARE && cg == 0) p.scale.p[r * p.scale.rs + bj * p.scale.cs] = Cut<FORMAT>::scale(row[i]);
        }
        if (SQUARE && threadIdx.x == 0) p.scale.p[bi * p.scale.rs + bj * p.scale.cs] = Cut<FORMAT>::scale(row[0]);
    }
    if (!p.qt) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        __builtin_amdgcn_sched_barrier(0);
        const Cut<FORMAT> cut(col[e]);
        *(u32x2*)(turned + (cg + e) * PITCH + rg) =
            u32x2{cut.four(v[0][e], v[1][e], v[2][e], v[3][e]), cut.four(v[4][e], v[5][e], v[6][e], v[7][e])};
        if (!SQUARE && rg == 0 && c0 + cg + e < p.cols)
            p.scale_t.p[(c0 + cg + e) * p.scale_t.rs + bi * p.scale_t.cs] = Cut<FORMAT>::scale(col[e]);
    }
    if (SQUARE && threadIdx.x == 0) p.scale_t.p[bj * p.scale_t.rs + bi * p.scale_t.cs] = Cut<FORMAT>::scale(col[0]);
    __syncthreads();
    for (int f = threadIdx.x; f < FP8_BLOCK * 16; f += 256) {
        const int c = f / 16, h = f % 16 * 8;
        if (c0 + c >= p.cols) break;
        put8(p.qt + (c0 + c) * p.qt_ld + r0 + h, *(const u32x2*)(turned + c * PITCH + h),
             (int)max((int64_t)0, min((int64_t)8, p.rows - r0 - h)));
    }
}

template <class T, bool WHOLE>
__global__ __launch_bounds__(256) void k_quantize_rows(QuantizeParams p, uint32_t across, int32_t format)
{
    if (format == MAG_E4M3)
        quantize_rows<T, MAG_E4M3, WHOLE>(p, across);
    else
        quantize_rows<T, MAG_E5M2, WHOLE>(p, across);
}

template <class T, bool SQUARE, bool WHOLE>
__global__ __launch_bounds__(256, 3) void k_quantize_tile(QuantizeParams p, uint32_t across, int32_t format)
{
    __shared__ float most_lds[4][FP8_BLOCK];
    __shared__ __attribute__((aligned(16))) uint8_t turned[FP8_BLOCK * PITCH];
    if (format == MAG_E4M3)
        quantize_tile<T, MAG_E4M3, SQUARE, WHOLE>(p, across, most_lds, turned);
    else
        quantize_tile<T, MAG_E5M2, SQUARE, WHOLE>(p, across, most_lds, turned);
}

// n rows from r0 on (where scales go with 128 rows, at a multiple of them)
template <class T>
QuantizeParams rows_of(const QuantizeParams& all, bool square, int64_t r0, int64_t n)
{
    QuantizeParams p = all;
    p.x = static_cast<const T*>(p.x) + r0 * p.rs;
    p.rows = n;
    if (p.q) {
        p.q += r0 * p.q_ld;
        p.scale.p += (square ? r0 / FP8_BLOCK : r0) * p.scale.rs;
    }
    if (p.qt) {
        p.qt += r0;
        p.scale_t.p += r0 / FP8_BLOCK * p.scale_t.cs;
    }
    return p;
}

// (a launch has less than 2^32 threads: many millions of rows take several)
template <class T, bool WHOLE>
hipError_t launch(const QuantizeParams& all, int format, bool square, hipStream_t stream)
{
    constexpr int64_t MOST = 0xffffff;   // workgroups
    const int64_t nb = (all.cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const bool by_rows = !square && !all.qt && (all.cs == 1 || all.cols <= 1);
    const int64_t across = by_rows ? (nb + BLOCKS - 1) / BLOCKS : nb, each = by_rows ? 16 : FP8_BLOCK;
    const int64_t most = MOST / across * each;   // (across: 2^23 at most)
    for (int64_t r0 = 0; r0 < all.rows; r0 += most) {
        const QuantizeParams p = rows_of<T>(all, square, r0, std::min(most, all.rows - r0));
        const dim3 grid((unsigned)(across * ((p.rows + each - 1) / each)));
        if (by_rows)
            hipLaunchKernelGGL((k_quantize_rows<T, WHOLE>), grid, dim3(256), 0, stream, p, (uint32_t)across, format);
        else if (square)
            hipLaunchKernelGGL((k_quantize_tile<T, true, WHOLE>), grid, dim3(256), 0, stream, p, (uint32_t)nb, format);
        else
            hipLaunchKernelGGL((k_quantize_tile<T, false, WHOLE>), grid, dim3(256), 0, stream, p, (uint32_t)nb, format);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// (rows that end amid eight neighbours: 32,768 x 1,021 and its transpose 61 us by
// element, so 50 us; its bounds cost whole blocks 5%)
template <class T>
hipError_t launch(const QuantizeParams& p, int format, bool square, hipStream_t stream)
{
    return p.cs == 1 && p.cols % FP8_BLOCK == 0 ? launch<T, true>(p, format, square, stream)
                                                : launch<T, false>(p, format, square, stream);
}

__global__ __launch_bounds__(256) void k_pack8(Pack8Params p)
{
    const int64_t per_row = (p.cols + 15) / 16, n = p.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = quotient(i, per_row), c = (i - r * per_row) * 16;
        const uint8_t* src = p.src + r * p.rs;
        uint8_t v[16];
        if (p.cs == 1 && c + 16 <= p.cols) {
            __builtin_memcpy(v, src + c, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = c + e < p.cols ? src[(c + e) * p.cs] : (uint8_t)0;
        }
        __builtin_memcpy(p.dst + r * p.ld + c, v, 16);
    }
}

}  // namespace

hipError_t launch_quantize(const QuantizeParams& p, int dtype, int format, bool square, hipStream_t stream)
{
    if (dtype == MAG_F32) return launch<float>(p, format, square, stream);
    if (dtype == MAG_F16) return launch<f16>(p, format, square, stream);
    return launch<bf16>(p, format, square, stream);
}

hipError_t launch_pack8(const Pack8Params& p, hipStream_t stream)
{
    const int64_t n = p.rows * ((p.cols + 15) / 16);
    hipLaunchKernelGGL(k_pack8, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
