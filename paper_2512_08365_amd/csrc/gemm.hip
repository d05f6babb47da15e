// gemm.hip -- what surrounds the products of the feed-forward block: operands
// laid out for them, the gradient through the activation, split sums joined.

#include <algorithm>

#include "mm.hpp"

namespace mag {
namespace {

typedef __attribute__((ext_vector_type(8))) short h8;

__device__ __forceinline__ short bits(bf16 v) { return __builtin_bit_cast(short, v); }

// An fp32 number as three bfloat16 parts that add up to it exactly: 8 bits of
// it, 8 of the rest, what is left (of numbers below 2^-110 the last part ends where
// bfloat16 does, half of 2^-133 off).  Rounding to nearest keeps every part's
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

// eight neighbours of row r, from element j of it, into an operand's rows (PARTS:
// in three parts)
template <class T, bool PARTS>
__device__ __forceinline__ void put8(const float* v, void* rows, int64_t ld, int64_t r, int64_t j)
{
    h8 o;
    if constexpr (PARTS) {
        h8 m, l;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            short a, b, c;
            three_parts(v[i], a, b, c);
            o[i] = a;
            m[i] = b;
            l[i] = c;
        }
        short* d = static_cast<short*>(rows) + r * ld + place<3>(j);
        *(h8*)d = o;
        *(h8*)(d + 32) = m;
        *(h8*)(d + 64) = l;
    } else {
        store8(static_cast<T*>(rows) + r * ld + j, v);
    }
}

// elements of an operand's row of n, without the parts
template <bool PARTS>
__host__ __device__ int64_t width_of(int64_t n)
{
    return PARTS ? (n + 31) / 32 * 32 : (n + 7) / 8 * 8;
}

// One thread's 8 neighbours of a packed row.
template <class T, bool PARTS>
__device__ __forceinline__ void pack_some(const PackParams& p, int64_t block, int64_t blocks)
{
    const int64_t per_row = width_of<PARTS>(p.cols) / 8, n = p.rows * per_row;
    for (int64_t i = block * 256 + threadIdx.x; i < n; i += blocks * 256) {
        const int64_t r = quotient(i, per_row), j = (i - r * per_row) * 8;
        float v[8];
        get8(static_cast<const T*>(p.src) + r * p.rs, p.cs, j, p.cols, v);
        put8<T, PARTS>(v, p.dst, p.ld, r, j);
    }
}

constexpr int SLOPE_COLS = 512;  // columns of a workgroup: 64 lanes of 8
constexpr int SLOPE_ROWS = 2;    // rows a wave has in flight (4: too many registers, 40 % slower)

// dz and the column sums of one chunk of rows.  dz is rounded to the operands' type,
// as x and weight are held, because the products' matrix instructions take no other:
// of two bytes the gradients are 1.4 times as far off as their own rounding (0.0023
// and 0.0017 of bfloat16); the sums take it unrounded.  Four waves take the rows in
// turn, 8 columns a lane, and add their sums up in LDS at the end.  Bound by
// memory (a prompt's 805 MB in 170 us).
template <class T, bool PARTS>
__global__ __launch_bounds__(256) void k_slope(SlopeParams p, int64_t chunk)
{
    __shared__ float sums[4][SLOPE_COLS + 4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t j = (int64_t)blockIdx.x * SLOPE_COLS + lane * 8;
    const int64_t i0 = (int64_t)blockIdx.y * chunk, i1 = min(i0 + chunk, p.M);
    const bool acts = p.act != MAG_ACT_NONE;
    float sum[8] = {};
    if (j < width_of<PARTS>(p.N))
        for (int64_t i = i0 + wave; i < i1; i += 4 * SLOPE_ROWS) {
            float d[SLOPE_ROWS][8], z[SLOPE_ROWS][8];
#pragma unroll
            for (int u = 0; u < SLOPE_ROWS; ++u) {
                const int64_t r = min(i + 4 * u, i1 - 1);
                get8(static_cast<const T*>(p.dy) + r * p.dy_rs, p.dy_cs, j, p.N, d[u]);
                if (acts) get8(static_cast<const T*>(p.pre) + r * p.pre_rs, p.pre_cs, j, p.N, z[u]);
            }
            if (acts) {
                slopes<T, 8 * SLOPE_ROWS>(z[0], p.act);
#pragma unroll
                for (int e = 0; e < 8 * SLOPE_ROWS; ++e) d[0][e] *= z[0][e];
            }
#pragma unroll
            for (int u = 0; u < SLOPE_ROWS; ++u) {
                if (i + 4 * u >= i1) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += d[u][e];
                if (p.dz) put8<T, PARTS>(d[u], p.dz, p.ldz, i + 4 * u, j);
            }
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

// 16 columns' sums of the chunks' sums, 16 threads each with all of their loads
// in flight
constexpr int SUM_COLS = 16;
template <class T>
__device__ __forceinline__ void column_sums(const ColumnSums& p, int64_t block)
{
    __shared__ float sums[16][SUM_COLS + 1];
    const int col = threadIdx.x % SUM_COLS, row = threadIdx.x / SUM_COLS;
    const int64_t j = block * SUM_COLS + col;
    float s[8] = {};
    if (j < p.N)
        for (int64_t c = row; c < p.chunks; c += 128)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (c + 16 * u < p.chunks) s[u] += p.part[(c + 16 * u) * p.N + j];
    sums[row][col] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (row || j >= p.N) return;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += sums[k][col];
    static_cast<T*>(p.out)[j] = (T)sum;
}

// What a layer's products need beforehand, side by side in one launch (each is
// a few us of latency): up to two matrices packed and the column sums finished.
template <class T, bool PARTS>
__global__ __launch_bounds__(256) void k_prepare(PackParams a, PackParams b, ColumnSums c,
                                                 uint32_t blocks_a, uint32_t blocks_b)
{
    if (blockIdx.x < blocks_a)
        pack_some<T, PARTS>(a, blockIdx.x, blocks_a);
    else if (blockIdx.x < blocks_a + blocks_b)
        pack_some<T, PARTS>(b, blockIdx.x - blocks_a, blocks_b);
    else
        column_sums<T>(c, blockIdx.x - blocks_a - blocks_b);
}

// Those of the m columns from s on of row r, a bit each, that have a NaN operand
// there; every lane of a wave asks for its own, of which only the ones that are
// wanted are looked at: each row and column once, by the whole wave.
__device__ __forceinline__ uint32_t nan_operands(const Mm& p, int64_t r, int64_t s, int m, bool wanted)
{
    uint32_t nan = 0;
    uint64_t left = __ballot(wanted);
    while (left) {   // by rows
        const int64_t row = __shfl(r, __ffsll((unsigned long long)left) - 1, 64);
        const uint64_t same = __ballot(r == row);
        if (row_has_nan(p.a, 0, row, p.K) && r == row) nan = 255u;
        left &= ~same;
    }
    left = __ballot(wanted && nan == 0);
    while (left) {   // ... and the others by columns
        const int lane = __ffsll((unsigned long long)left) - 1;
        const int64_t first = __shfl(s, lane, 64);
        const int count = __shfl(m, lane, 64);
        const uint64_t same = __ballot(s == first);
        uint32_t found = 0;
#pragma unroll 1
        for (int e = 0; e < count; ++e)
            if (row_has_nan(p.b, 0, first + e, p.K)) found |= 1u << e;
        if (s == first && nan == 0) nan = found;
        left &= ~same;
    }
    return nan;
}

// A split product's parts added up and stored, 8 neighbours of a row a thread.
// Bound by latency where there are few (1,920 x 384 of 3 parts: 5 us), else by
// memory.
template <class TO>
__global__ __launch_bounds__(256) void k_mm_join(Mm p)
{
    const int64_t per_row = p.partial_ld / 8, n = p.R * per_row;
    const int64_t plane = p.R * p.partial_ld;
    // (a wave's threads go together: they look for NaN operands side by side)
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x / 64 * 64; at < n; at += (int64_t)gridDim.x * 256) {
        const int64_t i = at + threadIdx.x % 64;
        const bool on = i < n;
        const int64_t r = quotient(on ? i : n - 1, per_row), s = ((on ? i : n - 1) - r * per_row) * 8;
        float v[8] = {};
        add_parts(p.partial + r * p.partial_ld + s, plane, p.splits, v);
        const int m = (int)min((int64_t)8, p.S - s);
        if constexpr (sizeof(TO) == 4)
            if (p.in_parts) {
                const uint32_t nan = nan_operands(p, r, s, m, !all_finite(v));
                make_whole(p, 0, r, s, m, nan, v);
            }
        if (on) store_linear<TO>(p.e, r, s, m, v);
    }
}

unsigned blocks_for(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16); }

}  // namespace

hipError_t launch_prepare(const PackParams* a, const PackParams* b, const ColumnSums* c, int kind,
                          hipStream_t stream)
{
    auto blocks = [](const PackParams* p) {
        return p ? blocks_for(p->rows * ((p->cols + 7) / 8)) : 0u;
    };
    const unsigned na = blocks(a), nb = blocks(b), nc = c ? (unsigned)((c->N + SUM_COLS - 1) / SUM_COLS) : 0u;
    if (na + nb + nc == 0) return hipSuccess;
    const PackParams none{};
    const ColumnSums no{};
    const dim3 grid(na + nb + nc), block(256);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, a ? *a : none, b ? *b : none, c ? *c : no, na, nb);
    };
    switch (kind) {
    case MM_F32: launch(k_prepare<float, false>); break;
    case MM_F32_PARTS: launch(k_prepare<float, true>); break;
    case MM_F16: launch(k_prepare<f16, false>); break;
    default: launch(k_prepare<bf16, false>); break;
    }
    return hipGetLastError();
}

// chunks of rows of the column sums: enough workgroups to fill the device
int64_t slope_chunks(int64_t M, int64_t N)
{
    const int64_t across = (N + SLOPE_COLS - 1) / SLOPE_COLS;
    // (256 at most: few columns' sums would be long in finishing them)
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(2048 / std::max<int64_t>(across, 1), 256));
    return std::max<int64_t>(1, std::min<int64_t>(want, (M + 4 * SLOPE_ROWS - 1) / (4 * SLOPE_ROWS)));
}

hipError_t launch_slope(const SlopeParams& p, int kind, hipStream_t stream)
{
    if (p.N == 0) return hipSuccess;
    const int64_t chunks = slope_chunks(p.M, p.N), chunk = (p.M + chunks - 1) / chunks;
    const dim3 grid((unsigned)((p.N + SLOPE_COLS - 1) / SLOPE_COLS), (unsigned)chunks), block(256);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, p, chunk); };
    switch (kind) {
    case MM_F32: launch(k_slope<float, false>); break;
    case MM_F32_PARTS: launch(k_slope<float, true>); break;
    case MM_F16: launch(k_slope<f16, false>); break;
    default: launch(k_slope<bf16, false>); break;
    }
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
