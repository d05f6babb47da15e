// norm.hip -- layer norm, forward and backward.
//
// Both passes are bound by memory: every row is read once into registers, and
// what a row needs of its neighbours is one reduction (the backward pass's two
// sums go together).  A row belongs to 64, 256, 512 or 1,024 threads, the fewest
// that hold it in 16 elements each: few enough registers that the rows'
// weights stay in them from row to row (a 2-byte row's fp32 weight and bias are
// four times its bytes, and would come from L2 each time), and so do the
// backward pass's sums over the rows.  Workgroups walk the rows and load the
// next one before they reduce the present one.
//
// A mean is a sum over 16 elements a thread and a tree; the variance is taken
// from squares about it, both in fp32.
//
// 32,768 x 4,096 bfloat16: forward 537 MB in 105 us, backward 805 MB in 151 us and
// its columns 8 us (5.1 and 5.1 TB/s); one row 2.8 us.

#include <algorithm>

#include "rows.hpp"

namespace mag {
namespace {

constexpr int HELD = 16;          // elements a thread
constexpr int64_t MOST_HELD = 1024 * HELD;  // width of a row that 1,024 threads hold
constexpr int BACK_WGS = 256;     // workgroups of the backward pass, each with its own sums over
                                  // rows (twice as many where a CU's registers hold two)

template <class T, class W, int G, int V, bool TAIL, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm(NormParams p)
{
    constexpr int ROWS = THREADS / G;  // at a time
    __shared__ float2 lds[2][THREADS / 64];
    const int lane = threadIdx.x % G, n = (int)p.N;
    const int sub = __builtin_amdgcn_readfirstlane((int)threadIdx.x / G);
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const T* x = static_cast<const T*>(p.x);
    float w[HELD], b[HELD];
    {
        Held<W, HELD> a{}, d{};
        if (p.weight) get<G, V, TAIL>(a, static_cast<const W*>(p.weight), lane, n);
        if (p.bias) get<G, V, TAIL>(d, static_cast<const W*>(p.bias), lane, n);
#pragma unroll
        for (int e = 0; e < HELD; ++e) {
            w[e] = p.weight ? (float)a.v[e] : 1.0f;
            b[e] = (float)d.v[e];
        }
    }
    Held<T, HELD> next{};
    const int64_t i0 = (int64_t)blockIdx.x * ROWS;
    if (i0 + sub < p.M) get<G, V, TAIL>(next, x + (i0 + sub) * p.x_rs, lane, n);
    // (the workgroup's rows go together: its barriers are everybody's)
    for (int64_t base = i0; base < p.M; base += step) {
        const int64_t i = base + sub;
        float v[HELD], s = 0.0f, unused = 0.0f;
#pragma unroll
        for (int e = 0; e < HELD; ++e) {
            v[e] = (float)next.v[e];
            s += v[e];
        }
        if (i + step < p.M) get<G, V, TAIL>(next, x + (i + step) * p.x_rs, lane, n);
        row_sums<G>(s, unused, lds[0]);
        const float mean = s / (float)n;
        s = 0.0f;
#pragma unroll
        for (int e = 0; e < HELD; ++e) {
            v[e] = column<G, V>(lane, e) < n ? v[e] - mean : 0.0f;
            s = fmaf(v[e], v[e], s);
        }
        row_sums<G>(s, unused, lds[1]);
        const float rstd = 1.0f / sqrtf(s / (float)n + p.eps);
        if (i >= p.M) continue;
#pragma unroll
        for (int e = 0; e < HELD; ++e) v[e] = fmaf(v[e] * rstd, w[e], b[e]);
        put<G, V, TAIL, HELD>(static_cast<T*>(p.y) + i * p.y_ld, lane, n, v);
        if (lane == 0) {
            if (p.mean) p.mean[i] = mean;
            if (p.rstd) p.rstd[i] = rstd;
        }
    }
}

// rows too wide for the threads' registers, or whose elements are not neighbours
// in memory: read three times (the second and third time from L2).  Workgroups
// walk the rows: one a row would pass a launch's 2^32 threads from 2^22 rows on.
template <class T, class W>
__global__ __launch_bounds__(1024) void k_norm_wide(NormParams p)
{
    __shared__ float2 lds[2][16];
    const int64_t n = p.N;
    const W *w = static_cast<const W*>(p.weight), *b = static_cast<const W*>(p.bias);
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + i * p.x_rs;
        float s = 0.0f, unused = 0.0f;
        for (int64_t j = threadIdx.x; j < n; j += 1024) s += (float)x[j * p.x_cs];
        row_sums<1024>(s, unused, lds[0]);
        const float mean = s / (float)n;
        s = 0.0f;
        for (int64_t j = threadIdx.x; j < n; j += 1024) {
            const float d = (float)x[j * p.x_cs] - mean;
            s = fmaf(d, d, s);
        }
        row_sums<1024>(s, unused, lds[1]);
        const float rstd = 1.0f / sqrtf(s / (float)n + p.eps);
        for (int64_t j = threadIdx.x; j < n; j += 1024)
            static_cast<T*>(p.y)[i * p.y_ld + j] =
                (T)fmaf(((float)x[j * p.x_cs] - mean) * rstd, w ? (float)w[j] : 1.0f, b ? (float)b[j] : 0.0f);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[i] = mean;
            if (p.rstd) p.rstd[i] = rstd;
        }
    }
}

// Gradients: each workgroup walks its rows, keeps the sums
// over them of its columns in registers, adds up the threads of one column at
// the end through LDS (one set of threads after another: a fixed order) and
// leaves one row of sums for weight and bias each.
template <class T, class W, int G, int V, bool TAIL, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_back(NormParams p)
{
    constexpr int ROWS = THREADS / G;
    // (1,024 threads have 128 registers each: no room for a row loaded ahead)
    constexpr bool AHEAD = THREADS < 1024;
    __shared__ float2 lds[2][THREADS / 64];
    __shared__ float sums[ROWS == 1 ? 1 : 2][ROWS == 1 ? 1 : G * HELD];
    const int lane = threadIdx.x % G, n = (int)p.N;
    const int sub = __builtin_amdgcn_readfirstlane((int)threadIdx.x / G);
    const int64_t step = (int64_t)gridDim.x * ROWS;
    const T *x = static_cast<const T*>(p.x), *dy = static_cast<const T*>(p.dy);
    float w[HELD], dw[HELD] = {}, db[HELD] = {};
    {
        Held<W, HELD> a{};
        if (p.weight) get<G, V, TAIL>(a, static_cast<const W*>(p.weight), lane, n);
#pragma unroll
        for (int e = 0; e < HELD; ++e) w[e] = p.weight ? (float)a.v[e] : 1.0f;
    }
    Held<T, HELD> nx{}, ny{};
    auto load = [&](int64_t i) {
        get<G, V, TAIL>(nx, x + i * p.x_rs, lane, n);
        get<G, V, TAIL>(ny, dy + i * p.dy_rs, lane, n);
    };
    const int64_t i0 = (int64_t)blockIdx.x * ROWS;
    if (AHEAD && i0 + sub < p.M) load(i0 + sub);
    int turn = 0;
    for (int64_t base = i0; base < p.M; base += step) {
        const int64_t i = base + sub;
        const bool on = i < p.M;
        const float mean = on ? p.mean[i] : 0.0f, r = on ? p.rstd[i] : 0.0f;
        if (!AHEAD && on) load(i);
        float xh[HELD], h[HELD], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int e = 0; e < HELD; ++e) {
            // (beyond the width, and for a row beyond the last: 0)
            const bool in = on && column<G, V>(lane, e) < n;
            xh[e] = in ? ((float)nx.v[e] - mean) * r : 0.0f;
            const float d = in ? (float)ny.v[e] : 0.0f;
            dw[e] = fmaf(d, xh[e], dw[e]);
            db[e] += d;
            h[e] = d * w[e];
            s1 += h[e];
            s2 = fmaf(h[e], xh[e], s2);
        }
        if (AHEAD && i + step < p.M) load(i + step);
        if (!p.y) continue;
        row_sums<G>(s1, s2, lds[turn ^= 1]);
        if (!on) continue;
        s1 /= (float)n;
        s2 /= (float)n;
#pragma unroll
        for (int e = 0; e < HELD; ++e) h[e] = r * (h[e] - s1 - xh[e] * s2);
        put<G, V, TAIL, HELD>(static_cast<T*>(p.y) + i * p.y_ld, lane, n, h);
    }
    if (!p.dweight && !p.dbias) return;
    float* part = p.part + (int64_t)blockIdx.x * 2 * n;
    if constexpr (ROWS == 1) {
        put<G, V, TAIL, HELD>(part, lane, n, dw);
        put<G, V, TAIL, HELD>(part + n, lane, n, db);
    } else {
        for (int t = 0; t < ROWS; ++t) {
            if (sub == t)
#pragma unroll
                for (int e = 0; e < HELD; ++e) {
                    // (by element, so that neighbouring lanes meet no bank twice)
                    const int at = e * G + lane;
                    sums[0][at] = t ? sums[0][at] + dw[e] : dw[e];
                    sums[1][at] = t ? sums[1][at] + db[e] : db[e];
                }
            __syncthreads();
        }
        for (int j = threadIdx.x; j < n; j += THREADS) {
            const int at = (j / V / G * V + j % V) * G + j / V % G;
            part[j] = sums[0][at];
            part[n + j] = sums[1][at];
        }
    }
}

// the workgroups' sums added up: 16 columns a workgroup, 64 threads each that
// have all of their loads in flight
template <class W>
__global__ __launch_bounds__(1024) void k_norm_columns(const float* part, int parts, int64_t n,
                                                       W* dweight, W* dbias)
{
    __shared__ float sums[64][17];
    const int col = threadIdx.x % 16, row = threadIdx.x / 16;
    const int64_t j = (int64_t)blockIdx.x * 16 + col;
    float t[8] = {};
    if (j < 2 * n)
        for (int k = row; k < parts; k += 512)
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + 64 * u < parts) t[u] += part[(int64_t)(k + 64 * u) * 2 * n + j];
    sums[row][col] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
    __syncthreads();
    if (threadIdx.x >= 16 || j >= 2 * n) return;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 64; ++k) s += sums[k][col];
    if (j < n && dweight) dweight[j] = (W)s;
    if (j >= n && dbias) dbias[j - n] = (W)s;
}

// rows as k_norm_wide's: the sums over the rows by column...
template <class T>
__global__ __launch_bounds__(256) void k_norm_back_wide_columns(NormParams p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.N) return;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t i = blockIdx.y; i < p.M; i += gridDim.y) {
        const float d = (float)static_cast<const T*>(p.dy)[i * p.dy_rs + j * p.dy_cs];
        const float xh = ((float)static_cast<const T*>(p.x)[i * p.x_rs + j * p.x_cs] - p.mean[i]) *
                         p.rstd[i];
        sw = fmaf(d, xh, sw);
        sb += d;
    }
    p.part[(int64_t)blockIdx.y * 2 * p.N + j] = sw;
    p.part[(int64_t)blockIdx.y * 2 * p.N + p.N + j] = sb;
}

// ... and dx by row, after them (dx may be written over x or dy)
template <class T, class W>
__global__ __launch_bounds__(1024) void k_norm_back_wide(NormParams p)
{
    __shared__ float2 lds[2][16];
    const int64_t n = p.N;
    const W* w = static_cast<const W*>(p.weight);
    int turn = 0;
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + i * p.x_rs;
        const T* dy = static_cast<const T*>(p.dy) + i * p.dy_rs;
        const float mean = p.mean[i], rstd = p.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t j = threadIdx.x; j < n; j += 1024) {
            const float h = (float)dy[j * p.dy_cs] * (w ? (float)w[j] : 1.0f);
            s1 += h;
            s2 = fmaf(h, ((float)x[j * p.x_cs] - mean) * rstd, s2);
        }
        row_sums<1024>(s1, s2, lds[turn ^= 1]);
        s1 /= (float)n;
        s2 /= (float)n;
        for (int64_t j = threadIdx.x; j < n; j += 1024) {
            const float h = (float)dy[j * p.dy_cs] * (w ? (float)w[j] : 1.0f);
            const float xh = ((float)x[j * p.x_cs] - mean) * rstd;
            static_cast<T*>(p.y)[i * p.y_ld + j] = (T)(rstd * (h - s1 - xh * s2));
        }
    }
}

// workgroups that walk M rows, one at a time each
dim3 wide_grid(int64_t M) { return dim3((unsigned)std::min<int64_t>(M, 1 << 16)); }

// threads of a row of width n
int threads_of(int64_t n) { return n <= 64 * HELD ? 64 : n <= 256 * HELD ? 256 : n <= 512 * HELD ? 512 : 1024; }
// rows that a workgroup of the backward pass takes at a time
int back_rows(int64_t n) { return n <= 64 * HELD ? 8 : n <= 256 * HELD ? 2 : 1; }

template <class T, class W, int V, bool TAIL>
void forward_held(const NormParams& p, hipStream_t stream)
{
    // as many workgroups as the device holds at once, the rows spread evenly
    // over them
    const int G = threads_of(p.N), rows = G == 64 ? 4 : 1;
    const int64_t groups = (p.M + rows - 1) / rows;
    const int64_t most = G == 1024 ? 512 : G == 512 ? 1024 : 2048, rounds = (groups + most - 1) / most;
    const dim3 grid((unsigned)((groups + rounds - 1) / rounds));
    if (G == 64)
        hipLaunchKernelGGL((k_norm<T, W, 64, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 256)
        hipLaunchKernelGGL((k_norm<T, W, 256, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 512)
        hipLaunchKernelGGL((k_norm<T, W, 512, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else
        hipLaunchKernelGGL((k_norm<T, W, 1024, V, TAIL, 1024>), grid, dim3(1024), 0, stream, p);
}

template <class T, class W>
hipError_t forward(const NormParams& p, hipStream_t stream)
{
    if (p.N > MOST_HELD || (p.N > 1 && p.x_cs != 1))   // (one column: its stride may be anything)
        hipLaunchKernelGGL((k_norm_wide<T, W>), wide_grid(p.M), dim3(1024), 0, stream, p);
    else if (p.N % 8 == 0)
        forward_held<T, W, 8, false>(p, stream);
    else
        forward_held<T, W, sizeof(T) == 4 ? 1 : 8, sizeof(T) == 2>(p, stream);
    return hipGetLastError();
}

template <class T, class W, int V, bool TAIL>
void backward_held(const NormParams& p, int parts, hipStream_t stream)
{
    const int G = threads_of(p.N);
    const dim3 grid(parts);
    if (G == 64)
        hipLaunchKernelGGL((k_norm_back<T, W, 64, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else if (G == 256)
        hipLaunchKernelGGL((k_norm_back<T, W, 256, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else if (G == 512)
        hipLaunchKernelGGL((k_norm_back<T, W, 512, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else
        hipLaunchKernelGGL((k_norm_back<T, W, 1024, V, TAIL, 1024>), grid, dim3(1024), 0, stream, p);
}

template <class T, class W>
hipError_t backward(const NormParams& p, hipStream_t stream)
{
    const bool sums = p.dweight || p.dbias;
    const bool wide = p.N > MOST_HELD || (p.N > 1 && (p.x_cs != 1 || p.dy_cs != 1));
    const int parts = norm_parts(p.M, p.N, sizeof(T) == 4 ? MAG_F32 : MAG_BF16);
    if (wide && sums)
        hipLaunchKernelGGL(k_norm_back_wide_columns<T>, dim3((unsigned)((p.N + 255) / 256), parts),
                           dim3(256), 0, stream, p);
    else if (!wide && (p.y || sums)) {
        if (p.N % 8 == 0)
            backward_held<T, W, 8, false>(p, parts, stream);
        else
            backward_held<T, W, sizeof(T) == 4 ? 1 : 8, sizeof(T) == 2>(p, parts, stream);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (sums) {
        hipLaunchKernelGGL(k_norm_columns<W>, dim3((unsigned)((2 * p.N + 15) / 16)), dim3(1024), 0,
                           stream, p.part, parts, p.N, static_cast<W*>(p.dweight),
                           static_cast<W*>(p.dbias));
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (wide && p.y && p.M > 0)
        hipLaunchKernelGGL((k_norm_back_wide<T, W>), wide_grid(p.M), dim3(1024), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

int norm_parts(int64_t M, int64_t N, int dtype)
{
    // the rows spread evenly over the workgroups
    const int64_t rows = back_rows(N);
    const int64_t most = dtype != MAG_F32 && rows > 1 ? 2 * BACK_WGS : BACK_WGS;
    const int64_t groups = std::max<int64_t>(1, (M + rows - 1) / rows), rounds = (groups + most - 1) / most;
    return (int)((groups + rounds - 1) / rounds);
}

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
