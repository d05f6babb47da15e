// clip.hip -- the common norm of many tensors, and the tensors scaled to it.
//
// Bound by memory: every tensor is read once for the norm and once more to be scaled.
// The elements of a launch's tensors are one run of chunks that workgroups go through
// side by side, so that a small tensor costs no more than its bytes; a chunk's tensor is
// found by bisection among the launch's arguments.  Squares are summed in fp64 (those of
// fp32 pass its range), a fixed number of partial sums in a fixed order.

#include <algorithm>
#include <type_traits>

#include "rows.hpp"
#include "step.hpp"

namespace mag {
namespace {

constexpr uint32_t STREAMED = 8192;   // chunks: 128 MB of two-byte numbers
constexpr int THREADS = 256, PER = (int)CHUNK / THREADS;   // elements a thread of a chunk

// the span of a chunk
__device__ __forceinline__ int span_of(const Spans& s, uint32_t chunk)
{
    int lo = 0, hi = s.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s.span[mid].first <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

template <class T>
struct Vec {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T Any __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// f over the elements of a chunk and their places in the output: 16 bytes a lane at
// once, or one element of a tensor's end or of one whose rows are apart
template <class T, class F>
__device__ __forceinline__ void each_of(const Span& s, uint32_t chunk, F& f)
{
    constexpr int N = Vec<T>::N;
    const int64_t from = (int64_t)(chunk - s.first) * CHUNK;
    const T* in = static_cast<const T*>(s.in);
    if (s.cols == 0 && from + CHUNK <= s.count) {
        typename Vec<T>::Any v[PER / N];
#pragma unroll
        for (int k = 0; k < PER / N; ++k) v[k] = *(const typename Vec<T>::Any*)(in + from + (k * THREADS + threadIdx.x) * N);
#pragma unroll
        for (int k = 0; k < PER / N; ++k) f.whole(s, v[k], from + (k * THREADS + threadIdx.x) * N);
        return;
    }
    for (int64_t i = from + threadIdx.x; i < min(s.count, from + CHUNK); i += THREADS) {
        int64_t a = i, b = i;
        if (s.cols) {
            const int64_t row = i / s.cols, col = i - row * s.cols;
            a = row * s.in_ld + col;
            b = row * s.out_ld + col;
        }
        f.one(s, in[a], b);
    }
}

// |v| as an unsigned number: larger ones are larger, infinity above all finite ones,
// NaN above that
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }

template <bool INF>
struct Sum {
    double s = 0.0;
    uint32_t m = 0;
    template <class T>
    __device__ __forceinline__ void one(const Span&, T x, int64_t)
    {
        const float v = (float)x;
        if constexpr (INF)
            m = max(m, magnitude(v));
        else
            s = fma((double)v, (double)v, s);
    }
    template <class Any>
    __device__ __forceinline__ void whole(const Span& p, const Any& v, int64_t)
    {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(Any) / sizeof(v[0])); ++i) one(p, v[i], 0);
    }
    static __device__ __forceinline__ bool done(const Span&) { return false; }
    // over the workgroup's threads, in every one
    __device__ __forceinline__ double over_threads(double (&lds)[THREADS / 64])
    {
        double v = INF ? (double)__builtin_bit_cast(float, m) : s;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) v = join(v, __shfl_xor(v, d, 64));
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = join(v, lds[w]);
        return v;
    }
    // (NaN is the largest of all)
    static __device__ __forceinline__ double join(double a, double b)
    {
        return INF ? (a != a || a > b ? a : b) : a + b;
    }
};

template <class F>
__device__ __forceinline__ void over_chunks(const Spans& s, bool backwards, F& f)
{
    for (uint32_t c = blockIdx.x; c < s.chunks; c += gridDim.x) {
        const uint32_t chunk = backwards ? s.chunks - 1 - c : c;
        const Span& span = s.span[span_of(s, chunk)];
        if (f.done(span)) continue;
        if (span.dtype == MAG_F32)
            each_of<float>(span, chunk, f);
        else if (span.dtype == MAG_F16)
            each_of<f16>(span, chunk, f);
        else
            each_of<bf16>(span, chunk, f);
    }
}

template <bool INF>
__global__ __launch_bounds__(THREADS) void k_clip_norm(Spans s, double* part)
{
    __shared__ double lds[THREADS / 64];
    Sum<INF> f;
    over_chunks(s, false, f);
    const double v = f.over_threads(lds);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

// PAST: stores go past the caches
template <bool PAST>
struct Scaling {
    // The factor is the two's product: one below 2^-126 would lack digits as a float, and
    // makes normal numbers of large ones all the same (below 2^-277 it makes zeros).
    float by, then;
    __device__ __forceinline__ explicit Scaling(double factor)
    {
        const double up = factor >= 0x1p-126 ? 1.0 : factor >= 0x1p-226 ? 0x1p100 : 0x1p149;
        by = (float)(factor * up);
        then = (float)(1.0 / up);
    }
    // nothing to do: in place, and not clipped (eight bfloat16 tensors of 4,096 x 16,384
    // 595 us, so 214 us)
    __device__ __forceinline__ bool done(const Span& s) const
    {
        return by == 1.0f && s.in == s.out && (!s.cols || s.in_ld == s.out_ld);
    }
    template <class T>
    __device__ __forceinline__ void one(const Span& s, T x, int64_t i)
    {
        static_cast<T*>(s.out)[i] = (T)((float)x * by * then);
    }
    template <class Any>
    __device__ __forceinline__ void whole(const Span& s, const Any& v, int64_t i)
    {
        using T = typename std::remove_cv<typename std::remove_reference<decltype(v[0])>::type>::type;
        Any o;
#pragma unroll
        for (int k = 0; k < (int)(sizeof(Any) / sizeof(T)); ++k) o[k] = (T)((float)v[k] * by * then);
        Any* to = (Any*)(static_cast<T*>(s.out) + i);
        if constexpr (PAST)
            __builtin_nontemporal_store(o, to);
        else
            *to = o;
    }
};

// Each workgroup adds the partial sums up itself: a launch less.  PAST: of tensors that no
// cache holds, part of what the norm read last is still there for the second reading,
// if what is written leaves it: four blocks' gradients, 1.1 GB, 631 us, so 588 us (by
// a run of chunks each; side by side 561 us).
// (Smaller lists' outputs are better kept for who reads them.)
template <bool INF, bool PAST>
__global__ __launch_bounds__(THREADS) void k_clip_scale(Spans s, const double* part, int parts, double most,
                                                        double eps, float* norm)
{
    __shared__ double lds[THREADS / 64];
    Sum<INF> sum;
    double v = 0.0;
    for (int i = threadIdx.x; i < parts; i += THREADS) v = Sum<INF>::join(v, part[i]);
    sum.s = v;
    if constexpr (INF) sum.m = magnitude((float)v);
    v = sum.over_threads(lds);
    if constexpr (!INF) v = sqrt(v);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)v;
    if (s.n == 0) return;
    const double by = most / (v + eps);
    // (a norm that is NaN makes all NaN)
    Scaling<PAST> f(by > 1.0 ? 1.0 : by);
    over_chunks(s, true, f);
}

}  // namespace

hipError_t launch_clip_norm(const Spans& s, double* part, int wgs, bool inf, hipStream_t stream)
{
    if (inf)
        hipLaunchKernelGGL(k_clip_norm<true>, dim3((unsigned)wgs), dim3(THREADS), 0, stream, s, part);
    else
        hipLaunchKernelGGL(k_clip_norm<false>, dim3((unsigned)wgs), dim3(THREADS), 0, stream, s, part);
    return hipGetLastError();
}

hipError_t launch_clip_scale(const Spans& s, const double* part, int parts, int wgs, bool inf, double most,
                             double eps, float* norm, hipStream_t stream)
{
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(THREADS), 0, stream, s, part, parts, most, eps, norm);
    };
    if (s.chunks >= STREAMED)
        inf ? launch(k_clip_scale<true, true>) : launch(k_clip_scale<false, true>);
    else
        inf ? launch(k_clip_scale<true, false>) : launch(k_clip_scale<false, false>);
    return hipGetLastError();
}

}  // namespace mag
