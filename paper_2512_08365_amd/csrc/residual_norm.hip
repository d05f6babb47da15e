// residual_norm.hip -- the norms around a block, fused with its gate, its residual scale
// and the addition between them, forward and backward.
//
// Both passes are bound by memory: the forward one reads the residual stream and the
// block's output and writes the new stream and its normed rows, the backward one
// reads four matrices and writes two.  Every row is read once into the registers of
// 64 to 1,024 threads, 8 elements each (of rows above 8,192 16), the next one while the
// present one's sums are taken.  A gate that many rows share is read once for a
// workgroup's rows of it.  Of a copy's 6.2 TB/s: 32,768 x 4,096 forward 5.2, backward 4.7;
// backward above 8,192 in two passes, 2.2 to 3.3.
//
// Sums over a row and over rows, statistics and gradients are fp32; the stream's sum
// is rounded to its type before the norm behind it reads it, as a reader of the
// stored rows would.

#include <algorithm>
#include <type_traits>

#include "rows.hpp"
#include "step.hpp"

namespace mag {
namespace {

constexpr int64_t MOST_HELD = 16384;   // width of a row that 1,024 threads hold
constexpr int64_t MOST_SUMMED = 8192;  // ... with its columns' sums
constexpr int VECTORS = 5;             // of partial sums

// v[j], of fp32 or of the rows' type T
template <class T>
__device__ __forceinline__ const void* from(const void* v, bool f32, int64_t j)
{
    return static_cast<const char*>(v) + j * (f32 ? 4 : (int64_t)sizeof(T));
}

// A vector's elements of this thread (ones or zeros: of one that is not there).  Weights
// are fp32 or of the rows' type; which, is looked at once a vector.
template <class W, int G, int V, bool TAIL, int E>
__device__ __forceinline__ void vector_as(float* to, const void* p, int lane, int n)
{
    Held<W, E> a{};
    fetch<G, V, TAIL>(a, static_cast<const W*>(p), lane, n);
    settle<G, V, TAIL>(a, lane, n);
#pragma unroll
    for (int e = 0; e < E; ++e) to[e] = (float)a.v[e];
}
template <class T, int G, int V, bool TAIL, int E>
__device__ __forceinline__ void vector(float* to, const void* p, bool f32, int lane, int n, float missing)
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = missing;
    } else if (sizeof(T) == 4 || f32) {
        vector_as<float, G, V, TAIL, E>(to, p, lane, n);
    } else {
        vector_as<T, G, V, TAIL, E>(to, p, lane, n);
    }
}

template <class T, int G, int V, bool TAIL, int E>
__device__ __forceinline__ void gate_of(float* to, const ResidualNorm& p, int64_t group, int lane)
{
    if (!p.gate) {
#pragma unroll
        for (int e = 0; e < E; ++e) to[e] = p.scale;
        return;
    }
    vector<T, G, V, TAIL, E>(to, from<T>(p.gate, p.gate_f32, group * p.gate_ld), p.gate_f32, lane, (int)p.N, 0.0f);
#pragma unroll
    for (int e = 0; e < E; ++e) to[e] *= p.scale;
}

// v, zeros behind the width, less its mean, which is left in `mean` (rms: as it is); the
// return value is 1 / sqrt(its mean square + eps)
template <int G, int V, int E, int WAVES>
__device__ __forceinline__ float centre(float* v, float& mean, bool rms, int lane, int n, float eps,
                                        float2 (&lds)[2][WAVES], int& turn)
{
    float s = 0.0f, unused = 0.0f;
    mean = 0.0f;
    if (!rms) {
#pragma unroll
        for (int e = 0; e < E; ++e) s += v[e];
        row_sums<G>(s, unused, lds[turn ^= 1]);
        mean = s / (float)n;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = column<G, V>(lane, e) < n ? v[e] - mean : 0.0f;
        s = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(v[e], v[e], s);
    row_sums<G>(s, unused, lds[turn ^= 1]);
    return 1.0f / sqrtf(s / (float)n + eps);
}

// h + g a in fp32, then in T (for halves the compiler has an instruction that leaves the
// first step out: another number in 1 of 16,000)
template <class T>
__device__ __forceinline__ T stored_sum(float g, float a, float h)
{
    float s = fmaf(g, a, h);
    if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(s));
    return (T)s;
}

template <class T, int G, int E, int V, bool TAIL, int THREADS>
__global__ __launch_bounds__(THREADS) void k_residual_norm(ResidualNorm p)
{
    constexpr int ROWS = THREADS / G;
    // (16 elements a thread: the vectors come from L2 for every row, there are no
    // registers for them)
    constexpr bool KEEP = E == 8;
    __shared__ float2 lds[2][THREADS / 64];
    int turn = 0;
    const int lane = threadIdx.x % G, n = (int)p.N;
    const int sub = __builtin_amdgcn_readfirstlane((int)threadIdx.x / G);
    // Workgroups go through the rows side by side, so that all of them read one stretch of
    // memory (32,768 x 4,096 by runs of neighbouring rows 218 us, so 204 us); where gates
    // would change every few rows, each takes a run.
    const int64_t rounds = (p.M + ROWS - 1) / ROWS;
    const bool runs = p.groups > 1 && p.length < 8 * (int64_t)gridDim.x * ROWS;
    const int64_t first = (runs ? rounds * blockIdx.x / gridDim.x : blockIdx.x) * ROWS;
    const int64_t last = runs ? min(p.M, rounds * (blockIdx.x + 1) / gridDim.x * ROWS) : p.M;
    const int64_t step = runs ? ROWS : (int64_t)gridDim.x * ROWS;
    float w[E], b[E], pw[E], pb[E], gate[E];
    auto pre_vectors = [&] {
        vector<T, G, V, TAIL, E>(w, p.weight, p.weight_f32, lane, n, 1.0f);
        vector<T, G, V, TAIL, E>(b, p.bias, p.weight_f32, lane, n, 0.0f);
    };
    auto post_vectors = [&] {
        vector<T, G, V, TAIL, E>(pw, p.post_weight, p.weight_f32, lane, n, 1.0f);
        vector<T, G, V, TAIL, E>(pb, p.post_bias, p.weight_f32, lane, n, 0.0f);
    };
    if constexpr (KEEP) {
        pre_vectors();
        post_vectors();
    }
    Held<T, E> nh{}, ny{};
    auto load = [&](int64_t i) {
        fetch<G, V, TAIL>(nh, static_cast<const T*>(p.h.p) + i * p.h.rs, lane, n);
        fetch<G, V, TAIL>(ny, static_cast<const T*>(p.y.p) + i * p.y.rs, lane, n);
    };
    if (first + sub < last) load(first + sub);
    int64_t group = -1, group_end = 0;
    // (the workgroup's rows go together: its barriers are everybody's)
    for (int64_t base = first; base < last; base += step) {
        const int64_t i = base + sub;
        const bool on = i < last;
        if (on && (!KEEP || i >= group_end)) {
            group = i / p.length;
            group_end = (group + 1) * p.length;
            gate_of<T, G, V, TAIL, E>(gate, p, group, lane);
        }
        float v[E], y[E], mean, rstd, post_mean, post_rstd;
        settle<G, V, TAIL>(nh, lane, n);
        settle<G, V, TAIL>(ny, lane, n);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = (float)nh.v[e];
            y[e] = (float)ny.v[e];
        }
        if (i + step < last) load(i + step);
        if (p.post) {
            post_rstd = centre<G, V, E>(y, post_mean, p.rms, lane, n, p.eps, lds, turn);
            if constexpr (!KEEP) post_vectors();
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(y[e] * post_rstd, pw[e], pb[e]);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[e] = (float)stored_sum<T>(gate[e], y[e], v[e]);
            if (column<G, V>(lane, e) >= n) v[e] = 0.0f;
        }
        if (on) put<G, V, TAIL, E>(static_cast<T*>(p.out) + i * p.out_ld, lane, n, v);
        rstd = centre<G, V, E>(v, mean, p.rms, lane, n, p.eps, lds, turn);
        if (!on) continue;
        if constexpr (!KEEP) pre_vectors();
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = fmaf(v[e] * rstd, w[e], b[e]);
        put<G, V, TAIL, E>(static_cast<T*>(p.normed) + i * p.normed_ld, lane, n, v);
        if (lane == 0) {
            if (p.mean) p.mean[i] = mean;
            if (p.rstd) p.rstd[i] = rstd;
            if (p.post && p.post_mean) p.post_mean[i] = post_mean;
            if (p.post && p.post_rstd) p.post_rstd[i] = post_rstd;
        }
    }
}

// The rows of a workgroup of the backward pass, ROWS at a time: whole groups [first,
// last), or a chunk of one group's, whose workgroups (SIDE) go through it side by side:
// 24,414 x 2,048 126 us, so 115 us.  From 512 threads on there is no register for a step.
template <int ROWS, bool SIDE>
struct Mine {
    int64_t first, last;
    int64_t begin, end;   // of the first group's rows
    typename std::conditional<SIDE, int64_t, std::integral_constant<int, ROWS>>::type step;
    __device__ __forceinline__ explicit Mine(const ResidualNorm& p, uint32_t part)
    {
        if (p.chunks) {
            first = part / (uint32_t)p.chunks;
            last = first + 1;
            const int64_t c = part % (uint32_t)p.chunks;
            if constexpr (SIDE) {
                begin = first * p.length + c * ROWS;
                end = (first + 1) * p.length;
                step = (int64_t)p.chunks * ROWS;
            } else {
                begin = first * p.length + p.length * c / p.chunks;
                end = first * p.length + p.length * (c + 1) / p.chunks;
            }
        } else {
            first = p.groups * part / p.parts;
            last = p.groups * (part + 1) / p.parts;
            begin = first * p.length;
            end = begin + p.length;
            if constexpr (SIDE) step = ROWS;
        }
    }
};

// g = dr + rstd (dn w - m1 - hh m2), dy = post ? post_rstd (d pw - m3 - yn m4) : d with d =
// scale gate g.  Each workgroup keeps its columns' sums over the rows in registers, of a
// group (g yn and g, from which the gate's and the post norm's gradients follow) and
// of all its rows; they meet at the end of a group, or in the partial sums.
//
// From 512 threads on, what a column has beside them lies in LDS, so that 128 registers do
// and two workgroups of 512 fit a CU: 32,768 x 4,096 with 184 registers 427 us, so 335 us.
// Smaller workgroups have registers for it (24,414 x 2,048 by LDS 136 us, so 129 us).
template <class T, int G, int V, bool TAIL, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 256 || sizeof(T) == 4 ? 2 : 4) void k_residual_norm_back(ResidualNorm p)
{
    constexpr int ROWS = THREADS / G, E = 8;
    static_assert(ROWS == 1 || THREADS == 256, "");
    __shared__ float2 lds[2][THREADS / 64];
    __shared__ float sums[ROWS == 1 ? 1 : G * E];
    // the weight, scale gate pw, and what the post norm's weight and bias have so far:
    // a thread's columns by four
    enum { WEIGHT, GATE, DPOST, DPOST_BIAS };
    __shared__ __attribute__((aligned(16))) float column_lds[4][2][G][4];
    constexpr bool HELD = THREADS == 256;
    float w[HELD ? E : 1], gate[HELD ? E : 1];
    int turn = 0;
    const int lane = threadIdx.x % G, n = (int)p.N;
    const int sub = __builtin_amdgcn_readfirstlane((int)threadIdx.x / G);
    auto to_lds = [&](int what, const float* v) {
#pragma unroll
        for (int e = 0; e < E; ++e) column_lds[what][e / 4][lane][e % 4] = v[e];
    };
    auto weight_of = [&](int e) { return HELD ? w[HELD ? e : 0] : column_lds[WEIGHT][e / 4][lane][e % 4]; };
    auto gate_of_column = [&](int e) { return HELD ? gate[HELD ? e : 0] : column_lds[GATE][e / 4][lane][e % 4]; };
    const Mine<ROWS, THREADS == 256> mine(p, blockIdx.x);
    float v[E];
    vector<T, G, V, TAIL, E>(v, p.weight, p.weight_f32, lane, n, 1.0f);
    if constexpr (HELD)
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = v[e];
    else
        to_lds(WEIGHT, v);
    if (sub == 0) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.0f;
        to_lds(DPOST, v);
        to_lds(DPOST_BIAS, v);
    }
    float dw[E] = {}, db[E] = {}, s1[E] = {}, s2[E] = {};
    Held<T, E> nh{}, ny{}, nn{}, nr{};
    auto load = [&](int64_t i) {
        fetch<G, V, TAIL>(nh, static_cast<const T*>(p.h.p) + i * p.h.rs, lane, n);
        fetch<G, V, TAIL>(ny, static_cast<const T*>(p.y.p) + i * p.y.rs, lane, n);
        fetch<G, V, TAIL>(nn, static_cast<const T*>(p.dn.p) + i * p.dn.rs, lane, n);
        if (p.dr.p) fetch<G, V, TAIL>(nr, static_cast<const T*>(p.dr.p) + i * p.dr.rs, lane, n);
    };
    // the sums of all threads of a column, in the first row's threads (a fixed order)
    auto over_rows = [&](float* v) {
        if constexpr (ROWS > 1) {
#pragma unroll 1
            for (int t = ROWS - 1; t >= 0; --t) {
                if (sub == t)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        // (by element, so that neighbouring lanes meet no bank twice)
                        const int at = e * G + lane;
                        v[e] = t == ROWS - 1 ? v[e] : sums[at] + v[e];
                        if (t > 0) sums[at] = v[e];
                    }
                __syncthreads();
            }
        }
    };
    float* const part = p.part + (int64_t)blockIdx.x * VECTORS * n;
    if (mine.begin + sub < mine.end) load(mine.begin + sub);
    int64_t begin = mine.begin, end = mine.end;
    for (int64_t group = mine.first; group < mine.last; ++group, begin = end, end += p.length) {
        gate_of<T, G, V, TAIL, E>(v, p, group, lane);
        {
            float pw[E];
            vector<T, G, V, TAIL, E>(pw, p.post ? p.post_weight : nullptr, p.weight_f32, lane, n, 1.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[e] *= pw[e];
                if constexpr (HELD) gate[e] = v[e];
            }
        }
        if constexpr (!HELD) to_lds(GATE, v);
        for (int64_t base = begin; base < end; base += mine.step) {
            const int64_t i = base + sub;
            const bool on = i < end;
            const float mean = on && !p.rms ? p.mean[i] : 0.0f, rstd = on ? p.rstd[i] : 0.0f;
            const float post_mean = on && p.post && !p.rms ? p.post_mean[i] : 0.0f;
            const float post_rstd = on && p.post ? p.post_rstd[i] : 0.0f;
            float hh[E], t[E], g[E], yn[E], m1 = 0.0f, m2 = 0.0f;
            settle<G, V, TAIL>(nh, lane, n);
            settle<G, V, TAIL>(ny, lane, n);
            settle<G, V, TAIL>(nn, lane, n);
            if (p.dr.p) settle<G, V, TAIL>(nr, lane, n);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // (beyond the width, and for a row beyond the last: 0)
                const bool in = on && column<G, V>(lane, e) < n;
                hh[e] = in ? ((float)nh.v[e] - mean) * rstd : 0.0f;
                const float d = in ? (float)nn.v[e] : 0.0f;
                dw[e] = fmaf(d, hh[e], dw[e]);
                db[e] += d;
                t[e] = d * weight_of(e);
                m1 += t[e];
                m2 = fmaf(t[e], hh[e], m2);
                g[e] = in && p.dr.p ? (float)nr.v[e] : 0.0f;
                yn[e] = in ? (float)ny.v[e] : 0.0f;
                if (p.post) yn[e] = in ? (yn[e] - post_mean) * post_rstd : 0.0f;
            }
            // the next row: of this group, or the next one's first
            const int64_t next = min(base + mine.step, end) + sub;
            const int64_t stop = base + mine.step < end ? end : group + 1 < mine.last ? end + p.length : 0;
            if (next < stop) load(next);
            row_sums<G>(m1, m2, lds[turn ^= 1]);
            m1 = p.rms ? 0.0f : m1 / (float)n;
            m2 /= (float)n;
            float m3 = 0.0f, m4 = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = on && column<G, V>(lane, e) < n;
                g[e] = in ? fmaf(rstd, t[e] - m1 - hh[e] * m2, g[e]) : 0.0f;
                s1[e] = fmaf(g[e], yn[e], s1[e]);
                s2[e] += g[e];
            }
            if (on && p.out) put<G, V, TAIL, E>(static_cast<T*>(p.out) + i * p.out_ld, lane, n, g);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] *= gate_of_column(e);
            if (p.post) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    m3 += g[e];
                    m4 = fmaf(g[e], yn[e], m4);
                }
                row_sums<G>(m3, m4, lds[turn ^= 1]);
                m3 = p.rms ? 0.0f : m3 / (float)n;
                m4 /= (float)n;
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = post_rstd * (g[e] - m3 - yn[e] * m4);
            }
            if (on && p.normed) put<G, V, TAIL, E>(static_cast<T*>(p.normed) + i * p.normed_ld, lane, n, g);
        }
        // the group's sums: the gate's gradient is scale (pw s1 + pb s2), the post norm's
        // weights' are scale gate s1 and scale gate s2
        over_rows(s1);
        over_rows(s2);
        if (sub == 0) {
            gate_of<T, G, V, TAIL, E>(v, p, group, lane);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float& dpost = column_lds[DPOST][e / 4][lane][e % 4];
                float& dpost_bias = column_lds[DPOST_BIAS][e / 4][lane][e % 4];
                dpost = fmaf(v[e], s1[e], dpost);
                dpost_bias = fmaf(v[e], s2[e], dpost_bias);
            }
            if (p.d_gate) {
                if (p.post) {
                    vector<T, G, V, TAIL, E>(v, p.post_weight, p.weight_f32, lane, n, 1.0f);
#pragma unroll
                    for (int e = 0; e < E; ++e) s1[e] *= v[e];
                    vector<T, G, V, TAIL, E>(v, p.post_bias, p.weight_f32, lane, n, 0.0f);
#pragma unroll
                    for (int e = 0; e < E; ++e) s1[e] = fmaf(v[e], s2[e], s1[e]);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) s1[e] *= p.scale;
                if (p.chunks)   // (one group, its gate's partial sums)
                    put<G, V, TAIL, E>(part + (int64_t)(VECTORS - 1) * n, lane, n, s1);
                else if (p.gate_f32)
                    put<G, V, TAIL, E>(static_cast<float*>(p.d_gate) + group * p.d_gate_ld, lane, n, s1);
                else
                    put<G, V, TAIL, E>(static_cast<T*>(p.d_gate) + group * p.d_gate_ld, lane, n, s1);
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) s1[e] = s2[e] = 0.0f;
    }
    auto leave = [&](bool wanted, float* v, int at) {
        if (!wanted) return;
        over_rows(v);
        if (sub == 0) put<G, V, TAIL, E>(part + (int64_t)at * n, lane, n, v);
    };
    leave(p.dweight, dw, 0);
    leave(p.dbias, db, 1);
    if (sub) return;
    for (int what : {DPOST, DPOST_BIAS}) {
        if (!(what == DPOST ? p.dpost_weight : p.dpost_bias)) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = column_lds[what][e / 4][lane][e % 4];
        put<G, V, TAIL, E>(part + (int64_t)(what - DPOST + 2) * n, lane, n, v);
    }
}

// Rows above 8,192: a workgroup's registers hold one row, and not its columns' sums
// (with both, 1,024 threads with 128 registers each, 3,051 x 16,384 took 720 us).  So the
// means of a row's elements come first...
template <class T, int V, bool TAIL>
__global__ __launch_bounds__(1024) void k_residual_norm_back_sums(ResidualNorm p)
{
    constexpr int G = 1024, E = 16;
    __shared__ float2 lds[2][16];
    int turn = 0;
    const int lane = threadIdx.x, n = (int)p.N;
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const int64_t group = i / p.length;
        Held<T, E> nh{}, ny{}, nn{}, nr{};
        float w[E];
        fetch<G, V, TAIL>(nh, static_cast<const T*>(p.h.p) + i * p.h.rs, lane, n);
        fetch<G, V, TAIL>(nn, static_cast<const T*>(p.dn.p) + i * p.dn.rs, lane, n);
        if (p.post) {
            fetch<G, V, TAIL>(ny, static_cast<const T*>(p.y.p) + i * p.y.rs, lane, n);
            if (p.dr.p) fetch<G, V, TAIL>(nr, static_cast<const T*>(p.dr.p) + i * p.dr.rs, lane, n);
        }
        const float mean = p.rms ? 0.0f : p.mean[i], rstd = p.rstd[i];
        settle<G, V, TAIL>(nh, lane, n);
        settle<G, V, TAIL>(nn, lane, n);
        vector<T, G, V, TAIL, E>(w, p.weight, p.weight_f32, lane, n, 1.0f);
        float m1 = 0.0f, m2 = 0.0f, m3 = 0.0f, m4 = 0.0f;
        auto normed = [&](int e) { return column<G, V>(lane, e) < n ? ((float)nh.v[e] - mean) * rstd : 0.0f; };
        auto above = [&](int e) { return (float)nn.v[e] * w[e]; };
#pragma unroll
        for (int e = 0; e < E; ++e) {
            m1 += above(e);
            m2 = fmaf(above(e), normed(e), m2);
        }
        row_sums<G>(m1, m2, lds[turn ^= 1]);
        m1 = p.rms ? 0.0f : m1 / (float)n;
        m2 /= (float)n;
        if (p.post) {
            const float post_mean = p.rms ? 0.0f : p.post_mean[i], post_rstd = p.post_rstd[i];
            settle<G, V, TAIL>(ny, lane, n);
            settle<G, V, TAIL>(nr, lane, n);
            float g[E];
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = fmaf(rstd, above(e) - m1 - normed(e) * m2, (float)nr.v[e]);
            float by[E];
            gate_of<T, G, V, TAIL, E>(by, p, group, lane);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] *= by[e];
            vector<T, G, V, TAIL, E>(by, p.post_weight, p.weight_f32, lane, n, 1.0f);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = column<G, V>(lane, e) < n;
                const float d = in ? g[e] * by[e] : 0.0f;
                m3 += d;
                m4 = fmaf(d, in ? ((float)ny.v[e] - post_mean) * post_rstd : 0.0f, m4);
            }
            row_sums<G>(m3, m4, lds[turn ^= 1]);
            m3 = p.rms ? 0.0f : m3 / (float)n;
            m4 /= (float)n;
        }
        if (lane == 0) {
            float* m = p.rows + i * 4;
            m[0] = m1, m[1] = m2, m[2] = m3, m[3] = m4;
        }
    }
}

// ... and with them every element stands for itself: 2,048 columns a workgroup, which
// walks rows, sums up and writes over what it alone has read.
template <class T, int V, bool TAIL>
__global__ __launch_bounds__(256) void k_residual_norm_back_walk(ResidualNorm p)
{
    constexpr int G = 256, E = 8;
    // (in vectors, lanes are counted through all workgroups: a row's last eight are whole)
    const int64_t c0 = V == 8 ? 0 : (int64_t)blockIdx.x * (G * E);
    const int lane = (int)threadIdx.x + (V == 8 ? (int)blockIdx.x * G : 0), n = (int)(p.N - c0);
    const Mine<1, true> mine(p, blockIdx.y);
    auto columns_of = [&](const void* v) { return v ? from<T>(v, p.weight_f32, c0) : nullptr; };
    float w[E], pw[E], gate[E];
    vector<T, G, V, TAIL, E>(w, columns_of(p.weight), p.weight_f32, lane, n, 1.0f);
    vector<T, G, V, TAIL, E>(pw, columns_of(p.post ? p.post_weight : nullptr), p.weight_f32, lane, n, 1.0f);
    float dw[E] = {}, db[E] = {}, dpw[E] = {}, dpb[E] = {}, s1[E] = {}, s2[E] = {};
    Held<T, E> nh{}, ny{}, nn{}, nr{};
    auto load = [&](int64_t i) {
        fetch<G, V, TAIL>(nh, static_cast<const T*>(p.h.p) + i * p.h.rs + c0, lane, n);
        fetch<G, V, TAIL>(ny, static_cast<const T*>(p.y.p) + i * p.y.rs + c0, lane, n);
        fetch<G, V, TAIL>(nn, static_cast<const T*>(p.dn.p) + i * p.dn.rs + c0, lane, n);
        if (p.dr.p) fetch<G, V, TAIL>(nr, static_cast<const T*>(p.dr.p) + i * p.dr.rs + c0, lane, n);
    };
    float* const part = p.part + (int64_t)blockIdx.y * VECTORS * p.N + c0;
    int64_t begin = mine.begin, end = mine.end;
    const int64_t last = p.chunks ? end : mine.last * p.length;
    if (begin < last) load(begin);
    for (int64_t group = mine.first; group < mine.last; ++group, begin = end, end += p.length) {
        ResidualNorm q{};
        q.gate = p.gate ? from<T>(p.gate, p.gate_f32, c0) : nullptr;
        q.gate_ld = p.gate_ld;
        q.gate_f32 = p.gate_f32;
        q.scale = p.scale;
        q.N = n;
        gate_of<T, G, V, TAIL, E>(gate, q, group, lane);
        for (int64_t i = begin; i < end; i += mine.step) {
            const float mean = p.rms ? 0.0f : p.mean[i], rstd = p.rstd[i];
            const float post_mean = p.post && !p.rms ? p.post_mean[i] : 0.0f;
            const float post_rstd = p.post ? p.post_rstd[i] : 1.0f;
            const float* m = p.rows + i * 4;
            const float m1 = m[0], m2 = m[1], m3 = m[2], m4 = m[3];
            settle<G, V, TAIL>(nh, lane, n);
            settle<G, V, TAIL>(ny, lane, n);
            settle<G, V, TAIL>(nn, lane, n);
            if (p.dr.p) settle<G, V, TAIL>(nr, lane, n);
            float g[E], yn[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float hh = ((float)nh.v[e] - mean) * rstd, d = (float)nn.v[e];
                dw[e] = fmaf(d, hh, dw[e]);
                db[e] += d;
                g[e] = fmaf(rstd, d * w[e] - m1 - hh * m2, p.dr.p ? (float)nr.v[e] : 0.0f);
                yn[e] = p.post ? ((float)ny.v[e] - post_mean) * post_rstd : (float)ny.v[e];
            }
            if (i + mine.step < last) load(i + mine.step);
            if (p.out) put<G, V, TAIL, E>(static_cast<T*>(p.out) + i * p.out_ld + c0, lane, n, g);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                s1[e] = fmaf(g[e], yn[e], s1[e]);
                s2[e] += g[e];
                g[e] *= gate[e];
                if (p.post) g[e] = post_rstd * (g[e] * pw[e] - m3 - yn[e] * m4);
            }
            if (p.normed) put<G, V, TAIL, E>(static_cast<T*>(p.normed) + i * p.normed_ld + c0, lane, n, g);
        }
        float pb[E];
        vector<T, G, V, TAIL, E>(pb, columns_of(p.post_bias), p.weight_f32, lane, n, 0.0f);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            dpw[e] = fmaf(gate[e], s1[e], dpw[e]);
            dpb[e] = fmaf(gate[e], s2[e], dpb[e]);
            s1[e] = p.scale * (p.post ? fmaf(pw[e], s1[e], pb[e] * s2[e]) : s1[e]);
            s2[e] = 0.0f;
        }
        if (p.d_gate) {
            if (p.chunks)
                put<G, V, TAIL, E>(part + (VECTORS - 1) * p.N, lane, n, s1);
            else if (p.gate_f32)
                put<G, V, TAIL, E>(static_cast<float*>(p.d_gate) + group * p.d_gate_ld + c0, lane, n, s1);
            else
                put<G, V, TAIL, E>(static_cast<T*>(p.d_gate) + group * p.d_gate_ld + c0, lane, n, s1);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) s1[e] = 0.0f;
    }
    if (p.dweight) put<G, V, TAIL, E>(part, lane, n, dw);
    if (p.dbias) put<G, V, TAIL, E>(part + p.N, lane, n, db);
    if (p.dpost_weight) put<G, V, TAIL, E>(part + 2 * p.N, lane, n, dpw);
    if (p.dpost_bias) put<G, V, TAIL, E>(part + 3 * p.N, lane, n, dpb);
}

// The workgroups' sums added up: 4 LANES columns a workgroup, by LANES threads of 4
// neighbours, ROWS times with 8 loads each in flight (widths up to 2,048 by 8 lanes: for
// 1,021 of them 8 workgroups of 32 lanes a vector took 7.9 us).  blockIdx.y: a vector's
// sums over all parts, or from the fifth on a group's gate over its chunks.
template <class T, int LANES>
__global__ __launch_bounds__(1024) void k_residual_norm_columns(ResidualNorm p)
{
    constexpr int U = 8, COLUMNS = 4 * LANES, ROWS = 1024 / LANES;
    typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ float sums[ROWS][COLUMNS], some[ROWS / 4][COLUMNS];
    const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES, n = (int)p.N;
    const int c0 = (int)blockIdx.x * COLUMNS, own = c0 + lane * 4;
    const int j = max(0, min(own, n - 4));   // (the last thread's four end with the width)
    const int vector = min((int)blockIdx.y, VECTORS - 1);
    void* const of[4] = {p.dweight, p.dbias, p.dpost_weight, p.dpost_bias};
    const int64_t group = (int64_t)blockIdx.y - (VECTORS - 1);
    const bool gate = group >= 0;
    if (!gate && !of[vector & 3]) return;
    const int first = gate ? (int)group * p.chunks : 0, count = gate ? p.chunks : p.parts;
    const float* part = p.part + ((int64_t)first * VECTORS + vector) * n + j;
    Four t[U] = {};
    if (own < n && n >= 4) {
        for (int k = row; k < count; k += ROWS * U)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + ROWS * u < count) t[u] += *(const Four*)(part + (int64_t)(k + ROWS * u) * VECTORS * n);
    } else if (own < n) {
        for (int k = row; k < count; k += ROWS)
            for (int e = 0; e < n; ++e) t[0][e] += part[(int64_t)k * VECTORS * n + e];
    }
#pragma unroll
    for (int d = U / 2; d > 0; d /= 2)
#pragma unroll
        for (int u = 0; u < d; ++u) t[u] += t[u + d];
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (j + e >= own && j + e < n) sums[row][j + e - c0] = t[0][e];
    __syncthreads();
    {
        const int c = threadIdx.x % COLUMNS, r = threadIdx.x / COLUMNS;
        some[r][c] = (sums[4 * r][c] + sums[4 * r + 1][c]) + (sums[4 * r + 2][c] + sums[4 * r + 3][c]);
    }
    __syncthreads();
    const int column = c0 + (int)threadIdx.x;
    if (threadIdx.x >= COLUMNS || column >= n) return;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < ROWS / 4; ++k) s += some[k][threadIdx.x];
    void* const to = gate ? p.d_gate : of[vector & 3];
    const int64_t at = gate ? group * p.d_gate_ld + column : column;
    if (gate ? p.gate_f32 : p.weight_f32)
        static_cast<float*>(to)[at] = s;
    else
        static_cast<T*>(to)[at] = (T)s;
}

// ------------------------------------------------- rows that no registers hold
// Too wide or narrow, or with elements that are not neighbours: read element by element, two or
// three times, the later ones from L2.

template <class T>
__device__ __forceinline__ float at(const Strided& m, int64_t i, int64_t j)
{
    return (float)static_cast<const T*>(m.p)[i * m.rs + j * m.cs];
}
template <class T>
__device__ __forceinline__ float at(const void* v, bool f32, int64_t j, float missing)
{
    return !v ? missing : f32 ? static_cast<const float*>(v)[j] : (float)static_cast<const T*>(v)[j];
}
template <class T>
__device__ __forceinline__ float gate_at(const ResidualNorm& p, int64_t group, int64_t j)
{
    if (!p.gate) return p.scale;
    return p.scale * (p.gate_f32 ? static_cast<const float*>(p.gate)[group * p.gate_ld + j]
                                 : (float)static_cast<const T*>(p.gate)[group * p.gate_ld + j]);
}

template <class F>
__device__ __forceinline__ float centre_wide(F value, int64_t n, bool rms, float eps, float& mean,
                                             float2 (&lds)[2][16], int& turn)
{
    float s = 0.0f, unused = 0.0f;
    mean = 0.0f;
    if (!rms) {
        for (int64_t j = threadIdx.x; j < n; j += 1024) s += value(j);
        row_sums<1024>(s, unused, lds[turn ^= 1]);
        mean = s / (float)n;
        s = 0.0f;
    }
    for (int64_t j = threadIdx.x; j < n; j += 1024) {
        const float d = value(j) - mean;
        s = fmaf(d, d, s);
    }
    row_sums<1024>(s, unused, lds[turn ^= 1]);
    return 1.0f / sqrtf(s / (float)n + eps);
}

template <class T>
__global__ __launch_bounds__(1024) void k_residual_norm_wide(ResidualNorm p)
{
    __shared__ float2 lds[2][16];
    int turn = 0;
    const int64_t n = p.N;
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const int64_t group = i / p.length;
        float mean, rstd, post_mean = 0.0f, post_rstd = 1.0f;
        if (p.post)
            post_rstd = centre_wide([&](int64_t j) { return at<T>(p.y, i, j); }, n, p.rms, p.eps, post_mean, lds, turn);
        T* out = static_cast<T*>(p.out) + i * p.out_ld;
        for (int64_t j = threadIdx.x; j < n; j += 1024) {
            float y = at<T>(p.y, i, j);
            if (p.post)
                y = fmaf((y - post_mean) * post_rstd, at<T>(p.post_weight, p.weight_f32, j, 1.0f), at<T>(p.post_bias, p.weight_f32, j, 0.0f));
            out[j] = stored_sum<T>(gate_at<T>(p, group, j), y, at<T>(p.h, i, j));
        }
        // (each thread reads what it wrote itself)
        rstd = centre_wide([&](int64_t j) { return (float)out[j]; }, n, p.rms, p.eps, mean, lds, turn);
        for (int64_t j = threadIdx.x; j < n; j += 1024)
            static_cast<T*>(p.normed)[i * p.normed_ld + j] =
                (T)fmaf(((float)out[j] - mean) * rstd, at<T>(p.weight, p.weight_f32, j, 1.0f), at<T>(p.bias, p.weight_f32, j, 0.0f));
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[i] = mean;
            if (p.rstd) p.rstd[i] = rstd;
            if (p.post && p.post_mean) p.post_mean[i] = post_mean;
            if (p.post && p.post_rstd) p.post_rstd[i] = post_rstd;
        }
    }
}

// an element's normed row, its stream's gradient and its normed block output
template <class T>
struct Element {
    float hh, dn, g, yn;
    __device__ __forceinline__ Element(const ResidualNorm& p, int64_t i, int64_t j, float m1, float m2)
    {
        const float rstd = p.rstd[i];
        hh = (at<T>(p.h, i, j) - (p.rms ? 0.0f : p.mean[i])) * rstd;
        dn = at<T>(p.dn, i, j);
        g = fmaf(rstd, dn * at<T>(p.weight, p.weight_f32, j, 1.0f) - m1 - hh * m2, p.dr.p ? at<T>(p.dr, i, j) : 0.0f);
        yn = at<T>(p.y, i, j);
        if (p.post) yn = (yn - (p.rms ? 0.0f : p.post_mean[i])) * p.post_rstd[i];
    }
};

// the means that a row's elements need of their neighbours
template <class T>
__global__ __launch_bounds__(1024) void k_residual_norm_back_means(ResidualNorm p)
{
    __shared__ float2 lds[2][16];
    int turn = 0;
    const int64_t n = p.N;
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const int64_t group = i / p.length;
        float m1 = 0.0f, m2 = 0.0f, m3 = 0.0f, m4 = 0.0f;
        for (int64_t j = threadIdx.x; j < n; j += 1024) {
            const Element<T> x(p, i, j, 0.0f, 0.0f);
            const float t = x.dn * at<T>(p.weight, p.weight_f32, j, 1.0f);
            m1 += t;
            m2 = fmaf(t, x.hh, m2);
        }
        row_sums<1024>(m1, m2, lds[turn ^= 1]);
        m1 = p.rms ? 0.0f : m1 / (float)n;
        m2 /= (float)n;
        if (p.post) {
            for (int64_t j = threadIdx.x; j < n; j += 1024) {
                const Element<T> x(p, i, j, m1, m2);
                const float d = x.g * gate_at<T>(p, group, j) * at<T>(p.post_weight, p.weight_f32, j, 1.0f);
                m3 += d;
                m4 = fmaf(d, x.yn, m4);
            }
            row_sums<1024>(m3, m4, lds[turn ^= 1]);
            m3 = p.rms ? 0.0f : m3 / (float)n;
            m4 /= (float)n;
        }
        if (threadIdx.x == 0) {
            float* m = p.rows + i * 4;
            m[0] = m1, m[1] = m2, m[2] = m3, m[3] = m4;
        }
    }
}

// the sums over the rows, by column...
template <class T>
__global__ __launch_bounds__(256) void k_residual_norm_back_wide_columns(ResidualNorm p)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x, n = p.N;
    if (j >= n) return;
    for (int64_t part = blockIdx.y; part < p.parts; part += gridDim.y) {
        const Mine<1, true> mine(p, (uint32_t)part);
        const float pw = at<T>(p.post_weight, p.weight_f32, j, 1.0f), pb = at<T>(p.post_bias, p.weight_f32, j, 0.0f);
        float dw = 0.0f, db = 0.0f, dpw = 0.0f, dpb = 0.0f, dg = 0.0f;
        int64_t begin = mine.begin, end = mine.end;
        for (int64_t group = mine.first; group < mine.last; ++group, begin = end, end += p.length) {
            const float gate = gate_at<T>(p, group, j);
            float s1 = 0.0f, s2 = 0.0f;
            for (int64_t i = begin; i < end; i += mine.step) {
                const Element<T> x(p, i, j, p.rows[i * 4], p.rows[i * 4 + 1]);
                dw = fmaf(x.dn, x.hh, dw);
                db += x.dn;
                s1 = fmaf(x.g, x.yn, s1);
                s2 += x.g;
            }
            dpw = fmaf(gate, s1, dpw);
            dpb = fmaf(gate, s2, dpb);
            dg = p.scale * (p.post ? fmaf(pw, s1, pb * s2) : s1);
            if (p.d_gate && !p.chunks) {
                if (p.gate_f32)
                    static_cast<float*>(p.d_gate)[group * p.d_gate_ld + j] = dg;
                else
                    static_cast<T*>(p.d_gate)[group * p.d_gate_ld + j] = (T)dg;
            }
        }
        float* to = p.part + part * VECTORS * n + j;
        to[0] = dw, to[n] = db, to[2 * n] = dpw, to[3 * n] = dpb, to[4 * n] = dg;
    }
}

// ... and the rows' gradients, after them (they may be written over what was read)
template <class T>
__global__ __launch_bounds__(1024) void k_residual_norm_back_wide(ResidualNorm p)
{
    for (int64_t i = blockIdx.x; i < p.M; i += gridDim.x) {
        const int64_t group = i / p.length;
        const float* m = p.rows + i * 4;
        for (int64_t j = threadIdx.x; j < p.N; j += 1024) {
            const Element<T> x(p, i, j, m[0], m[1]);
            float d = x.g * gate_at<T>(p, group, j);
            if (p.post) d = p.post_rstd[i] * (d * at<T>(p.post_weight, p.weight_f32, j, 1.0f) - m[2] - x.yn * m[3]);
            if (p.out) static_cast<T*>(p.out)[i * p.out_ld + j] = (T)x.g;
            if (p.normed) static_cast<T*>(p.normed)[i * p.normed_ld + j] = (T)d;
        }
    }
}

// ------------------------------------------------------------------------ launches

bool neighbours(const Strided& m, int64_t n) { return !m.p || n <= 1 || m.cs == 1; }

// threads of a row of width n, and rows that a workgroup takes at a time (48,000 x 1,024
// backward by 256 threads, half of them idle, 168 us, by 128 130 us)
int threads_of(int64_t n) { return n <= 512 ? 64 : n <= 1024 ? 128 : n <= 2048 ? 256 : n <= 4096 ? 512 : 1024; }
int rows_at_once(int64_t n) { return n <= 512 ? 4 : n <= 1024 ? 2 : 1; }

template <class T, int V, bool TAIL>
void forward_held(const ResidualNorm& p, hipStream_t stream)
{
    const int64_t rounds = (p.M + rows_at_once(p.N) - 1) / rows_at_once(p.N);
    const int G = threads_of(p.N);
    const int64_t most = G == 1024 ? 512 : G == 512 ? 1024 : 2048;
    const dim3 grid((unsigned)std::min(rounds, most));
    if (G == 64)
        hipLaunchKernelGGL((k_residual_norm<T, 64, 8, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 128)
        hipLaunchKernelGGL((k_residual_norm<T, 128, 8, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 256)
        hipLaunchKernelGGL((k_residual_norm<T, 256, 8, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 512)
        hipLaunchKernelGGL((k_residual_norm<T, 512, 8, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else if (p.N <= 8192)
        hipLaunchKernelGGL((k_residual_norm<T, 1024, 8, V, TAIL, 1024>), grid, dim3(1024), 0, stream, p);
    else
        hipLaunchKernelGGL((k_residual_norm<T, 1024, 16, V, TAIL, 1024>), grid, dim3(1024), 0, stream, p);
}

template <class T, int V, bool TAIL>
void backward_held(const ResidualNorm& p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.parts);
    // (groups of fewer rows than a workgroup would take at a time: 65,536 x 512 with a gate
    // for each row 807 us, so 557 us; a row's columns have a thread each also where there
    // are no rows, and sums of zero are left)
    const int G = p.length < rows_at_once(p.N) ? std::max(256, threads_of(p.N)) : threads_of(p.N);
    if (p.N > MOST_SUMMED) {
        if (p.M > 0)
            hipLaunchKernelGGL((k_residual_norm_back_sums<T, V, TAIL>), dim3((unsigned)std::min<int64_t>(p.M, 1024)),
                               dim3(1024), 0, stream, p);
        hipLaunchKernelGGL((k_residual_norm_back_walk<T, V, TAIL>),
                           dim3((unsigned)((p.N + 2047) / 2048), (unsigned)p.parts), dim3(256), 0, stream, p);
        return;
    }
    if (G == 64)
        hipLaunchKernelGGL((k_residual_norm_back<T, 64, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 128)
        hipLaunchKernelGGL((k_residual_norm_back<T, 128, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 256)
        hipLaunchKernelGGL((k_residual_norm_back<T, 256, V, TAIL, 256>), grid, dim3(256), 0, stream, p);
    else if (G == 512)
        hipLaunchKernelGGL((k_residual_norm_back<T, 512, V, TAIL, 512>), grid, dim3(512), 0, stream, p);
    else
        hipLaunchKernelGGL((k_residual_norm_back<T, 1024, V, TAIL, 1024>), grid, dim3(1024), 0, stream, p);
}

// workgroups that walk M rows, one at a time each
dim3 wide_grid(int64_t M) { return dim3((unsigned)std::min<int64_t>(M, 1 << 16)); }

bool wide(const ResidualNorm& p)
{
    return p.N < 8 || p.N > MOST_HELD || !neighbours(p.h, p.N) || !neighbours(p.y, p.N) || !neighbours(p.dn, p.N) ||
           !neighbours(p.dr, p.N);
}

template <class T>
hipError_t forward(const ResidualNorm& p, hipStream_t stream)
{
    if (wide(p))
        hipLaunchKernelGGL((k_residual_norm_wide<T>), wide_grid(p.M), dim3(1024), 0, stream, p);
    else if (p.N % 8 == 0)
        forward_held<T, 8, false>(p, stream);
    else
        forward_held<T, sizeof(T) == 4 ? 1 : 8, sizeof(T) == 2>(p, stream);
    return hipGetLastError();
}

template <class T>
hipError_t backward(const ResidualNorm& p, hipStream_t stream)
{
    const bool sums = p.dweight || p.dbias || p.dpost_weight || p.dpost_bias || p.d_gate;
    if (!sums && !p.out && !p.normed) return hipSuccess;
    const bool by_element = wide(p);
    hipError_t e = hipSuccess;
    if (by_element) {
        if (p.M > 0)
            hipLaunchKernelGGL((k_residual_norm_back_means<T>), wide_grid(p.M), dim3(1024), 0, stream, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (sums)
            hipLaunchKernelGGL((k_residual_norm_back_wide_columns<T>),
                               dim3((unsigned)((p.N + 255) / 256), (unsigned)std::min(p.parts, 1024)), dim3(256), 0,
                               stream, p);
    } else if (p.N % 8 == 0) {
        backward_held<T, 8, false>(p, stream);
    } else {
        backward_held<T, sizeof(T) == 4 ? 1 : 8, sizeof(T) == 2>(p, stream);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (sums) {
        const int64_t jobs = VECTORS - 1 + (p.d_gate && p.chunks ? p.groups : 0);
        if (p.N <= 2048)
            hipLaunchKernelGGL((k_residual_norm_columns<T, 8>), dim3((unsigned)((p.N + 31) / 32), (unsigned)jobs),
                               dim3(1024), 0, stream, p);
        else
            hipLaunchKernelGGL((k_residual_norm_columns<T, 32>), dim3((unsigned)((p.N + 127) / 128), (unsigned)jobs),
                               dim3(1024), 0, stream, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (by_element && p.M > 0 && (p.out || p.normed))
        hipLaunchKernelGGL((k_residual_norm_back_wide<T>), wide_grid(p.M), dim3(1024), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

// A group of many rows is cut into chunks, each a workgroup; many groups are dealt out
// whole, so that a workgroup writes their gates' gradients itself.
RowParts residual_norm_parts(const ResidualNorm& p)
{
    const bool by_element = wide(p);
    const int64_t rows = by_element ? 1 : rows_at_once(p.N);
    const int64_t most = by_element || p.N <= 4096 ? 512 : p.N <= MOST_SUMMED ? 256 : 128;
    if (p.M == 0) return {1, 0};
    if (2 * p.groups > most) return {(int)std::min(most, p.groups), 0};
    const int64_t rounds = (p.length + rows - 1) / rows;
    const int64_t chunks = std::max<int64_t>(1, std::min(most / p.groups, rounds));
    return {(int)(chunks * p.groups), (int)chunks};
}

hipError_t launch_residual_norm(const ResidualNorm& p, int dtype, hipStream_t stream)
{
    if (p.M == 0) return hipSuccess;
    return dtype == MAG_F32 ? forward<float>(p, stream) : dtype == MAG_F16 ? forward<f16>(p, stream) : forward<bf16>(p, stream);
}

hipError_t launch_residual_norm_backward(const ResidualNorm& p, int dtype, hipStream_t stream)
{
    return dtype == MAG_F32   ? backward<float>(p, stream)
           : dtype == MAG_F16 ? backward<f16>(p, stream)
                              : backward<bf16>(p, stream);
}

}  // namespace mag
