// rows.hpp -- rows of a matrix in the registers of a group of threads, and what the
// threads of a row add up.
#pragma once

#include "block.hpp"

namespace mag {

// The G threads of a row hold E elements of it each: V neighbours, G V further on the
// next V, and so on.  V is 8 (the hardware takes vector loads and stores at any
// element); TAIL: the width is no multiple of 8, and one thread has elements of fewer.
// fp32 rows of such widths go element by element, V = 1: 64 lanes' 4 bytes are
// whole lines at once (13,399 x 791: 16 us, in vectors 20 us; bfloat16, 3,739 x
// 11,918 backward: 94 us in vectors, 201 us by element).
template <class T, int E>
struct Held {
    T v[E];
};

template <int G, int V>
__device__ __forceinline__ int column(int lane, int e)
{
    return (e / V * G + lane) * V + e % V;
}

template <int G, int V, bool TAIL, class T, int E>
__device__ __forceinline__ void get(Held<T, E>& r, const T* row, int lane, int n)
{
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
        const int j = (c * G + lane) * V;
        T* to = r.v + c * V;
        if (j + (TAIL ? V - 1 : 0) < n) {
            // (at once: by memcpy, what else TAIL loads comes into the same registers by
            // copies, ten too many for two workgroups of the backward pass a CU)
            typedef T Piece __attribute__((ext_vector_type(TAIL ? V : 1), aligned(sizeof(T))));
            if constexpr (TAIL) {
                const Piece t = *(const Piece*)(row + j);
#pragma unroll
                for (int i = 0; i < V; ++i) to[i] = t[i];
            } else {
                __builtin_memcpy(to, row + j, V * sizeof(T));
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) to[i] = (T)0.0f;
            if (TAIL && j < n)
#pragma unroll
                for (int i = 0; i < V - 1; ++i)
                    if (j + i < n) to[i] = row[j + i];
        }
    }
}

// The same, of rows of at least 8, in two steps without a wait between them: fetch() has the thread at a row's
// end load the eight elements that end there, settle() moves them down to their
// places (zeros behind).  By element, each of the seven is a load of its own that is
// waited for: 48,000 x 1,021 forward 188 us, so 95 us (two-byte numbers).
template <int G, int V, bool TAIL, class T, int E>
__device__ __forceinline__ void fetch(Held<T, E>& r, const T* row, int lane, int n)
{
    if constexpr (!TAIL) {
        get<G, V, TAIL>(r, row, lane, n);
    } else {
#pragma unroll
        for (int c = 0; c < E / V; ++c) {
            typedef T Piece __attribute__((ext_vector_type(V), aligned(sizeof(T))));
            const Piece t = *(const Piece*)(row + min((c * G + lane) * V, n - V));
#pragma unroll
            for (int i = 0; i < V; ++i) r.v[c * V + i] = t[i];
        }
    }
}

// words w, moved down by so many bytes (whole elements of SIZE; zeros behind)
template <int SIZE, int WORDS>
__device__ __forceinline__ void move_down(uint32_t* w, uint32_t bytes)
{
    if constexpr (SIZE < 4)
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            w[i] = __builtin_amdgcn_alignbyte(i + 1 < WORDS ? w[i + 1] : 0u, w[i], bytes & (4 - SIZE));
#pragma unroll
    for (int d = 1; d <= WORDS; d *= 2)
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const uint32_t from = i + d < WORDS ? w[i + d] : 0u;
            w[i] = bytes & (4 * d) ? from : w[i];
        }
}

template <int G, int V, bool TAIL, class T, int E>
__device__ __forceinline__ void settle(Held<T, E>& r, int lane, int n)
{
    if constexpr (TAIL) {
        static_assert(V == 8, "");
#pragma unroll
        for (int c = 0; c < E / V; ++c) {
            const int by = (c * G + lane) * V - (n - V);   // places to move, from 8 on: none is left
            if (__builtin_amdgcn_ballot_w64(by > 0) == 0) continue;
            // (in words: single halves would take a register each)
            uint32_t w[V * sizeof(T) / 4];
            __builtin_memcpy(w, r.v + c * V, sizeof w);
            move_down<sizeof(T), V * sizeof(T) / 4>(w, by <= 0 ? 0 : by >= V ? V * sizeof(T) : by * sizeof(T));
            __builtin_memcpy(r.v + c * V, w, sizeof w);
        }
    }
}

template <int G, int V, bool TAIL, int E, class T>
__device__ __forceinline__ void put(T* row, int lane, int n, const float* v)
{
#pragma unroll
    for (int c = 0; c < E / V; ++c) {
        const int j = (c * G + lane) * V;
        T o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = (T)v[c * V + i];
        if (j + (TAIL ? V - 1 : 0) < n) {
            __builtin_memcpy(row + j, o, V * sizeof(T));
        } else if (TAIL && j < n) {
#pragma unroll
            for (int i = 0; i < V - 1; ++i)
                if (j + i < n) row[j + i] = o[i];
        }
    }
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// The sums of a and b over the G threads of a row.  lds: two floats a wave,
// another place from one call to the next of the same row and the next row's
// first (one barrier a call: a place is written again two calls later).
template <int G>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* lds)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (G > 64) {
        constexpr int WAVES = G / 64;
        const int wave = threadIdx.x / 64, first = wave / WAVES * WAVES;
        if (threadIdx.x % 64 == 0) lds[wave] = float2{a, b};
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 s = lds[first + w];
            a += s.x;
            b += s.y;
        }
    }
}

}  // namespace mag
