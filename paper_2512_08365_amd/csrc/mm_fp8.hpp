// mm_fp8.hpp -- the matrix-core tile product of 8-bit operands with scaled blocks.
#pragma once

#include "fp8.hpp"
#include "mm.hpp"

namespace mag {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;

// D = A B^T of a block's 128 k: A's row lane % 16, its 32 bytes any k that B's row of the
// same lane has too; a lane gets rows 4 (lane / 16) on of A, row lane % 16 of B
template <int FA, int FB>
__device__ __forceinline__ f32x4 mfma8(i32x8 a, i32x8 b)
{
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, zero, FA == MAG_E5M2, FB == MAG_E5M2, 0, 0, 0, 0);
}

// out[r][s]: SIDE x SIDE of them a tile, WR x WS waves.  A step is a block of 128 k:
// what the instruction sums of a block is multiplied by the operands' scales and
// added to the sums in registers, so there is one multiplication and addition a
// sum and step beside the products: half of the matrix cores' time, and beside it as
// long as the products do not wait for their results.  Scales for each s cost a
// multiplication more, of the scales with each other: sums times one of them and then
// the other would leave fp32's range where a tiny one meets a huge one.  Scales that lie
// by columns, as quantization leaves them, are read as a tile's rows beside one
// another; by rows each is in a line of its own (16,384 x 8,192 by 4,096, four sets of
// operands in turn: 620 us, by rows 750).
template <int SIDE_, int WR_, int WS_>
struct Shape8 {
    static constexpr int SIDE = SIDE_, WR = WR_, WS = WS_;
    static constexpr int THREADS = 64 * WR * WS;
    static constexpr int RF = SIDE / WR / 16, SF = SIDE / WS / 16;   // a wave's rows and columns, in 16s
    static constexpr int BYTES = SIDE * FP8_BLOCK;
};

// Rows of an operand, a step of 128 bytes of them at a time, on their way to LDS without
// registers in chunks of 16 bytes: chunk c of row r sits at c ^ (r & 7), so that 8 rows'
// chunks of one k cover all banks.  A thread's chunks are THREADS / 8 rows apart: one
// register says where they all lie.  Chunks of rows behind the last one, and those that
// do not end inside the rows, are not read: zeros take their place.
template <class Sh>
struct Rows8 {
    static constexpr int APART = Sh::THREADS / 8, LOADS = Sh::SIDE / APART;
    const char* base;   // of the tile's first row and the step's first k
    int ld, rows;       // rows of the tile that there are
    uint32_t off;

    static __device__ __forceinline__ int line() { return (int)threadIdx.x / 8; }
    static __device__ __forceinline__ int first_k() { return (((int)threadIdx.x & 7) ^ (line() & 7)) * 16; }
    __device__ __forceinline__ void init(const uint8_t* p, int64_t distance, int64_t row, int64_t rows_, int64_t k)
    {
        ld = (int)distance;
        base = (const char*)p + row * distance + k;
        rows = (int)min((int64_t)Sh::SIDE, rows_ - row);
        off = (uint32_t)(line() * ld + first_k());
    }
    // k_left: of the rows from the step's first k on
    __device__ __forceinline__ void load(char* lds, int k_left, int wave)
    {
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7fffffff, 0x00020000);
        const int at = first_k() + 16 <= k_left ? line() : Sh::SIDE;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(lds + (i * Sh::THREADS + wave * 64) * 16), 16,
                at < rows - i * APART ? off : NOWHERE, i * APART * ld, 0, 0);
        base += FP8_BLOCK;
    }
};

// Eight neighbours of N column fragments each (32 columns apart), as they are stored.
template <int N, class T>
struct Added {
    typedef T Eight __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    Eight v[N ? N : 1];
    // from p + at + s on, where there are eight (p NULL: none)
    __device__ __forceinline__ void load(const Epilogue& e, const void* p, int64_t at, int64_t s, int64_t S)
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (p && e.vec && s + 32 * j + 8 <= S) v[j] = *(const Eight*)(static_cast<const T*>(p) + at + s + 32 * j);
    }
    __device__ __forceinline__ void add(int j, float* z) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += (float)v[j][i];
    }
};

template <class Sh, int FA, int FB, bool BY_ROW, class TO, bool PARTIAL, class Arrays>
__device__ __forceinline__ void walk8(Mm8 p, const Arrays& lds)
{
    constexpr int SIDE = Sh::SIDE, RF = Sh::RF, SF = Sh::SF, THREADS = Sh::THREADS;
    const int tid = (int)threadIdx.x, lane = tid & 63, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int wr = wave / Sh::WS * (RF * 16), ws = wave % Sh::WS * (SF * 16);
    const uint32_t tr = (uint32_t)((p.R + SIDE - 1) / SIDE), ts = (uint32_t)((p.S + SIDE - 1) / SIDE);
    const uint32_t tiles = tr * ts, units = tiles * (uint32_t)p.splits;
    const int64_t steps = (p.K + FP8_BLOCK - 1) / FP8_BLOCK;

    Rows8<Sh> ta, tb;
    Reader<uint8_t, SIDE, false, 1> ra, rb;
    ra.init(wr);
    rb.init(ws);
    int64_t r0, s0;
    uint32_t plane;
    int count;
    const float *psa, *psb;   // the step's scales of the tile's first row and column
    int row_a, row_b;         // of this thread's row and (by row) column, from there
    int k_left;
    auto begin_tile = [&](uint32_t g) __attribute__((always_inline)) {
        uint32_t ti, tj;
        const uint32_t unit = in_run(g, units);
        plane = PARTIAL ? unit / tiles : 0;
        tile_of(unit - plane * tiles, tr, ts, ti, tj);
        // (its division runs in vector registers: the loads' bases would stay there)
        ti = __builtin_amdgcn_readfirstlane(ti);
        tj = __builtin_amdgcn_readfirstlane(tj);
        const int64_t t0 = PARTIAL ? steps * plane / p.splits : 0;
        const int64_t t1 = PARTIAL ? steps * (plane + 1) / p.splits : steps;
        count = (int)(t1 - t0);
        r0 = (int64_t)ti * SIDE;
        s0 = (int64_t)tj * SIDE;
        ta.init(p.a, p.lda, r0, p.R, t0 * FP8_BLOCK);
        tb.init(p.b, p.ldb, s0, p.S, t0 * FP8_BLOCK);
        psa = p.sa.p + r0 * p.sa.rs + t0 * p.sa.cs;
        row_a = min(tid % SIDE, (int)min(p.R - r0, (int64_t)SIDE) - 1) * (int)p.sa.rs;
        if constexpr (BY_ROW) {
            psb = p.sb.p + s0 * p.sb.rs + t0 * p.sb.cs;
            row_b = min(tid % SIDE, (int)min(p.S - s0, (int64_t)SIDE) - 1) * (int)p.sb.rs;
        } else {
            psb = p.sb.p + min(s0 + ws, p.S - 1) / FP8_BLOCK * p.sb.rs + t0 * p.sb.cs;
            row_b = 0;
        }
        k_left = (int)(min(p.K, t1 * FP8_BLOCK) - t0 * FP8_BLOCK);
    };
    // The next step's operands on their way to LDS (chunks of 16 bytes that lie
    // inside the rows; zeros behind), its scales to registers.
    float next_a = 0.0f, next_b = 0.0f;
    auto load = [&](char* la, char* lb) __attribute__((always_inline)) {
        ta.load(la, k_left, wave);
        tb.load(lb, k_left, wave);
        next_a = psa[row_a];
        next_b = psb[row_b];
        psa += p.sa.cs;
        psb += p.sb.cs;
        k_left -= FP8_BLOCK;
    };
    // The arguments once more, as the compiler sees it: what the loop over the steps does
    // not need is then fetched where it is, instead of held in registers throughout.
    auto arguments = []() __attribute__((always_inline)) {
        auto k = (const __attribute__((address_space(4))) Mm8*)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(k));
        return (const Mm8*)k;
    };
    // What rows have beyond their last whole 16 bytes, put in its place byte by byte: no
    // byte behind a row is read.
    auto tail = [&](char* la, char* lb) __attribute__((always_inline)) {
        const Mm8& p = *arguments();
        const int in = (int)(p.K % FP8_BLOCK);
        int f = tid;
        asm volatile("" : "+v"(f));   // (nothing of this is worked out ahead of the loop)
#pragma unroll 1
        for (; f < 2 * SIDE; f += THREADS) {
            const int row = f % SIDE;
            const bool of_a = f < SIDE;
            const uint8_t* src = of_a ? p.a + min(r0 + row, p.R - 1) * p.lda : p.b + min(s0 + row, p.S - 1) * p.ldb;
            uint8_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = e < in % 16 ? src[p.K - in % 16 + e] : (uint8_t)0;
            __builtin_memcpy((of_a ? la : lb) + row * FP8_BLOCK + ((in / 16 ^ (row & 7)) << 4), v, 16);
        }
    };
    auto fragment = [&](const Reader<uint8_t, SIDE, false, 1>& r, const char* l, int i) __attribute__((always_inline)) {
        const i32x4 lo = __builtin_bit_cast(i32x4, r.get(l, i, 0)), hi = __builtin_bit_cast(i32x4, r.get(l, i, 1));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    float acc[RF][SF][4];   // (as single numbers: the compiler keeps these where they are)
    // A step that lies in la, lb, its scales in sa, sb; meanwhile the next one is loaded.
    auto step = [&](char* la, char* lb, float* sa, float* sb, char* na, char* nb, bool last,
                    bool more) __attribute__((always_inline)) {
        // (everybody is done with what na, nb and the scales' places held)
        sa[tid % SIDE] = next_a;
        if constexpr (BY_ROW) sb[tid % SIDE] = next_b;
        const float one_b = next_b;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (last && p.K % 16) {
            if (!PARTIAL || plane == (uint32_t)p.splits - 1) {
                tail(la, lb);
                __syncthreads();
            }
        }
        if (more) load(na, nb);
        ra.renew();
        rb.renew();
        i32x8 b[SF], a[2];
#pragma unroll
        for (int j = 0; j < SF; ++j) b[j] = fragment(rb, lb, j);
        f32x4 sbv[BY_ROW ? SF : 1];
        if constexpr (BY_ROW)
#pragma unroll
            for (int j = 0; j < SF; ++j) sbv[j] = *(const f32x4*)(sb + ws + 16 * j + 4 * q);
        a[0] = fragment(ra, la, 0);
        // (a product's result is used LATE products later)
        constexpr int LATE = 2, ALL = RF * SF;
        // products in the order written: 8,192 x 4,096 by 16,384 with tanh GELU and
        // pre-activation 605 us, so 591, 16,384 x 8,192 by 4,096 by row 610, so 594; with
        // more workgroups on a CU 1% slower
        constexpr bool PINNED = SIDE == 256;
        f32x4 t[LATE + 1];
        float s[2];
#pragma unroll
        for (int k = 0; k < ALL + LATE; ++k) {
            const int i = k / SF, j = k % SF;
            if (k < ALL) {
                if (j == 0) {
                    // (fragments of two rounds at most are held)
                    __builtin_amdgcn_sched_barrier(0);
                    if (i + 1 < RF) a[(i + 1) & 1] = fragment(ra, la, i + 1);
                    s[i & 1] = sa[wr + 16 * i + (lane & 15)];
                    if constexpr (!BY_ROW) s[i & 1] *= one_b;
                }
                if constexpr (PINNED) __builtin_amdgcn_sched_barrier(0);
                t[k % (LATE + 1)] = mfma8<FB, FA>(b[j], a[i & 1]);
                // (here: the compiler would put it off to its use, and wait for it there)
                if constexpr (PINNED) {
                    asm volatile("" ::"v"(t[k % (LATE + 1)]));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (k >= LATE) {
                const int m = k - LATE, mi = m / SF, mj = m % SF;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float by = BY_ROW ? s[mi & 1] * sbv[BY_ROW ? mj : 0][e] : s[mi & 1];
                    acc[mi][mj][e] = fmaf(t[m % (LATE + 1)][e], by, acc[mi][mj][e]);
                    if constexpr (PINNED) asm volatile("" : "+v"(acc[mi][mj][e]));
                }
            }
        }
    };

    for (uint32_t g = blockIdx.x; g < units; g += gridDim.x) {
        begin_tile(g);
        __syncthreads();
        if (count > 0) load(lds.la0, lds.lb0);   // (in = 0: nothing)
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int j = 0; j < SF; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
        for (int t = 0; t < count; t += 2) {
            step(lds.la0, lds.lb0, lds.sa0, lds.sb0, lds.la1, lds.lb1, t + 1 == count, t + 1 < count);
            if (t + 1 < count)
                step(lds.la1, lds.lb1, lds.sa1, lds.sb1, lds.la0, lds.lb0, t + 2 == count, t + 2 < count);
        }
        // Two fragments' columns 4 q on, exchanged between lanes 16 apart: 8 neighbours
        // of a row a lane.
        const Mm8& e = *arguments();
        int at = lane;
        asm volatile("" : "+v"(at));   // (as the arguments)
        const int64_t st = s0 + ws + (at >> 5) * 8 + (at >> 4 & 1) * 16;
        // What is added to sums is read ahead of the stores: waiting for it later would
        // be waiting for them too (8,192 x 4,096 by 16,384 with bias: 565 us, so 557).
        // Scales by row take the registers that this needs, and their products, of
        // gradients, have neither.
        constexpr bool AHEAD = !PARTIAL && !BY_ROW;
        Added<AHEAD ? SF / 2 : 0, TO> bias, res, next;
        if constexpr (AHEAD) {
            bias.load(e.e, e.e.bias, 0, st, e.S);
            res.load(e.e, r0 + wr + (at & 15) < e.R ? e.e.res : nullptr, (r0 + wr + (at & 15)) * e.e.res_rs, st, e.S);
        }
#pragma unroll 1
        for (int i = 0; i < RF; ++i) {
            const int64_t r = r0 + wr + 16 * i + (at & 15);
            if constexpr (AHEAD)
                next.load(e.e, i + 1 < RF && r + 16 < e.R ? e.e.res : nullptr, (r + 16) * e.e.res_rs, st, e.S);
            float sum[SF][4];
#pragma unroll
            for (int k = 0; k < RF; ++k)
                if (k == i)
#pragma unroll
                    for (int j = 0; j < SF; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            sum[j][c] = acc[k][j][c];
                            asm volatile("" : "+v"(sum[j][c]));   // (a branch, no selects)
                        }
#pragma unroll
            for (int j = 0; j < SF; j += 2) {
                float v[8];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const auto x = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, sum[j][c]),
                                                                    __builtin_bit_cast(unsigned, sum[j + 1][c]),
                                                                    false, false);
                    const unsigned lo = x[0], hi = x[1];
                    v[c] = __builtin_bit_cast(float, lo);
                    v[4 + c] = __builtin_bit_cast(float, hi);
                    // (by all lanes: the compiler would put it behind the branch below)
                    asm volatile("" : "+v"(v[c]), "+v"(v[4 + c]));
                }
                const int64_t s = st + j * 16;
                if (r >= e.R || s >= e.S) continue;
                const int n = (int)min((int64_t)8, e.S - s);
                if constexpr (PARTIAL) {
                    // (the rows of the partial sums are padded to 8)
                    store8(e.partial + ((int64_t)plane * e.R + r) * e.partial_ld + s, v);
                } else if (AHEAD && e.e.vec && n == 8) {
                    if (e.e.bias) bias.add(j / 2, v);
                    if (e.e.pre) store8(static_cast<TO*>(e.e.pre) + r * e.e.pre_ld + s, v);
                    activate<TO, 8>(v, e.e.act);
                    if (e.e.res) res.add(j / 2, v);
                    store8(static_cast<TO*>(e.e.y) + r * e.e.y_ld + s, v);
                } else {
                    store_linear<TO>(e.e, r, s, n, v);
                }
            }
            res = next;
        }
    }
}

template <class T>
struct Result {
    using Type = T;
};

struct Lds8 {
    char *la0, *lb0, *la1, *lb1;
    float *sa0, *sb0, *sa1, *sb1;
};

template <class Sh, int FA, int FB, bool BY_ROW, class TO, bool PARTIAL>
__global__ __launch_bounds__(Sh::THREADS, Sh::SIDE == 256 ? 2 : Sh::SIDE == 128 ? 2 : 4) void k_mm8(Mm8 p)
{
#ifdef __HIP_DEVICE_COMPILE__
    // each an array of its own: what one is read from is not what is being filled
    __shared__ __attribute__((aligned(1024))) char la0[Sh::BYTES], lb0[Sh::BYTES], la1[Sh::BYTES], lb1[Sh::BYTES];
    __shared__ __attribute__((aligned(16))) float sa0[Sh::SIDE], sb0[Sh::SIDE], sa1[Sh::SIDE], sb1[Sh::SIDE];
    walk8<Sh, FA, FB, BY_ROW, TO, PARTIAL>(p, Lds8{la0, lb0, la1, lb1, sa0, sb0, sa1, sb1});
#endif
}

template <class Sh>
hipError_t launch_mm8(const Mm8& p, int dtype, hipStream_t stream)
{
    const int64_t tiles = ((p.R + Sh::SIDE - 1) / Sh::SIDE) * ((p.S + Sh::SIDE - 1) / Sh::SIDE);
    if (tiles > 0x7fffffffLL / p.splits) return hipErrorInvalidConfiguration;
    const int64_t units = tiles * p.splits;
    const int64_t fit = (int64_t)device_cu_count() * (Sh::SIDE == 256 ? 1 : Sh::SIDE == 128 ? 2 : 4);
    const dim3 grid((unsigned)(units < fit ? units : fit)), block(Sh::THREADS);
    auto by_type = [&](auto fa, auto fb, auto by_row) {
        constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;
        constexpr bool BR = decltype(by_row)::value;
        if (dtype == MAG_F32)
            hipLaunchKernelGGL((k_mm8<Sh, FA, FB, BR, float, true>), grid, block, 0, stream, p);
        else if (dtype == MAG_F16)
            hipLaunchKernelGGL((k_mm8<Sh, FA, FB, BR, f16, false>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((k_mm8<Sh, FA, FB, BR, bf16, false>), grid, block, 0, stream, p);
    };
    auto by_scale = [&](auto fa, auto fb) {
        if (p.by_row)
            by_type(fa, fb, std::true_type{});
        else
            by_type(fa, fb, std::false_type{});
    };
    using E4 = std::integral_constant<int, MAG_E4M3>;
    using E5 = std::integral_constant<int, MAG_E5M2>;
    if (p.fa == MAG_E4M3)
        p.fb == MAG_E4M3 ? by_scale(E4{}, E4{}) : by_scale(E4{}, E5{});
    else
        p.fb == MAG_E4M3 ? by_scale(E5{}, E4{}) : by_scale(E5{}, E5{});
    return hipGetLastError();
}

}  // namespace mag
