// mm.hpp -- the matrix-core tile product of the feed-forward block's operators.
#pragma once

#include <type_traits>

#include "activation.hpp"
#include "block.hpp"

namespace mag {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

template <class T>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c)
{
    if constexpr (__is_same(T, bf16))
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The same with the sums in accumulation registers, in place: left to itself the
// compiler copies a large tile's sums from registers to registers in the loop.
// It does not see what this writes and when: the sums are only read behind
// settle(), and none is added to twice within four products.
template <class T>
__device__ __forceinline__ void mfma_in_place(s16x8 a, s16x8 b, f32x4& c)
{
    if constexpr (__is_same(T, bf16))
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else
        asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// ------------------------------------------------------------------- operands
// A tile of an operand is a step of the reduction (128 bytes, 64 k of two bytes;
// of operands in P = 2 or 3 parts, which lie 32 k of each part after another in
// memory, 32 k) by ROWS rows of the output, in LDS as 16-byte chunks of 8
// elements (fp32: 4), filled by loads that go from memory to LDS without
// registers.  Such a load writes 64 chunks one after
// another, so a permutation against bank conflicts is made in what each lane
// reads.
//   along k (MC false): element (row, k) at row * ld + k.  An LDS row has the 8 or
//     12 chunks of a row; chunk c of row r sits at c ^ (r & 7), of 12 at c ^
//     (r / 2 & 3), so that 8 rows' chunks of one k cover all banks.  Read as they
//     are: 8 consecutive k of a row a lane.
//   along rows (MC true): element at k * ld + row.  An LDS row is one k; chunk c
//     of it sits at c ^ mc_swizzle(k).  Read through the transposing LDS load: 16
//     lanes hand in 4 steps of 16 rows and get 4 consecutive k of a row each (fp32:
//     one number at a time, the chunks of lanes 16 apart in other banks).
constexpr uint32_t NOWHERE = 0x80000000u;    // a buffer offset past every extent: reads zeros

template <class T>
constexpr int step_of(int P) { return P == 1 ? 128 / (int)sizeof(T) : 32; }

// what chunk c of step k is XORed with: 16 lanes read 4 steps' 32 bytes each, 32
// lanes those of 8 steps further on too (CH: chunks of an LDS row); of fp32, 64
// lanes read 4 steps' 64 bytes, 4 steps apart
template <class T, int CH>
__device__ __forceinline__ int mc_swizzle(int k)
{
    if constexpr (sizeof(T) == 4) return k & 12;
    return 2 * ((k & 3) | (CH % 16 == 0 ? k >> 1 & 4 : 0));
}

template <class T, int ROWS, bool MC, int P, int THREADS>
struct Tile {
    static constexpr int STEP = step_of<T>(P);
    static constexpr int SIZE = sizeof(T), PER = 16 / SIZE;   // elements a chunk
    static constexpr int BYTES = ROWS * STEP * P * SIZE;
    static constexpr int LOADS = BYTES / 16 / THREADS;        // chunks a thread
    static constexpr int CH = (MC ? ROWS : STEP) * P / PER;   // chunks an LDS row

    // whether the thread's chunks lie alike in their lines
    static constexpr bool ALIKE = THREADS % CH == 0;

    uint32_t off[LOADS];  // byte offset of the thread's chunks in a tile of the operand
    int k0[ALIKE ? 1 : LOADS];  // their first k (of the first chunk, if alike)

    // the first k of the thread's i-th chunk
    static __device__ __forceinline__ int first(int i)
    {
        const int f = i * THREADS + (int)threadIdx.x, line = f / CH;
        return MC ? line : source(line, f % CH) * PER % STEP;
    }
    // the chunk that lies at `pos` of a line
    static __device__ __forceinline__ int source(int line, int pos)
    {
        return pos ^ (MC ? mc_swizzle<T, CH>(line) : P == 3 ? line >> 1 & 3 : line & 7);
    }

    // rows of the operand from this tile's first one on; ld in elements
    __device__ __forceinline__ void init(int64_t ld, int64_t rows_left)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int f = i * THREADS + (int)threadIdx.x;
            const int line = f / CH;
            int c = source(line, f % CH);
            if (i < (ALIKE ? 1 : LOADS)) k0[i] = first(i);
            // (rows past the last one: any others, nothing of theirs is stored)
            if constexpr (MC) {
                if ((int64_t)c * PER >= padded(rows_left)) c = 0;
                off[i] = (uint32_t)(line * ld * SIZE + c * 16);
            } else {
                const int64_t r = line < rows_left ? line : rows_left - 1;
                off[i] = (uint32_t)(r * ld * SIZE + c * 16);
            }
        }
    }
    // elements that n rows take in a line
    static __device__ __forceinline__ int64_t padded(int64_t n)
    {
        return P == 1 ? n : (n + 31) / 32 * (32 * P);
    }

    // The thread's i-th chunk.  base: the operand at this tile's first row and
    // the step's first k; k_left: of the reduction from there on (zeros behind).
    // No branch: what a step costs beside its products is paid by every wave.
    __device__ __forceinline__ void load(const char* base, int k_left, char* lds, int wave, int i) const
    {
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7fffffff, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rs, (__attribute__((address_space(3))) void*)(lds + (i * THREADS + wave * 64) * 16), 16,
            (ALIKE ? k0[0] < k_left - (MC ? i * (THREADS / CH) : 0) : k0[i] < k_left) ? off[i] : NOWHERE, 0, 0, 0);
    }
};

// Fragments of a wave's part of a tile: 16 rows, 32 k (fp32: 16); row lane % 16, k
// 8 (lane / 16) on (fp32: 4 (lane / 16)).  What depends on the lane is worked out once, the rest is the load's
// own constant offset.
template <class T, int ROWS, bool MC, int P>
struct Reader {
    static constexpr int LINE = (MC ? ROWS : step_of<T>(P)) * P * (int)sizeof(T);  // bytes of an LDS row
    // along rows: what repeats from 16 rows to 16 rows (the swizzle XORs up to 16
    // chunks: 128 rows, or 32 P-part ones a 64-byte part)
    static constexpr int CYCLE = P == 1 ? 8 : P == 2 ? 4 : 8;
    static constexpr int KEPT_I = ROWS / 32 < CYCLE ? ROWS / 32 : CYCLE;
    static constexpr int KEPT = MC ? KEPT_I * (P == 1 ? 1 : P) : P == 3 ? 1 : 2;
    int at[KEPT];

    // The compiler takes the places for new: it would otherwise work the address
    // of every read that lies too far on for a constant offset out before the
    // loop, and hold a register for each.
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int i = 0; i < KEPT; ++i) asm volatile("" : "+v"(at[i]));
    }

    __device__ __forceinline__ void init(int row)
    {
        const int lane = (int)threadIdx.x & 63, q = lane & 15;
        if constexpr (MC && sizeof(T) == 4) {
            const int k = (lane >> 4) * 4;
#pragma unroll
            for (int i = 0; i < KEPT_I; ++i) {
                const int n = row + 16 * i + q;
                at[i] = k * LINE + (((n >> 2) ^ mc_swizzle<T, LINE / 16>(k)) << 4) + (n & 3) * 4;
            }
        } else if constexpr (MC) {
            const int k = (lane >> 4) * 8 + (q >> 2), b = (q & 3) >> 1;
#pragma unroll
            for (int i = 0; i < KEPT_I; ++i)
#pragma unroll
                for (int s = 0; s < (P == 1 ? 1 : P); ++s) {
                    const int n = row + 16 * i;
                    const int c = (P == 1 ? n / 8 : n / 32 * (4 * P) + s * 4 + n % 32 / 8) + b;
                    // (k + 4 and, of one part, k + 32 have the same place in their rows)
                    at[i * (P == 1 ? 1 : P) + s] =
                        k * LINE + ((c ^ mc_swizzle<T, LINE / 16>(k)) << 4) + ((q & 1) << 3);
                }
        } else if constexpr (P == 3) {
            at[0] = (row + q) * LINE + (((lane >> 4) ^ (q >> 1 & 3)) << 4);
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s)
                at[s] = (row + q) * LINE + (((s * 4 + (lane >> 4)) ^ (q & 7)) << 4);
        }
    }

    // rows 16 i on; s: half of a step, or part
    __device__ __forceinline__ s16x8 get(const char* lds, int i, int s) const
    {
        if constexpr (MC && sizeof(T) == 4) {
            static_assert(KEPT_I * 32 == ROWS, "");
            const char* p = lds + at[i] + s * 16 * LINE;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *(const float*)(p + e * LINE);
            return __builtin_bit_cast(s16x8, v);
        } else if constexpr (MC) {
            const char* p = lds + at[i % KEPT_I * (P == 1 ? 1 : P) + (P == 1 ? 0 : s)] +
                            (i / KEPT_I * KEPT_I * 32 * P + (P == 1 ? s * 32 * LINE : 0));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(p + 4 * LINE));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else if constexpr (P == 3) {
            return *(const s16x8*)(lds + at[0] + i * 16 * LINE + s * 64);
        } else {
            return *(const s16x8*)(lds + at[s] + i * 16 * LINE);
        }
    }
};

// ------------------------------------------------------------------ epilogues

// element j of a row of P parts: the place of its first part (the next ones follow 32 on)
template <int P>
__device__ __forceinline__ int64_t place(int64_t j)
{
    return P == 1 ? j : j / 32 * (32 * P) + j % 32;
}

// A sum of products of three-part fp32 operands that is not finite, taken again
// from the operands in fp32 (a part of an infinite operand times a part that is
// zero is NaN where the product may be infinite, and parts of huge operands may
// overflow where the sum does not).  The parts of a finite number add up to it
// exactly; an infinite or NaN one is its first part.  A NaN operand needs none of
// this, and is common where a step has diverged: one lane after the whole reduction
// of every sum would take a thousand times the product's own time.
__device__ __forceinline__ float whole_sum(const Mm& p, int64_t bt, int64_t r, int64_t s)
{
    auto value = [](const MmOperand& o, int64_t bt, int64_t row, int64_t k) {
        const bf16* h = static_cast<const bf16*>(o.p) + bt * o.batch +
                        (o.mc ? k * o.ld + place<3>(row) : row * o.ld + place<3>(k));
        return (float)h[0] + ((float)h[32] + (float)h[64]);
    };
    float sum = 0.0f;
#pragma unroll 1
    for (int64_t k = 0; k < p.K && sum == sum; ++k) sum = fmaf(value(p.a, bt, r, k), value(p.b, bt, s, k), sum);
    return sum;
}

// whether a row of an operand in three parts holds a NaN, by the 64 lanes of a wave
static __device__ __forceinline__ bool row_has_nan(const MmOperand& o, int64_t bt, int64_t row, int64_t K)
{
    const bf16* h = static_cast<const bf16*>(o.p) + bt * o.batch + (o.mc ? place<3>(row) : row * o.ld);
    bool nan = false;
#pragma unroll 4
    for (int64_t k = threadIdx.x % 64; k < K; k += 64) {
        const float v = (float)h[o.mc ? k * o.ld : place<3>(k)];
        nan = nan || v != v;
    }
    return __any(nan);
}

// Those of up to 64 rows of an operand in three parts that hold a NaN, a bit each (a
// call: within the tile product its code would cost the loop registers, and the
// whole product a tenth of its time).
__device__ __attribute__((noinline)) inline uint64_t rows_with_nan(const bf16* h, int64_t ld, bool across, int64_t row,
                                                                  int rows, int64_t K)
{
    const MmOperand o{h, ld, 0, across};
    uint64_t found = 0;
#pragma unroll 1
    for (int i = 0; i < rows; ++i)
        if (row_has_nan(o, 0, row + i, K)) found |= 1ull << i;
    return found;
}

__device__ __forceinline__ bool all_finite(const float* v)
{
    bool all = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) all = all && fabsf(v[i]) < __builtin_inff();
    return all;
}

// ... of 8 neighbours of a row, from column s on (n of them); nan: those, a bit each,
// that have a NaN operand
__device__ __forceinline__ void make_whole(const Mm& p, int64_t bt, int64_t r, int64_t s, int n, uint32_t nan,
                                           float* v)
{
    if (__builtin_expect(all_finite(v), 1)) return;
#pragma unroll 1
    for (int e = 0; e < n; ++e) {
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x = i == e ? v[i] : x;
        if (nan >> e & 1 || fabsf(x) < __builtin_inff()) continue;
        x = whole_sum(p, bt, r, s + e);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i == e ? x : v[i];
    }
}

// eight neighbours of a row, at any element (the hardware takes vector loads and
// stores at every alignment)
template <class T>
__device__ __forceinline__ void load8(const T* p, float* v)
{
    constexpr int PER = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
#pragma unroll
    for (int h = 0; h < 8 / PER; ++h) {
        const Piece t = *(const Piece*)(p + h * PER);
#pragma unroll
        for (int i = 0; i < PER; ++i) v[h * PER + i] = (float)t[i];
    }
}

template <class T>
__device__ __forceinline__ void store8(T* p, const float* v)
{
    constexpr int PER = 16 / sizeof(T);
    typedef T Piece __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
#pragma unroll
    for (int h = 0; h < 8 / PER; ++h) {
        Piece t;
#pragma unroll
        for (int i = 0; i < PER; ++i) t[i] = (T)v[h * PER + i];
        *(Piece*)(p + h * PER) = t;
    }
}

// the sums of a split product's parts, one plane after another, N planes' loads
// in flight
template <int N>
__device__ __forceinline__ void add_parts(const float* q, int64_t plane, int splits, float* v)
{
    for (int k = 0; k < splits; k += N) {
        float w[N][8];
#pragma unroll
        for (int u = 0; u < N; ++u) load8(q + min(k + u, splits - 1) * plane, w[u]);
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (k + u < splits)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += w[u][e];
    }
}

__device__ __forceinline__ void add_parts(const float* q, int64_t plane, int splits, float* v)
{
    if (splits <= 2)
        add_parts<2>(q, plane, splits, v);
    else if (splits <= 4)
        add_parts<4>(q, plane, splits, v);
    else
        add_parts<8>(q, plane, splits, v);
}

// eight neighbours from column j on (zeros from column `cols` on); neighbours in
// memory are loaded at once, whatever their alignment
template <class T>
__device__ __forceinline__ void get8(const T* p, int64_t cs, int64_t j, int64_t cols, float* v)
{
    if (cs == 1 && j + 8 <= cols) {
        load8(p + j, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = j + i < cols ? (float)p[(j + i) * cs] : 0.0f;
    }
}

// z = sum + bias, pre, y = act(z) + res for n <= 8 neighbours of a row
template <class T>
__device__ __forceinline__ void store_linear(const Epilogue& e, int64_t r, int64_t s, int n, float* z)
{
    if (e.vec && n == 8) {
        float b[8];
        if (e.bias) {
            load8(static_cast<const T*>(e.bias) + s, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] += b[i];
        }
        if (e.pre) store8(static_cast<T*>(e.pre) + r * e.pre_ld + s, z);
        activate<T, 8>(z, e.act);
        if (e.res) {
            load8(static_cast<const T*>(e.res) + r * e.res_rs + s, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] += b[i];
        }
        store8(static_cast<T*>(e.y) + r * e.y_ld + s, z);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= n) break;
            float v = z[i];
            if (e.bias) v += (float)static_cast<const T*>(e.bias)[s + i];
            if (e.pre) static_cast<T*>(e.pre)[r * e.pre_ld + s + i] = (T)v;
            activate<T, 1>(&v, e.act);
            if (e.res) v += (float)static_cast<const T*>(e.res)[r * e.res_rs + (s + i) * e.res_cs];
            static_cast<T*>(e.y)[r * e.y_ld + s + i] = (T)v;
        }
    }
}

// a / b of numbers >= 0: the 64-bit division takes some hundred instructions
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)
{
    return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// v as the sum of two halves
__device__ __forceinline__ void two_halves(float v, f16& hi, f16& lo)
{
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

// z = scale v + mix m (and the diagonal) for n <= 8 neighbours of a row (the rest
// of an iteration's padding: zeros)
static __device__ __forceinline__ void store_orth(const Mm& p, int64_t bt, int64_t r, int64_t s,
                                                  int n, const float* sum)
{
    const OrthStore& o = p.o;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = o.scale * sum[i];
    if (o.m) {
        const f16* m = o.m + bt * o.m_batch + r * o.m_ld + place<2>(s);
        float hi[8], lo[8];
        load8(m, hi);
        load8(m + 32, lo);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(o.mix, hi[i] + lo[i], v[i]);
    }
    if (o.diagonal != 0.0f)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += s + i == r ? o.diagonal : 0.0f;
    if (o.z) {
        s16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f16 h, l;
            two_halves(i < n ? v[i] : 0.0f, h, l);
            hi[i] = __builtin_bit_cast(short, h);
            lo[i] = __builtin_bit_cast(short, l);
        }
        f16* z = o.z + bt * o.z_batch + r * o.z_ld + place<2>(s);
        *(s16x8*)z = hi;
        *(s16x8*)(z + 32) = lo;
    } else {
        const int64_t at = bt * o.out_batch + r * o.out_ld + s;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= n) break;
            if (o.dtype == MAG_F32)
                static_cast<float*>(o.out)[at + i] = v[i];
            else if (o.dtype == MAG_F16)
                static_cast<f16*>(o.out)[at + i] = (f16)v[i];
            else
                static_cast<bf16*>(o.out)[at + i] = (bf16)v[i];
        }
    }
}

// ------------------------------------------------------------------ the kernel

// The b-th piece of work of `count`: the XCDs (workgroups go round them, 8 at a
// time) get runs of neighbours, so that an XCD's L2 holds the operands of what
// runs on it together (12 matrices of 832 x 921, not so: 107 us, so: 80 us).
__device__ __forceinline__ uint32_t in_run(uint32_t b, uint32_t count)
{
    const uint32_t per = count / 8, rest = count % 8, x = b % 8;
    return x * per + min(x, rest) + b / 8;
}

// the g-th tile: bands of 8 tile rows
__device__ __forceinline__ void tile_of(uint32_t g, uint32_t tr, uint32_t ts, uint32_t& ti, uint32_t& tj)
{
    const uint32_t band = g / (8 * ts);
    const uint32_t height = min(8u, tr - band * 8);
    const uint32_t in = g - band * 8 * ts;
    ti = band * 8 + in % height;
    tj = in / height;
}

// the g-th tile (ti <= tj) on and above the diagonal of n x n: bands of 8 tile
// columns, row by row, so that neighbours share operands both ways (column by
// column, five steps of 4096 x 4096 took 5.06 ms, so they take 3.79)
__device__ __forceinline__ void tile_above(uint32_t g, uint32_t n, uint32_t& ti, uint32_t& tj)
{
    // its column, were they taken one by one: the bands hold the same tiles
    uint32_t c = (uint32_t)((sqrtf(8.0f * (float)g + 1.0f) - 1.0f) * 0.5f);
    while (c * (c + 1) / 2 > g) --c;
    while ((c + 1) * (c + 2) / 2 <= g) ++c;
    const uint32_t c0 = c / 8 * 8, width = min(8u, n - c0);
    uint32_t in = g - c0 * (c0 + 1) / 2;
    if (in < c0 * width) {
        ti = in / width;
        tj = c0 + in % width;
        return;
    }
    in -= c0 * width;
    uint32_t r = 0;
    for (; in >= width - r; ++r) in -= width - r;
    ti = c0 + r;
    tj = c0 + r + in;
}

// Workgroups that a CU holds, by its 160 KB of LDS and 512 registers a lane.
constexpr int wgs_per_cu(int side, int P, int stages)
{
    return side == 256 || (side == 128 && (P == 3 || stages == 4)) || (P == 3 && stages == 4) ? 1 : 2;
}

// out[r][s] = sum over k of a(r, k) b(s, k).  Bound by the matrix cores in the
// 256 tile (8,192 x 16,384 x 4,096 bfloat16 with its epilogue 920 us, 1,195
// TFLOP/s; two such gradients 1,670 us, 1,315), by what the L2s deliver to LDS, 10
// to 12 TB/s, in the smaller ones: a 64 tile moves four times a 256 one's bytes.
// Steps of 128 bytes a row: half as long ones double the L2's requests.
//
// Workgroups (as many as fit) walk the tiles.  Four waves hold a quarter of a
// tile's sums each.  Fragments are read from LDS a few at a time while the
// products of the ones before run, and the loads of the step that takes the
// present one's place in LDS are issued between products too: one barrier a
// step, where everybody is done reading one step and has the next.  The next
// tile's first steps are loaded before the present one's sums are stored,
// through LDS of their own.
//   one part:    the halves of a step, 0 0 | 1 1
//   two parts:   high high | low high | high low
//   three parts: 1 1 | 1 2, 2 1, 2 2 | 3 1, 1 3 (the products below 2^-24 left out)
//
// This workgroup: pieces of work first(), first() + stride(), ...  (p by value: by
// reference, the 256 tile spills 15 registers more.)
template <int BYTES, int STAGES, int COLS>
struct Lds {
    // each tile an array of its own: what one is read from is not what is being
    // filled
    char (&la0)[BYTES], (&lb0)[BYTES], (&la1)[BYTES], (&lb1)[BYTES];
    char (&la2)[STAGES > 2 ? BYTES : 16], (&lb2)[STAGES > 2 ? BYTES : 16];
    char (&la3)[STAGES > 2 ? BYTES : 16], (&lb3)[STAGES > 2 ? BYTES : 16];
    char (&lo)[4 * 16 * COLS * 4];
};
#define MM_LDS(T, SIDE, STAGES, P)                                                                     \
    constexpr int BYTES_ = Tile<T, SIDE, false, P, 256>::BYTES, MORE_ = STAGES > 2 ? BYTES_ : 16;      \
    __shared__ __attribute__((aligned(1024))) char la0[BYTES_], lb0[BYTES_], la1[BYTES_], lb1[BYTES_]; \
    __shared__ __attribute__((aligned(1024))) char la2[MORE_], lb2[MORE_], la3[MORE_], lb3[MORE_];     \
    __shared__ __attribute__((aligned(1024))) char lo[4 * 16 * (SIDE / 2) * 4];                        \
    const Lds<BYTES_, STAGES, SIDE / 2> lds{la0, lb0, la1, lb1, la2, lb2, la3, lb3, lo}

template <class T, class TO, int EPI, int SIDE, int STAGES, int P, bool AMC, bool BMC, class First, class Stride, class Arrays>
__device__ __forceinline__ void walk(Mm p, First first, Stride stride, const Arrays& lds)
{
    constexpr int THREADS = 256, W = 2;          // 2 x 2 waves
    constexpr int COLS = SIDE / W, F = COLS / 16;  // a wave's rows and columns, in 16s
    constexpr int STEP = step_of<T>(P);
    constexpr int SIZE = sizeof(T);
    constexpr bool IN_PLACE = F >= 8;
    using TA = Tile<T, SIDE, AMC, P, THREADS>;
    using TB = Tile<T, SIDE, BMC, P, THREADS>;
    constexpr int L = TA::LOADS;
    static_assert(TA::LOADS == TB::LOADS, "");
    auto &la0 = lds.la0, &lb0 = lds.lb0, &la1 = lds.la1, &lb1 = lds.lb1;
    auto &la2 = lds.la2, &lb2 = lds.lb2, &la3 = lds.la3, &lb3 = lds.lb3;
    auto& lo = lds.lo;

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int lane = (int)threadIdx.x & 63;
    const int wr = wave / W * COLS, ws = wave % W * COLS;
    const uint32_t tr = (uint32_t)((p.R + SIDE - 1) / SIDE), ts = (uint32_t)((p.S + SIDE - 1) / SIDE);
    const uint32_t tiles = EPI != MM_LINEAR && p.symmetric ? tr * (tr + 1) / 2 : tr * ts;
    // pieces of work: of every matrix, and every share of the steps, each tile
    const uint32_t units = tiles * (uint32_t)p.splits * (uint32_t)p.batch;
    const int64_t steps = (p.K + STEP - 1) / STEP;
    const int64_t a_step = AMC ? STEP * p.a.ld * SIZE : STEP * P * SIZE;
    const int64_t b_step = BMC ? STEP * p.b.ld * SIZE : STEP * P * SIZE;

    TA ta;
    TB tb;
    Reader<T, SIDE, AMC, P> ra;
    Reader<T, SIDE, BMC, P> rb;
    ra.init(wr);
    rb.init(ws);
    int64_t r0, s0;
    uint32_t plane;
    int count;
    bool mirror;
    const char *pa, *pb;
    int k_left;  // none behind this workgroup's last step
    auto advance = [&] {
        pa += a_step;
        pb += b_step;
        k_left -= STEP;
    };
    auto load = [&](char* la, char* lb) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            ta.load(pa, k_left, la, wave, i);
            tb.load(pb, k_left, lb, wave, i);
        }
        advance();
    };
    auto begin_tile = [&](uint32_t g) {
        uint32_t ti, tj;
        const uint32_t unit = in_run(g, units);
        plane = EPI == MM_LINEAR ? 0 : unit / tiles;   // (linear layers: one matrix, not split)
        const uint32_t tile = unit - plane * tiles;
        if (EPI != MM_LINEAR && p.symmetric)
            tile_above(tile, ts, ti, tj);
        else
            tile_of(tile, tr, ts, ti, tj);
        const int64_t bt = EPI == MM_PARTIAL ? plane / p.splits : plane;
        const int64_t share = EPI == MM_PARTIAL ? plane % p.splits : 0;
        const int64_t t0 = EPI == MM_PARTIAL ? steps * share / p.splits : 0;
        const int64_t t1 = EPI == MM_PARTIAL ? steps * (share + 1) / p.splits : steps;
        count = (int)(t1 - t0);
        mirror = EPI == MM_ORTH && p.symmetric && ti != tj;
        r0 = (int64_t)ti * SIDE;
        s0 = (int64_t)tj * SIDE;
        ta.init(p.a.ld, p.R - r0);
        tb.init(p.b.ld, p.S - s0);
        pa = static_cast<const char*>(p.a.p) + SIZE * (bt * p.a.batch + (AMC ? r0 * P : r0 * p.a.ld)) + t0 * a_step;
        pb = static_cast<const char*>(p.b.p) + SIZE * (bt * p.b.batch + (BMC ? s0 * P : s0 * p.b.ld)) + t0 * b_step;
        k_left = (int)(min(p.K, t1 * STEP) - t0 * STEP);
        load(la0, lb0);
        load(la1, lb1);
        if constexpr (STAGES > 2) {
            load(la2, lb2);
            load(la3, lb3);
        }
    };

    f32x4 acc[F][F];
    // everybody is done with what was read before, and has all but the last
    // `ahead` steps that were loaded
    auto meet = [](auto ahead) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(ahead)::value * 2 * L) : "memory");
    };
    using None = std::integral_constant<int, 0>;
    using Ahead = std::integral_constant<int, STAGES - 2>;
    auto products = [&](const s16x8& a, const s16x8* b, int i) {
        if constexpr (SIZE == 4) {
            const f32x4 x = __builtin_bit_cast(f32x4, a);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < F; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, b[j])[k], x[k],
                                                                     acc[i][j], 0, 0, 0);
            return;
        } else
#pragma unroll
        for (int j = 0; j < F; ++j) {
            // (b first: a lane then holds four neighbours of one output row)
            if constexpr (IN_PLACE)
                mfma_in_place<T>(b[j], a, acc[i][j]);
            else
                acc[i][j] = mfma<T>(b[j], a, acc[i][j]);
        }
    };
    // what wrote the sums is done, whatever reads them comes later
    auto settle = [&] {
        if constexpr (IN_PLACE) {
            asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
            for (int i = 0; i < F; ++i)
#pragma unroll
                for (int j = 0; j < F; ++j) asm volatile("" : "+a"(acc[i][j]));
        }
    };
    // A step in la, lb, whose first fragments are in xa, xb; the next one's are left
    // in za, with `xb` or `zb` (one part: za, zb are read first, and the next ones
    // go where the present ones were).
    s16x8 xa[F], xb[F], za[F], zb[F], ya[P == 3 ? F : 1], yb[P == 3 ? F : 1];
    auto begin_next = [&](const char* na, const char* nb, char* la, char* lb, s16x8* fa, s16x8* fb,
                          int i) __attribute__((always_inline)) {
        fb[i] = rb.get(nb, i, 0);
        fa[i] = ra.get(na, i, 0);
#pragma unroll
        for (int l = i * L / F; l < (i + 1) * L / F; ++l) {
            ta.load(pa, k_left, la, wave, l);
            tb.load(pb, k_left, lb, wave, l);
        }
    };
    auto step = [&](char* la, char* lb, const char* na, const char* nb, s16x8* pxa, s16x8* pxb,
                    s16x8* pza, s16x8* pzb) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            pzb[i] = rb.get(lb, i, 1);
            pza[i] = ra.get(la, i, 1);
            products(pxa[i], pxb, i);
        }
        if constexpr (P == 1) {
            meet(Ahead{});
#pragma unroll
            for (int i = 0; i < F; ++i) {
                begin_next(na, nb, la, lb, pxa, pxb, i);
                products(pza[i], pzb, i);
            }
        } else if constexpr (P == 2) {
#pragma unroll
            for (int i = 0; i < F; ++i) products(pza[i], pxb, i);
            meet(Ahead{});
#pragma unroll
            for (int i = 0; i < F; ++i) {
                begin_next(na, nb, la, lb, pza, pxb, i);
                products(pxa[i], pzb, i);
            }
        } else {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                yb[i] = rb.get(lb, i, 2);
                ya[i] = ra.get(la, i, 2);
                products(pxa[i], pzb, i);
                products(pza[i], pxb, i);
                products(pza[i], pzb, i);
            }
            meet(Ahead{});
#pragma unroll
            for (int i = 0; i < F; ++i) {
                products(ya[i], pxb, i);
                begin_next(na, nb, la, lb, pza, pzb, i);
                products(pxa[i], yb, i);
            }
        }
        advance();
    };
    // the steps of a round of stages: operands' registers change places from step
    // to step
    auto pair = [&](char* a0, char* b0, char* a1, char* b1, const char* a2, const char* b2) {
        if constexpr (IN_PLACE) {
            ra.renew();
            rb.renew();
        }
        if constexpr (P == 1) {
            step(a0, b0, a1, b1, xa, xb, za, zb);
            step(a1, b1, a2, b2, xa, xb, za, zb);
        } else if constexpr (P == 2) {
            step(a0, b0, a1, b1, xa, xb, za, zb);
            step(a1, b1, a2, b2, za, xb, xa, zb);
        } else {
            step(a0, b0, a1, b1, xa, xb, za, zb);
            step(a1, b1, a2, b2, za, zb, xa, xb);
        }
    };

    uint32_t g = first();
    begin_tile(g);
    while (true) {
        // (said to the compiler too, which would otherwise wait in the loop for what it
        // takes to be on its way to the fragments' registers: with it for the steps' loads)
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
        meet(None{});
#pragma unroll
        for (int i = 0; i < F; ++i) {
            xb[i] = rb.get(lb0, i, 0);
            xa[i] = ra.get(la0, i, 0);
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        settle();
        // (a round of the stages at a time: behind the last step come zeros)
        for (int t = 0; t < count; t += STAGES) {
            if constexpr (STAGES == 2) {
                pair(la0, lb0, la1, lb1, la0, lb0);
            } else {
                pair(la0, lb0, la1, lb1, la2, lb2);
                pair(la2, lb2, la3, lb3, la0, lb0);
            }
        }
        meet(None{});
        settle();
        const int64_t rt = r0 + wr, st = s0 + ws;
        const int64_t bt = plane;
        // the wave's rows and columns that hold a NaN, looked for once a sum is not finite
        uint64_t nan_rows = 0, nan_cols = 0;
        bool looked = !(P == 3 && EPI == MM_LINEAR);
        // of the 8 neighbours from column s on of row r
        auto nans = [&](int64_t r, int64_t s) -> uint32_t {
            return nan_rows >> (r - rt) & 1 ? 255u : (uint32_t)(nan_cols >> (s - st)) & 255u;
        };
        const bool mirrored = mirror;
        g += stride();
        if (g < units) begin_tile(g);

        // The sums go to rows through a wave's own piece of LDS, 16 rows at a
        // time in 16-byte chunks that sit at (chunk ^ row): 8 neighbours of a
        // row a lane.
        constexpr int CHUNKS = COLS / 4, LANES = COLS / 8;
        char* mine = lo + wave * (16 * COLS * 4);
        auto at = [&](int row, int chunk) {
            return mine + (row * CHUNKS + (chunk ^ (row & (CHUNKS - 1)))) * 16;
        };
        const int64_t s8 = st + lane % LANES * 8;
        // a tile that lies inside the output, whole vectors: what a row needs of
        // memory is asked for before its sums come back from LDS
        bool inside = false;
        float bias[8] = {};
        if constexpr (EPI == MM_LINEAR) {
            inside = p.e.vec && rt + COLS <= p.R && st + COLS <= p.S;
            if (inside && p.e.bias) load8(static_cast<const TO*>(p.e.bias) + s8, bias);
        }
#pragma unroll 1
        for (int ph = 0; ph < F; ++ph) {
            constexpr int PASSES = 16 * LANES / 64;
            const int64_t r8 = rt + ph * 16 + lane / LANES;
            float res[EPI == MM_LINEAR ? PASSES : 1][8];
            if constexpr (EPI == MM_LINEAR)
                if (inside && p.e.res)
#pragma unroll
                    for (int q = 0; q < PASSES; ++q)
                        load8(static_cast<const TO*>(p.e.res) + (r8 + q * (64 / LANES)) * p.e.res_rs + s8, res[q]);
            float zero = 0.0f;
#pragma unroll
            for (int i = 0; i < F; ++i)
                if (i == ph)
#pragma unroll
                    for (int j = 0; j < F; ++j) {
                        *(f32x4*)at(lane & 15, j * 4 + (lane >> 4)) = acc[i][j];
                        if constexpr (P == 3 && EPI == MM_LINEAR)
#pragma unroll
                            for (int e = 0; e < 4; ++e) zero = fmaf(acc[i][j][e], 0.0f, zero);
                    }
            if (!looked && __builtin_expect(__any(zero != 0.0f), 0)) {
                looked = true;
                nan_rows = rows_with_nan(static_cast<const bf16*>(p.a.p) + bt * p.a.batch, p.a.ld, p.a.mc, rt,
                                         (int)min((int64_t)COLS, p.R - rt), p.K);
                nan_cols = rows_with_nan(static_cast<const bf16*>(p.b.p) + bt * p.b.batch, p.b.ld, p.b.mc, st,
                                         (int)min((int64_t)COLS, p.S - st), p.K);
            }
            if constexpr (EPI == MM_LINEAR)
                if (inside) {
                    float v[PASSES][8];
#pragma unroll
                    for (int q = 0; q < PASSES; ++q) {
                        const int row = lane / LANES + q * (64 / LANES);
                        *(f32x4*)v[q] = *(const f32x4*)at(row, lane % LANES * 2);
                        *(f32x4*)(v[q] + 4) = *(const f32x4*)at(row, lane % LANES * 2 + 1);
                    }
#pragma unroll
                    for (int q = 0; q < PASSES; ++q) {
                        const int64_t r = r8 + q * (64 / LANES);
                        if constexpr (P == 3) make_whole(p, bt, r, s8, 8, nans(r, s8), v[q]);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[q][e] += bias[e];
                        if (p.e.pre) store8(static_cast<TO*>(p.e.pre) + r * p.e.pre_ld + s8, v[q]);
                    }
                    activate<TO, 8 * PASSES>(v[0], p.e.act);
#pragma unroll
                    for (int q = 0; q < PASSES; ++q) {
                        if (p.e.res)
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[q][e] += res[q][e];
                        store8(static_cast<TO*>(p.e.y) + (r8 + q * (64 / LANES)) * p.e.y_ld + s8, v[q]);
                    }
                    continue;
                }
            const int64_t rp = rt + ph * 16;
#pragma unroll 1
            for (int row = lane / LANES; row < 16; row += 64 / LANES) {
                const int64_t r = rp + row, s = s8;
                float v[8];
                *(f32x4*)v = *(const f32x4*)at(row, lane % LANES * 2);
                *(f32x4*)(v + 4) = *(const f32x4*)at(row, lane % LANES * 2 + 1);
                if (r >= p.R || s >= (EPI == MM_ORTH && p.o.z ? p.o.z_ld / 2 : p.S)) continue;
                const int n = (int)max((int64_t)0, min((int64_t)8, p.S - s));
                if constexpr (EPI == MM_PARTIAL) {
                    // (the rows of the partial sums are padded to 8)
                    float* q = p.partial + (bt * p.R + r) * p.partial_ld + s;
                    *(f32x4*)q = *(f32x4*)v;
                    *(f32x4*)(q + 4) = *(f32x4*)(v + 4);
                } else if constexpr (EPI == MM_LINEAR) {
                    if constexpr (P == 3) make_whole(p, bt, r, s, n, nans(r, s), v);
                    store_linear<TO>(p.e, r, s, n, v);
                } else {
                    store_orth(p, bt, r, s, n, v);
                }
            }
            if (EPI == MM_ORTH && mirrored) {
                // the transpose: 8 neighbours of a column a lane
#pragma unroll 1
                for (int i = lane; i < COLS * 2; i += 64) {
                    const int c = i / 2, e0 = i % 2 * 8;
                    const int64_t r = st + c, s = rp + e0;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = *(const float*)(at(e0 + e, c / 4) + c % 4 * 4);
                    if (r >= p.S || s >= p.R) continue;
                    store_orth(p, bt, r, s, (int)min((int64_t)8, p.R - s), v);
                }
            }
        }
        if (g >= units) break;
    }
}

template <class T, class TO, int EPI, int SIDE, int STAGES, int P, bool AMC, bool BMC>
__global__ __launch_bounds__(256, wgs_per_cu(SIDE, P, STAGES)) void k_mm(Mm p)
{
#ifdef __HIP_DEVICE_COMPILE__
    MM_LDS(T, SIDE, STAGES, P);
    walk<T, TO, EPI, SIDE, STAGES, P, AMC, BMC>(
        p, [] { return blockIdx.x; }, [] { return gridDim.x; }, lds);
#endif
}

// A small layer's two gradients side by side, which would leave CUs idle one
// after the other (1,000 x 777 by 2,050 half: 13 and 15 us, together 19): the
// first `wgs` workgroups walk dx = dz weight, the others dweight = dz^T x.
template <class T, class TO, int P>
__global__ __launch_bounds__(256, wgs_per_cu(64, P, 4)) void k_mm_two(Mm dx, Mm dw, uint32_t wgs)
{
#ifdef __HIP_DEVICE_COMPILE__
    MM_LDS(T, 64, 4, P);
    if (blockIdx.x < wgs)
        walk<T, TO, MM_LINEAR, 64, 4, P, false, true>(
            dx, [] { return blockIdx.x; }, [=] { return wgs; }, lds);
    else
        walk<T, TO, MM_LINEAR, 64, 4, P, true, true>(
            dw, [=] { return blockIdx.x - wgs; }, [=] { return gridDim.x - wgs; }, lds);
#endif
}

template <class T, class TO, int P>
hipError_t launch_mm_two_tiles(const Mm& dx, const Mm& dw, int wgs_dx, int wgs_dw, hipStream_t stream)
{
    hipLaunchKernelGGL((k_mm_two<T, TO, P>), dim3((unsigned)(wgs_dx + wgs_dw)), dim3(256), 0, stream, dx, dw,
                       (uint32_t)wgs_dx);
    return hipGetLastError();
}

template <class T, class TO, int EPI, int SIDE, int STAGES, int P>
hipError_t launch_mm_tile(const Mm& p, hipStream_t stream)
{
    const int64_t tr = (p.R + SIDE - 1) / SIDE, ts = (p.S + SIDE - 1) / SIDE;
    const int64_t tiles = p.symmetric ? tr * (tr + 1) / 2 : tr * ts;
    if (tiles > 0x7fffffffLL / p.splits / p.batch) return hipErrorInvalidConfiguration;
    const int64_t fit = (int64_t)device_cu_count() * wgs_per_cu(SIDE, P, STAGES);
    const int64_t units = tiles * p.splits * p.batch;
    const dim3 grid((unsigned)(units < fit ? units : fit));
    const dim3 block(256);
    if (p.a.mc)
        if (p.b.mc)
            hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, STAGES, P, true, true>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, STAGES, P, true, false>), grid, block, 0, stream, p);
    else if (p.b.mc)
        hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, STAGES, P, false, true>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, STAGES, P, false, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

// The 128 tile, with four steps in LDS where every workgroup has a CU of its own
// and the reduction is long (2,048 x 2,048 bfloat16: by 8,192 74 us, with two steps
// 78 us; by 1,024, where starting counts, 16 and 13 us).
template <class T, class TO, int EPI, int P>
hipError_t launch_mm_128(const Mm& p, hipStream_t stream)
{
    const int64_t tr = (p.R + 127) / 128, ts = (p.S + 127) / 128;
    const int64_t units = (p.symmetric ? tr * (tr + 1) / 2 : tr * ts) * p.splits * p.batch;
    if (units <= device_cu_count() && p.K >= 32 * step_of<T>(P))
        return launch_mm_tile<T, TO, EPI, 128, 4, P>(p, stream);
    return launch_mm_tile<T, TO, EPI, 128, 2, P>(p, stream);
}

}  // namespace mag
