// mm.hpp -- the matrix-core tile product of the feed-forward block's operators.
#pragma once

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
    if constexpr (sizeof(T) == 2 && __is_same(T, bf16))
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
// A tile of an operand is 64 steps of the reduction by ROWS rows of the output,
// in LDS as 16-byte chunks of 8 elements, filled by loads that go from memory
// to LDS without registers.  Such a load writes 64 chunks one after another, so
// a permutation against bank conflicts is made in what each lane reads.
//   along k (MC false): element (row, k) at row * ld + k.  LDS row of 8 chunks;
//     chunk c of row r sits at c ^ (r & 7), so 8 rows' chunks of one k cover
//     all banks.  Read as they are: 8 consecutive k of a row a lane.
//   along rows (MC true): element at k * ld + row.  LDS row (one k) of ROWS / 8
//     chunks; chunk c of step k sits at c ^ mc_swizzle(k).  Read through the
//     transposing LDS load: 16 lanes hand in 4 steps of 16 rows and get 4
//     consecutive k of a row each.
constexpr int STEP = 64;                     // reduction per tile
constexpr uint32_t NOWHERE = 0x80000000u;    // a buffer offset past every extent: reads zeros

// what chunk c of step k is XORed with: 16 lanes read 4 steps' 32 bytes each, 32
// lanes those of 8 steps further on too
template <int ROWS>
__device__ __forceinline__ int mc_swizzle(int k)
{
    return 2 * ((k & 3) | (ROWS >= 128 ? k >> 1 & 4 : 0));
}

template <int ROWS, bool MC, int THREADS>
struct Tile {
    static constexpr int BYTES = ROWS * STEP * 2;
    static constexpr int LOADS = BYTES / 16 / THREADS;  // chunks a thread
    static constexpr int CH = MC ? ROWS / 8 : 8;        // chunks an LDS row

    uint32_t off[LOADS];  // byte offset of the thread's chunks in a tile of the operand
    int first;            // k of the first one (along k: of all)

    // rows of the operand from this tile's first one on; ld in elements
    __device__ __forceinline__ void init(int64_t ld, int64_t rows_left)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int f = i * THREADS + (int)threadIdx.x;
            const int line = f / CH, pos = f % CH;
            if constexpr (MC) {
                int c = pos ^ mc_swizzle<ROWS>(line);
                // (rows past the last one: any others, nothing of theirs is stored)
                if ((int64_t)c * 8 >= rows_left) c = 0;
                if (i == 0) first = line;
                off[i] = (uint32_t)(line * ld * 2 + c * 16);
            } else {
                const int c = pos ^ (line & 7);
                const int64_t r = line < rows_left ? line : rows_left - 1;
                if (i == 0) first = c * 8;
                off[i] = (uint32_t)(r * ld * 2 + c * 16);
            }
        }
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
            first + (MC ? i * (THREADS / CH) : 0) < k_left ? off[i] : NOWHERE, 0, 0, 0);
    }
};

// Fragments of a wave's part of a tile: 16 rows, 32 k; row lane % 16, k 8 (lane /
// 16) on.  What depends on the lane is worked out once, the rest is the load's
// own constant offset.
template <int ROWS, bool MC>
struct Reader {
    static constexpr int KEPT = MC ? (ROWS >= 256 ? 8 : ROWS >= 128 ? 4 : 2) : 2;
    uint32_t at[KEPT];

    __device__ __forceinline__ void init(int row)
    {
        const int lane = (int)threadIdx.x & 63, q = lane & 15;
        if constexpr (MC) {
            const int k = (lane >> 4) * 8 + (q >> 2);
#pragma unroll
            for (int i = 0; i < KEPT; ++i) {
                const int c = (row >> 3) + 2 * i + ((q & 3) >> 1);
                // (k + 4 and k + 32 have the same place in their rows)
                at[i] = (uint32_t)(k * (ROWS * 2) + ((c ^ mc_swizzle<ROWS>(k)) << 4) + ((q & 1) << 3));
            }
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s)
                at[s] = (uint32_t)((row + q) * 128 + (((s * 4 + (lane >> 4)) ^ (q & 7)) << 4));
        }
    }

    // rows 16 i on, half s of the step
    __device__ __forceinline__ s16x8 get(const char* lds, int i, int s) const
    {
        if constexpr (MC) {
            const char* p = lds + at[i % KEPT] + (i / KEPT * KEPT * 32 + s * 32 * ROWS * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(p + 4 * ROWS * 2));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            return *(const s16x8*)(lds + at[s] + i * 2048);
        }
    }
};

// ------------------------------------------------------------------ epilogues

template <class T>
__device__ __forceinline__ float part_sum(const T* h, int64_t plane, int64_t i)
{
    return (float)h[i] + ((float)h[i + plane] + (float)h[i + 2 * plane]);
}

// A sum of products of three-part fp32 operands that is not finite, taken again
// from the operands in fp32 (a part of an infinite operand times a part that is
// zero is NaN where the product may be infinite, and parts of huge operands may
// overflow where the sum does not).  The parts of a finite number add up to it
// exactly; an infinite or NaN one is its first part.
__device__ __forceinline__ float whole_sum(const Mm& p, int64_t bt, int64_t r, int64_t s)
{
    const bf16* A = static_cast<const bf16*>(p.a.p) + bt * p.a.batch;
    const bf16* B = static_cast<const bf16*>(p.b.p) + bt * p.b.batch;
    const int64_t as = p.a.mc ? p.a.ld : 1, bs = p.b.mc ? p.b.ld : 1;
    int64_t a = p.a.mc ? r : r * p.a.ld, b = p.b.mc ? s : s * p.b.ld;
    float sum = 0.0f;
#pragma unroll 1
    for (int64_t k = 0; k < p.K; ++k, a += as, b += bs)
        sum = fmaf(part_sum(A, p.a.plane, a), part_sum(B, p.b.plane, b), sum);
    return sum;
}

__device__ __forceinline__ void fix(float* v, int e, float x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i == e ? x : v[i];
}

// eight neighbours from column j on (zeros from column `cols` on); neighbours in
// memory are loaded at once, whatever their alignment
template <class T>
__device__ __forceinline__ void get8(const T* p, int64_t cs, int64_t j, int64_t cols, float* v)
{
    if (cs == 1 && j + 8 <= cols) {
        T t[8];
        __builtin_memcpy(t, p + j, sizeof(t));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = j + i < cols ? (float)p[(j + i) * cs] : 0.0f;
    }
}

// eight neighbours of a row, two bytes or four each
template <class T>
__device__ __forceinline__ void load8(const T* p, float* v)
{
    if constexpr (sizeof(T) == 4) {
        const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    } else {
        const s16x8 a = *(const s16x8*)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)__builtin_bit_cast(T, (short)a[i]);
    }
}

template <class T>
__device__ __forceinline__ void store8(T* p, const float* v)
{
    if constexpr (sizeof(T) == 4) {
        *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        s16x8 a;
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = __builtin_bit_cast(short, (T)v[i]);
        *(s16x8*)p = a;
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
        activate<8>(z, e.act);
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
            activate<1>(&v, e.act);
            if (e.res) v += (float)static_cast<const T*>(e.res)[r * e.res_rs + (s + i) * e.res_cs];
            static_cast<T*>(e.y)[r * e.y_ld + s + i] = (T)v;
        }
    }
}

// v as the sum of two halves
__device__ __forceinline__ void two_halves(float v, f16& hi, f16& lo)
{
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

// z = scale v + mix m for n <= 8 neighbours of a row (the rest of an
// iteration's planes' padding: zeros)
static __device__ __forceinline__ void store_orth(const Mm& p, int64_t bt, int64_t r, int64_t s,
                                                  int n, const float* sum)
{
    const OrthStore& o = p.o;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = o.scale * sum[i];
    if (o.m) {
        const f16* m = o.m + bt * o.m_batch + r * o.m_ld + s;
        float hi[8], lo[8];
        load8(m, hi);
        load8(m + o.m_plane, lo);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(o.mix, hi[i] + lo[i], v[i]);
    }
    if (o.z) {
        s16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f16 h, l;
            two_halves(i < n ? v[i] : 0.0f, h, l);
            hi[i] = __builtin_bit_cast(short, h);
            lo[i] = __builtin_bit_cast(short, l);
        }
        f16* z = o.z + bt * o.z_batch + r * o.z_ld + s;
        *(s16x8*)z = hi;
        *(s16x8*)(z + o.z_plane) = lo;
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

// Tile number -> tile: the XCDs (workgroups go round them, 8 at a time) get runs
// of neighbouring tiles, and a run walks bands of 8 tile rows, so that an XCD's
// L2 holds the operands of what runs on it together.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t count, uint32_t tr, uint32_t ts,
                                        uint32_t& ti, uint32_t& tj)
{
    const uint32_t per = count / 8, rest = count % 8;
    const uint32_t x = b % 8;
    const uint32_t g = x * per + min(x, rest) + b / 8;
    const uint32_t band = g / (8 * ts);
    const uint32_t height = min(8u, tr - band * 8);
    const uint32_t in = g - band * 8 * ts;
    ti = band * 8 + in % height;
    tj = in / height;
}

// the b-th tile (ti <= tj) on and above the diagonal, column by column
__device__ __forceinline__ void tile_above(uint32_t b, uint32_t& ti, uint32_t& tj)
{
    tj = (uint32_t)((sqrtf(8.0f * (float)b + 1.0f) - 1.0f) * 0.5f);
    while (tj * (tj + 1) / 2 > b) --tj;
    while ((tj + 1) * (tj + 2) / 2 <= b) ++tj;
    ti = b - tj * (tj + 1) / 2;
}

// Workgroups that the device holds at once, by tile.
constexpr int wgs_per_cu(int side) { return side == 256 ? 1 : side == 128 ? 2 : 4; }

// Workgroups (as many as fit) walk the tiles.  Four waves hold a quarter of a
// tile's sums each.  Two steps' operands are in LDS; a step's 64 k are taken as
// two halves, and the fragments of a half are read from LDS, a few at a time,
// while the products of the half before it run, as are the loads of the step
// after the next issued: one barrier a step, where everybody is done reading one
// step and has the next.  The next tile's first steps are loaded before the
// present one's sums are stored, through LDS of their own.
template <class T, class TO, int EPI, int SIDE, bool AMC, bool BMC>
__global__ __launch_bounds__(256, SIDE == 256 ? 1 : SIDE == 128 ? 2 : 4) void k_mm(Mm p)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int THREADS = 256, W = 2;          // 2 x 2 waves
    constexpr int COLS = SIDE / W, F = COLS / 16;  // a wave's rows and columns, in 16s
    constexpr bool IN_PLACE = F >= 8;
    using TA = Tile<SIDE, AMC, THREADS>;
    using TB = Tile<SIDE, BMC, THREADS>;
    // two tiles of each operand, as separate arrays: what one is read from is
    // not what is being filled
    __shared__ __attribute__((aligned(1024))) char la0[TA::BYTES], lb0[TB::BYTES];
    __shared__ __attribute__((aligned(1024))) char la1[TA::BYTES], lb1[TB::BYTES];
    __shared__ __attribute__((aligned(1024))) char lo[4 * 16 * COLS * 4];

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int lane = (int)threadIdx.x & 63;
    const int wr = wave / W * COLS, ws = wave % W * COLS;
    const uint32_t tr = (uint32_t)((p.R + SIDE - 1) / SIDE), ts = (uint32_t)((p.S + SIDE - 1) / SIDE);
    const uint32_t tiles = EPI == MM_ORTH && p.symmetric ? tr * (tr + 1) / 2 : tr * ts;
    const int64_t bt = blockIdx.z;
    // this workgroup's share of the steps: all products of parts, K each
    const int per_product = max(1, (int)((p.K + STEP - 1) / STEP));
    const int64_t steps = (int64_t)per_product * p.products;
    const int64_t t0 = steps * blockIdx.y / p.splits, t1 = steps * (blockIdx.y + 1) / p.splits;
    const int count = (int)(t1 - t0);
    const int64_t a_step = AMC ? STEP * p.a.ld * 2 : STEP * 2;
    const int64_t b_step = BMC ? STEP * p.b.ld * 2 : STEP * 2;

    TA ta;
    TB tb;
    Reader<SIDE, AMC> ra;
    Reader<SIDE, BMC> rb;
    ra.init(wr);
    rb.init(ws);
    int64_t r0, s0;
    bool mirror;
    const char *A, *B, *pa, *pb;
    int product, k_left, steps_left;
    auto begin_product = [&](int kstep) {
        pa = A + 2 * (p.parts_a >> (4 * product) & 15) * p.a.plane + kstep * a_step;
        pb = B + 2 * (p.parts_b >> (4 * product) & 15) * p.b.plane + kstep * b_step;
        k_left = (int)(p.K - (int64_t)kstep * STEP);
    };
    auto advance = [&] {
        pa += a_step;
        pb += b_step;
        k_left -= STEP;
        --steps_left;
        if (__builtin_expect(k_left <= 0, 0)) {
            product = min(product + 1, p.products - 1);
            begin_product(0);
        }
    };
    auto load = [&](char* la, char* lb) {
        const int have = steps_left > 0 ? k_left : 0;
#pragma unroll
        for (int i = 0; i < TA::LOADS; ++i) ta.load(pa, have, la, wave, i);
#pragma unroll
        for (int i = 0; i < TB::LOADS; ++i) tb.load(pb, have, lb, wave, i);
        advance();
    };
    auto begin_tile = [&](uint32_t g) {
        uint32_t ti, tj;
        if (EPI == MM_ORTH && p.symmetric)
            tile_above(g, ti, tj);
        else
            tile_of(g, tiles, tr, ts, ti, tj);
        mirror = EPI == MM_ORTH && p.symmetric && ti != tj;
        r0 = (int64_t)ti * SIDE;
        s0 = (int64_t)tj * SIDE;
        ta.init(p.a.ld, p.R - r0);
        tb.init(p.b.ld, p.S - s0);
        A = static_cast<const char*>(p.a.p) + 2 * (bt * p.a.batch + (AMC ? r0 : r0 * p.a.ld));
        B = static_cast<const char*>(p.b.p) + 2 * (bt * p.b.batch + (BMC ? s0 : s0 * p.b.ld));
        product = (int)(t0 / per_product);
        steps_left = count;
        begin_product((int)(t0 % per_product));
        load(la0, lb0);
        load(la1, lb1);
    };

    f32x4 acc[F][F];
    s16x8 a0[F], b0[F], a1[F], b1[F];  // fragments of a step's halves
    auto meet = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    auto product_of = [&](s16x8 a, s16x8 b, f32x4& c) {
        // (b first: a lane then holds four neighbours of one output row)
        if constexpr (IN_PLACE)
            mfma_in_place<T>(b, a, c);
        else
            c = mfma<T>(b, a, c);
    };
    // what wrote the sums is done, whatever reads them comes later
    auto settle = [&] {
        if constexpr (IN_PLACE) {
            auto hold = [&] {
#pragma unroll
                for (int i = 0; i < F; ++i)
#pragma unroll
                    for (int j = 0; j < F; ++j) asm volatile("" : "+a"(acc[i][j]));
            };
            asm volatile("s_nop 15\n\ts_nop 15");
            hold();
        }
    };
    // a step in la, lb, whose first half is in a0, b0; the next one's is left there
    auto step = [&](char* la, char* lb, char* na, char* nb) {
#pragma unroll
        for (int i = 0; i < F; ++i) {
            b1[i] = rb.get(lb, i, 1);
            a1[i] = ra.get(la, i, 1);
#pragma unroll
            for (int j = 0; j < F; ++j) product_of(a0[i], b0[j], acc[i][j]);
        }
        meet();
        const int have = steps_left > 0 ? k_left : 0;
#pragma unroll
        for (int i = 0; i < F; ++i) {
            b0[i] = rb.get(nb, i, 0);
            a0[i] = ra.get(na, i, 0);
#pragma unroll
            for (int l = i * TA::LOADS / F; l < (i + 1) * TA::LOADS / F; ++l) {
                ta.load(pa, have, la, wave, l);
                tb.load(pb, have, lb, wave, l);
            }
#pragma unroll
            for (int j = 0; j < F; ++j) product_of(a1[i], b1[j], acc[i][j]);
        }
        advance();
    };

    uint32_t g = blockIdx.x;
    begin_tile(g);
    while (true) {
        meet();
#pragma unroll
        for (int i = 0; i < F; ++i) {
            b0[i] = rb.get(lb0, i, 0);
            a0[i] = ra.get(la0, i, 0);
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        settle();
        // (steps are taken two by two: behind the last one come zeros)
        for (int t = 0; t < count; t += 2) {
            step(la0, lb0, la1, lb1);
            step(la1, lb1, la0, lb0);
        }
        meet();
        settle();
        const int64_t rt = r0 + wr, st = s0 + ws;
        const bool mirrored = mirror;
        g += gridDim.x;
        if (g < tiles) begin_tile(g);

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
#pragma unroll
            for (int i = 0; i < F; ++i)
                if (i == ph)
#pragma unroll
                    for (int j = 0; j < F; ++j)
                        *(f32x4*)at(lane & 15, j * 4 + (lane >> 4)) = acc[i][j];
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
                        if constexpr (sizeof(TO) == 4)
#pragma unroll 1
                            for (int e = 0; e < 8; ++e) {
                                float x = 0.0f;
#pragma unroll
                                for (int i = 0; i < 8; ++i) x = i == e ? v[q][i] : x;
                                if (!(fabsf(x) < __builtin_inff())) fix(v[q], e, whole_sum(p, bt, r, s8 + e));
                            }
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[q][e] += bias[e];
                        if (p.e.pre) store8(static_cast<TO*>(p.e.pre) + r * p.e.pre_ld + s8, v[q]);
                    }
                    activate<8 * PASSES>(v[0], p.e.act);
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
                if (r >= p.R || s >= (EPI == MM_ORTH && p.o.z ? p.o.z_ld : p.S)) continue;
                const int n = (int)max((int64_t)0, min((int64_t)8, p.S - s));
                if constexpr (EPI == MM_PARTIAL) {
                    // (the rows of the partial sums are padded to 8)
                    float* q = p.partial + ((blockIdx.z * p.splits + blockIdx.y) * p.R + r) * p.partial_ld + s;
                    *(f32x4*)q = *(f32x4*)v;
                    *(f32x4*)(q + 4) = *(f32x4*)(v + 4);
                } else if constexpr (EPI == MM_LINEAR) {
                    if constexpr (sizeof(TO) == 4)
#pragma unroll 1
                        for (int e = 0; e < n; ++e)
                            if (!(fabsf(*(const float*)(at(row, lane % LANES * 2 + e / 4) + e % 4 * 4)) < __builtin_inff()))
                                fix(v, e, whole_sum(p, bt, r, s + e));
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
        if (g >= tiles) break;
    }
#endif
}

template <class T, class TO, int EPI, int SIDE>
hipError_t launch_mm_tile(const Mm& p, hipStream_t stream)
{
    const int64_t tr = (p.R + SIDE - 1) / SIDE, ts = (p.S + SIDE - 1) / SIDE;
    const int64_t tiles = p.symmetric ? tr * (tr + 1) / 2 : tr * ts;
    if (tiles > 0x7fffffffLL || p.batch > 65535) return hipErrorInvalidConfiguration;
    const int64_t fit = (int64_t)device_cu_count() * wgs_per_cu(SIDE);
    const int64_t each = (fit + (int64_t)p.splits * p.batch - 1) / ((int64_t)p.splits * p.batch);
    const dim3 grid((unsigned)(tiles < each ? tiles : each), (unsigned)p.splits, (unsigned)p.batch);
    const dim3 block(256);
    if (p.a.mc)
        if (p.b.mc)
            hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, true, true>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, true, false>), grid, block, 0, stream, p);
    else if (p.b.mc)
        hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, false, true>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((k_mm<T, TO, EPI, SIDE, false, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
