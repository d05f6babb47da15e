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

// ------------------------------------------------------------------- operands
// A tile of an operand is 64 steps of the reduction by ROWS rows of the output,
// in LDS as 16-byte chunks of 8 elements, filled by loads that go from memory
// to LDS without registers.  Such a load writes 64 chunks one after another, so
// a permutation against bank conflicts is made in what each lane reads.
//   along k (MC false): element (row, k) at row * ld + k.  LDS row of 8 chunks;
//     chunk c of row r sits at c ^ (r & 7), so 8 rows' chunks of one k cover
//     all banks.  Read as they are: 8 consecutive k of a row a lane.
//   along rows (MC true): element at k * ld + row.  LDS row (one k) of ROWS / 8
//     chunks; chunk c of step k sits at c ^ 2 (k & 3).  Read through the
//     transposing LDS load: 16 lanes hand in 4 steps of 16 rows and get 4
//     consecutive k of a row each.
constexpr int STEP = 64;                     // reduction per tile
constexpr uint32_t NOWHERE = 0x80000000u;    // a buffer offset past every extent: reads zeros

template <int ROWS, bool MC, int THREADS>
struct Tile {
    static constexpr int BYTES = ROWS * STEP * 2;
    static constexpr int LOADS = BYTES / 16 / THREADS;  // chunks a thread
    static constexpr int CH = MC ? ROWS / 8 : 8;        // chunks an LDS row

    uint32_t off[LOADS];  // byte offset of the thread's chunks in a tile of the operand
    int kk[LOADS];        // their first k

    // rows of the operand from this tile's first one on; ld in elements
    __device__ void init(int64_t ld, int64_t rows_left)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int f = i * THREADS + (int)threadIdx.x;
            const int line = f / CH, pos = f % CH;
            if constexpr (MC) {
                int c = pos ^ (2 * (line & 3));
                // (rows past the last one: any others, nothing of theirs is stored)
                if ((int64_t)c * 8 >= rows_left) c = 0;
                kk[i] = line;
                off[i] = (uint32_t)(line * ld * 2 + c * 16);
            } else {
                const int c = pos ^ (line & 7);
                const int64_t r = line < rows_left ? line : rows_left - 1;
                kk[i] = c * 8;
                off[i] = (uint32_t)(r * ld * 2 + c * 16);
            }
        }
    }

    // base: the operand at this tile's first row and step's first k; k_left:
    // steps of the reduction from there on
    __device__ __forceinline__ void load(const char* base, int k_left, char* lds) const
    {
        const __amdgpu_buffer_rsrc_t rs =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0x7fffffff, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
        if (k_left >= STEP) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rs, (__attribute__((address_space(3))) void*)(lds + (i * THREADS + wave * 64) * 16),
                    16, off[i], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rs, (__attribute__((address_space(3))) void*)(lds + (i * THREADS + wave * 64) * 16),
                    16, kk[i] < k_left ? off[i] : NOWHERE, 0, 0, 0);
        }
    }
};

// the 16 rows from `row`, 32 steps from 32 s: row lane % 16, k 8 (lane / 16) ..
template <int ROWS, bool MC>
__device__ __forceinline__ s16x8 fragment(const char* lds, int row, int s)
{
    const int lane = (int)threadIdx.x & 63;
    if constexpr (MC) {
        const int q = lane & 15;
        const int k = s * 32 + (lane >> 4) * 8 + (q >> 2);
        const int c = (row >> 3) + ((q & 3) >> 1);
        const int at = ((c ^ (2 * (k & 3))) << 4) + ((q & 1) << 3);
        const char* p = lds + k * (ROWS * 2) + at;  // (k + 4 has the same place in its row)
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(p + 4 * ROWS * 2));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        const int r = row + (lane & 15), c = s * 4 + (lane >> 4);
        return *(const s16x8*)(lds + r * 128 + ((c ^ (r & 7)) << 4));
    }
}

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
        if (e.act != MAG_ACT_NONE)
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = activation(z[i], e.act);
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
            v = activation(v, e.act);
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

// Workgroup number -> tile: the XCDs (workgroups go round them) get runs of
// neighbouring tiles, and a run walks bands of 8 tile rows, so that an XCD's
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

template <class T, class TO, int EPI, int BM, int BN, int WM, int WN, bool AMC, bool BMC>
__global__ __launch_bounds__(WM* WN * 64, BM == 64 ? 4 : 2) void k_mm(Mm p)
{
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int THREADS = WM * WN * 64;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    using TA = Tile<BM, AMC, THREADS>;
    using TB = Tile<BN, BMC, THREADS>;
    // two tiles of each operand, as separate arrays: what one is read from is
    // not what is being filled
    __shared__ __attribute__((aligned(1024))) char la0[TA::BYTES], lb0[TB::BYTES];
    __shared__ __attribute__((aligned(1024))) char la1[TA::BYTES], lb1[TB::BYTES];

    const uint32_t tr = (uint32_t)((p.R + BM - 1) / BM), ts = (uint32_t)((p.S + BN - 1) / BN);
    uint32_t ti, tj;
    if (EPI == MM_ORTH && p.symmetric)
        tile_above(blockIdx.x, ti, tj);
    else
        tile_of(blockIdx.x, tr * ts, tr, ts, ti, tj);
    const int64_t bt = blockIdx.z;
    const int64_t r0 = (int64_t)ti * BM, s0 = (int64_t)tj * BN;
    // this workgroup's share of the steps: all products of parts, K each
    const int per_product = max(1, (int)((p.K + STEP - 1) / STEP));
    const int64_t steps = (int64_t)per_product * p.products;
    const int64_t t0 = steps * blockIdx.y / p.splits, t1 = steps * (blockIdx.y + 1) / p.splits;

    TA ta;
    TB tb;
    ta.init(p.a.ld, p.R - r0);
    tb.init(p.b.ld, p.S - s0);
    const char* A = static_cast<const char*>(p.a.p) +
                    2 * (bt * p.a.batch + (AMC ? r0 : r0 * p.a.ld));
    const char* B = static_cast<const char*>(p.b.p) +
                    2 * (bt * p.b.batch + (BMC ? s0 : s0 * p.b.ld));
    const int64_t a_step = AMC ? STEP * p.a.ld * 2 : STEP * 2;
    const int64_t b_step = BMC ? STEP * p.b.ld * 2 : STEP * 2;
    int product = (int)(t0 / per_product), kstep = (int)(t0 % per_product);
    const char *pa, *pb;
    auto begin_product = [&] {
        pa = A + 2 * (p.parts_a >> (4 * product) & 15) * p.a.plane + kstep * a_step;
        pb = B + 2 * (p.parts_b >> (4 * product) & 15) * p.b.plane + kstep * b_step;
    };
    begin_product();
    const int k_last = (int)(p.K - (int64_t)(per_product - 1) * STEP);  // of a product's last step

    auto load = [&](char* la, char* lb) {
        const bool last = kstep + 1 == per_product;
        const int left = last ? k_last : STEP;
        ta.load(pa, left, la);
        tb.load(pb, left, lb);
        if (last) {
            kstep = 0;
            ++product;
            begin_product();
        } else {
            ++kstep;
            pa += a_step;
            pb += b_step;
        }
    };

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int wr = wave / WN * (BM / WM), ws = wave % WN * (BN / WN);
    f32x4 acc[FM][FN] = {};
    auto multiply = [&](const char* la, const char* lb) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            // (the second half's fragments not before the first half is done
            // with its own: registers)
            if (s) __builtin_amdgcn_sched_barrier(0);
            s16x8 fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = fragment<BM, AMC>(la, wr + i * 16, s);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = fragment<BN, BMC>(lb, ws + j * 16, s);
            // (b first: a lane then holds four neighbours of one output row)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma<T>(fb[j], fa[i], acc[i][j]);
        }
    };
    auto meet = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // meet: what was loaded has arrived, and nobody reads the other tiles any more
    const int count = (int)(t1 - t0);
    if (count > 0) load(la0, lb0);
    int step = 0;
    for (; step + 1 < count; step += 2) {
        meet();
        load(la1, lb1);
        multiply(la0, lb0);
        meet();
        if (step + 2 < count) load(la0, lb0);
        multiply(la1, lb1);
    }
    if (step < count) {
        meet();
        multiply(la0, lb0);
    }

    // The sums go through LDS, where the tiles were, a wave's own part of it at a
    // time: 64 or 32 columns a row, in 16-byte chunks that sit at (chunk ^ row),
    // and come back as 8 neighbours of a row a lane.
    meet();
    constexpr int COLS = BN / WN, CHUNKS = COLS / 4;
    constexpr int WAVES = WM * WN, REGION = 2 * (TA::BYTES + TB::BYTES) / WAVES;
    constexpr int PHASES = (FM * 16 * COLS * 4 + REGION - 1) / REGION, FI = FM / PHASES;
    static_assert(TA::BYTES == TB::BYTES && WAVES % 4 == 0 && FM % PHASES == 0 &&
                  FI * 16 * COLS * 4 <= REGION, "a wave's region lies within one array");
    const int array = wave / (WAVES / 4);
    char* mine = (array == 0 ? la0 : array == 1 ? lb0 : array == 2 ? la1 : lb1) +
                 wave % (WAVES / 4) * REGION;
    auto at = [&](int row, int chunk) { return mine + (row * CHUNKS + (chunk ^ (row & (CHUNKS - 1)))) * 16; };
    const int lane = (int)threadIdx.x & 63;
    const bool mirror = EPI == MM_ORTH && p.symmetric && ti != tj;
#pragma unroll
    for (int ph = 0; ph < PHASES; ++ph) {
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
                *(f32x4*)at(i * 16 + (lane & 15), j * 4 + (lane >> 4)) = acc[ph * FI + i][j];
        const int64_t rp = r0 + wr + ph * FI * 16, sp = s0 + ws;
        constexpr int LANES = COLS / 8;  // of a row
#pragma unroll 1
        for (int row = lane / LANES; row < FI * 16; row += 64 / LANES) {
            const int64_t r = rp + row, s = sp + lane % LANES * 8;
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
        if (EPI == MM_ORTH && mirror) {
            // the transpose: 8 neighbours of a column a lane
#pragma unroll 1
            for (int i = lane; i < COLS * FI * 2; i += 64) {
                const int c = i / (FI * 2), g = i % (FI * 2) * 8;
                const int64_t r = sp + c, s = rp + g;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = *(const float*)(at(g + e, c / 4) + c % 4 * 4);
                if (r >= p.S || s >= p.R) continue;
                store_orth(p, bt, r, s, (int)min((int64_t)8, p.R - s), v);
            }
        }
    }
#endif
}

template <class T, class TO, int EPI, int BM, int BN, int WM, int WN>
hipError_t launch_mm_tile(const Mm& p, hipStream_t stream)
{
    const int64_t tr = (p.R + BM - 1) / BM, ts = (p.S + BN - 1) / BN;
    const int64_t tiles = p.symmetric ? tr * (tr + 1) / 2 : tr * ts;
    if (tiles > 0x7fffffffLL || p.batch > 65535) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)tiles, (unsigned)p.splits, (unsigned)p.batch), block(WM * WN * 64);
    if (p.a.mc)
        if (p.b.mc)
            hipLaunchKernelGGL((k_mm<T, TO, EPI, BM, BN, WM, WN, true, true>), grid, block, 0, stream, p);
        else
            hipLaunchKernelGGL((k_mm<T, TO, EPI, BM, BN, WM, WN, true, false>), grid, block, 0, stream, p);
    else if (p.b.mc)
        hipLaunchKernelGGL((k_mm<T, TO, EPI, BM, BN, WM, WN, false, true>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((k_mm<T, TO, EPI, BM, BN, WM, WN, false, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace mag
