// fp8.hip -- host side of the 8-bit operands' quantization and linear layers: argument
// checks, plans, workspace carving and launch sequences.  See include/magneton.h.

#include "fp8.hpp"

#include <math.h>

#include <algorithm>

#include "block_host.hpp"

namespace {

constexpr int64_t MOST_LD = 1LL << 23;          // a tile's offsets have 31 bits
constexpr int64_t MOST_SCALE_ROW = 1LL << 22;   // floats from a row's scale to the next one's

bool known_format(int f) { return f == MAG_E4M3 || f == MAG_E5M2; }
int64_t blocks_of(int64_t n) { return (n + MAG_FP8_BLOCK - 1) / MAG_FP8_BLOCK; }

int check_bytes(const mag_matrix& m)
{
    if (m.rows > 0 && m.cols > 0 && !m.data) return set_error(MAG_E_NULL, "a matrix's data is NULL");
    return MAG_OK;
}

// scales that are read
int check_scales(const mag_matrix& m)
{
    TRY(check_shape(m, false));
    if (m.rows > 1 && m.row_stride > MOST_SCALE_ROW)
        return set_error(MAG_E_SIZE, "scales of neighbouring rows are more than 2^22 floats apart");
    return check_data(m, MAG_F32);
}

// scales that are written, by rows or by columns
int check_scales_out(const mag_matrix& m, int64_t rows, int64_t cols)
{
    if (!same_shape(m, rows, cols)) return set_error(MAG_E_SIZE, "scales must be one a block");
    TRY(check_shape(m, false));
    const bool by_rows = (m.cols <= 1 || m.col_stride == 1) && (m.rows <= 1 || m.row_stride >= m.cols);
    const bool by_cols = (m.rows <= 1 || m.row_stride == 1) && (m.cols <= 1 || m.col_stride >= m.rows);
    if (!by_rows && !by_cols)
        return set_error(MAG_E_SIZE, "scales need one stride of 1 and lines that do not overlap");
    return check_data(m, MAG_F32);
}

mag::Scales scales(const mag_matrix& m)
{
    return {static_cast<float*>(m.data), m.rows > 1 ? m.row_stride : 0, m.cols > 1 ? m.col_stride : 0};
}

// ------------------------------------------------------------------- linear

int check_linear(const mag_linear_fp8_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    TRY(check_shape(a->x, false));
    TRY(check_shape(a->weight, false));
    if (a->x.cols != a->weight.cols) return set_error(MAG_E_SIZE, "x and weight differ in their columns");
    if (a->weight.rows > MAG_MAX_FEATURES || a->weight.cols > MAG_MAX_EXTENT)
        return set_error(MAG_E_SIZE, "out exceeds MAG_MAX_FEATURES");
    return MAG_OK;
}

// what a tile product reads where it lies: rows along the reduction at multiples of 16 bytes
bool in_place(const mag_matrix& m)
{
    return aligned(m.data, 16) && (m.cols <= 1 || m.col_stride == 1) &&
           (m.rows <= 1 || (m.row_stride % 16 == 0 && m.row_stride < MOST_LD));
}

// bytes of a packed row: whole lines of 128, but for narrow ones
int64_t packed_ld(int64_t n) { return (int64_t)(n > 128 ? round_up((size_t)n, 128) : round_up((size_t)n, 16)); }

// What a workgroup's step, its tile beside the steps, and the call cost, in us, with
// the CU to itself and with others on it.  Of 44 sizes (33 to 16,384 rows, reductions of
// 128 to 16,384, 64 to 16,384 outputs), every tile and split timed: what these choose is
// within 3% of the fastest at 37 and 18% slower at the worst (7,781 x 208 by 1,842: tiles
// of 256, 19.6 us, where tiles of 64 take 16.7); beyond the 8 us of the host's call they
// foretell 7% more to 25% less than is measured, 11% less in the middle.
struct TileCost {
    int per_cu;
    double step, tile;   // (of as many as fit)
};
const TileCost TILE_COST[mag::TILES] = {{4, 0.60, 3.0}, {2, 1.0, 5.0}, {1, 1.6, 9.0}};
constexpr double CALL_COST = 2.5, JOIN_COST = 3.5;
constexpr double PARTIAL_BYTES = 4.5e6;   // of partial sums a us, written or read

struct Plan {
    bool skinny;
    bool pack_x, pack_w;
    int64_t ld_x, ld_w;
    uint8_t *x, *w;
    // tiles: the reduction in `slabs` launches of `slab` each (the last one what is left)
    int64_t slab;
    int slabs;
    int tile, splits;   // splits: of a slab
    float* partial;     // of slabs x splits
};

void choose(int64_t R, int64_t S, int64_t K, Plan& pl)
{
    constexpr int64_t CUS = 256;
    const int64_t steps = std::max<int64_t>(1, blocks_of(K));
    double least = 1e300;
    for (int t = 0; t < mag::TILES; ++t) {
        const TileCost& c = TILE_COST[t];
        const int64_t side = mag::TILE_SIDE[t];
        const int64_t tiles = ((R + side - 1) / side) * ((S + side - 1) / side);
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > 1 && steps < 2 * s) break;
            const int64_t wgs = tiles * s, fit = CUS * c.per_cu;
            const double each = (double)((steps + s - 1) / s);
            // a last round of fewer workgroups takes a share of a full one's time
            const int64_t full = wgs / fit, rest = (wgs % fit + CUS - 1) / CUS;
            const double share = rest ? 0.4 + 0.6 * (double)rest / c.per_cu : 0.0;
            double cost = CALL_COST + ((double)full + share) * (each * c.step + c.tile);
            if (s > 1) cost += JOIN_COST + 2.0 * (double)s * (double)R * (double)S * 4.0 / PARTIAL_BYTES;
            if (cost < least) least = cost, pl.tile = t, pl.splits = s;
        }
    }
}

size_t plan_linear(const mag_linear_fp8_args* a, void* ws, Plan& pl)
{
    pl = Plan{};
    pl.skinny = a->x.rows <= mag::SKINNY_ROWS;
    pl.pack_x = pl.skinny ? a->x.cols > 1 && a->x.col_stride != 1 : !in_place(a->x);
    pl.pack_w = pl.skinny ? a->weight.cols > 1 && a->weight.col_stride != 1 : !in_place(a->weight);
    // (few rows: 16 bytes of a row at least)
    if (pl.skinny && a->x.cols > 0 && a->x.cols < 16) pl.pack_x = pl.pack_w = true;
    pl.ld_x = pl.pack_x ? packed_ld(a->x.cols) : a->x.rows > 1 ? a->x.row_stride : 0;
    pl.ld_w = pl.pack_w ? packed_ld(a->weight.cols) : a->weight.rows > 1 ? a->weight.row_stride : 0;
    pl.splits = pl.slabs = 1;
    pl.slab = a->x.cols;
    if (!pl.skinny) {
        // Rows whose pitch a tile's offsets do not reach over are packed a part of the
        // reduction at a time, each in the place of the one before.
        if ((pl.pack_x && pl.ld_x >= MOST_LD) || (pl.pack_w && pl.ld_w >= MOST_LD)) {
            constexpr int64_t MOST_SLAB = MOST_LD - MAG_FP8_BLOCK;
            pl.slabs = (int)((a->x.cols + MOST_SLAB - 1) / MOST_SLAB);
            pl.slab = blocks_of((a->x.cols + pl.slabs - 1) / pl.slabs) * MAG_FP8_BLOCK;
            if (pl.pack_x) pl.ld_x = pl.slab;
            if (pl.pack_w) pl.ld_w = pl.slab;
        }
        choose(a->x.rows, a->weight.rows, pl.slab, pl);
    }
    Carve c{static_cast<char*>(ws)};
    pl.x = pl.pack_x ? c.take<uint8_t>((size_t)(a->x.rows * pl.ld_x)) : static_cast<uint8_t*>(a->x.data);
    pl.w = pl.pack_w ? c.take<uint8_t>((size_t)(a->weight.rows * pl.ld_w)) : static_cast<uint8_t*>(a->weight.data);
    if (pl.slabs * pl.splits > 1)
        pl.partial = c.take<float>((size_t)(pl.slabs * pl.splits * a->x.rows * up8(a->weight.rows) * 4));
    return c.off;
}

// columns [from, from + n) of m
int pack(const mag_matrix& m, int64_t from, int64_t n, uint8_t* dst, int64_t ld, hipStream_t stream)
{
    mag::Pack8Params p{};
    p.rs = m.rows > 1 ? m.row_stride : 0;
    p.cs = m.cols > 1 ? m.col_stride : 1;
    p.src = static_cast<const uint8_t*>(m.data) + from * p.cs;
    p.rows = m.rows;
    p.cols = n;
    p.dst = dst;
    p.ld = ld;
    TRY_HIP(mag::launch_pack8(p, stream), "linear_fp8 launch");
    return MAG_OK;
}

}  // namespace

extern "C" {

int mag_quantize_fp8(const mag_quantize_args* a, hipStream_t stream)
{
    clear_error();
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    if (!known_format(a->format)) return set_error(MAG_E_SIZE, "unknown 8-bit format");
    if (a->block_rows != 1 && a->block_rows != MAG_FP8_BLOCK)
        return set_error(MAG_E_SIZE, "block_rows must be 1 or 128");
    const bool square = a->block_rows != 1;
    const int64_t M = a->x.rows, N = a->x.cols;
    TRY(check_shape(a->x, false));
    TRY(check_data(a->x, a->dtype));
    if (a->q.data) {
        if (!same_shape(a->q, M, N)) return set_error(MAG_E_SIZE, "q must be [rows, cols]");
        TRY(check_shape(a->q, true));
        TRY(check_scales_out(a->scale, square ? blocks_of(M) : M, blocks_of(N)));
    }
    if (a->qt.data) {
        if (!same_shape(a->qt, N, M)) return set_error(MAG_E_SIZE, "qt must be [cols, rows]");
        TRY(check_shape(a->qt, true));
        TRY(check_scales_out(a->scale_t, square ? blocks_of(N) : N, blocks_of(M)));
    }
    if (M == 0 || N == 0 || (!a->q.data && !a->qt.data)) return MAG_OK;
    mag::QuantizeParams p{};
    p.x = a->x.data;
    p.rs = M > 1 ? a->x.row_stride : 0;
    p.cs = N > 1 ? a->x.col_stride : 1;
    p.rows = M;
    p.cols = N;
    p.q = static_cast<uint8_t*>(a->q.data);
    p.q_ld = a->q.row_stride;
    p.qt = static_cast<uint8_t*>(a->qt.data);
    p.qt_ld = a->qt.row_stride;
    if (p.q) p.scale = scales(a->scale);
    if (p.qt) p.scale_t = scales(a->scale_t);
    // x stored by columns: its transpose, the outputs in each other's place
    if (p.cs != 1 && p.rs == 1) {
        std::swap(p.rs, p.cs);
        std::swap(p.rows, p.cols);
        std::swap(p.q, p.qt);
        std::swap(p.q_ld, p.qt_ld);
        std::swap(p.scale, p.scale_t);
    }
    TRY_HIP(mag::launch_quantize(p, a->dtype, a->format, square, stream), "quantize_fp8 launch");
    return MAG_OK;
}

int mag_linear_fp8_workspace_size(const mag_linear_fp8_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_linear(args));
    Plan pl;
    *bytes = plan_linear(args, nullptr, pl);
    return MAG_OK;
}

int mag_linear_fp8(const mag_linear_fp8_args* a, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    clear_error();
    TRY(check_linear(a));
    if (a->dtype != MAG_F16 && a->dtype != MAG_BF16) return set_error(MAG_E_SIZE, "dtype must be MAG_F16 or MAG_BF16");
    if (!known_act(a->activation)) return set_error(MAG_E_SIZE, "unknown activation");
    if (!known_format(a->x_format) || !known_format(a->weight_format))
        return set_error(MAG_E_SIZE, "unknown 8-bit format");
    const int64_t M = a->x.rows, N = a->weight.rows, K = a->x.cols;
    if (!same_shape(a->y, M, N)) return set_error(MAG_E_SIZE, "y must be [rows, out]");
    TRY(check_shape(a->y, true));
    if (a->residual.data) {
        if (!same_shape(a->residual, M, N)) return set_error(MAG_E_SIZE, "residual must be [rows, out]");
        TRY(check_shape(a->residual, false));
        TRY(check_data(a->residual, a->dtype));
    }
    if (a->pre.data) {
        if (!same_shape(a->pre, M, N)) return set_error(MAG_E_SIZE, "pre must be [rows, out]");
        TRY(check_shape(a->pre, true));
        TRY(check_data(a->pre, a->dtype));
    }
    if (!same_shape(a->x_scale, M, blocks_of(K)))
        return set_error(MAG_E_SIZE, "x_scale must be [rows, ceil(in / 128)]");
    const bool by_row = a->weight_scale.rows == N && N > 1;
    if (!same_shape(a->weight_scale, by_row ? N : blocks_of(N), blocks_of(K)))
        return set_error(MAG_E_SIZE, "weight_scale must be [ceil(out / 128) or out, ceil(in / 128)]");
    TRY(check_bytes(a->x));
    TRY(check_bytes(a->weight));
    TRY(check_scales(a->x_scale));
    TRY(check_scales(a->weight_scale));
    TRY(check_data(a->y, a->dtype));
    TRY(check_vector(a->bias, a->dtype));
    Plan pl;
    TRY(check_workspace(workspace, workspace_bytes, plan_linear(a, nullptr, pl)));
    if (M == 0 || N == 0) return MAG_OK;
    plan_linear(a, workspace, pl);
    mag::Mm8 p{};
    p.lda = pl.ld_x;
    p.ldb = pl.ld_w;
    p.R = M;
    p.S = N;
    p.by_row = by_row;
    p.fa = a->x_format;
    p.fb = a->weight_format;
    p.splits = pl.splits;
    p.partial_ld = up8(N);
    p.e.bias = a->bias;
    p.e.act = a->activation;
    p.e.res = a->residual.data;
    p.e.res_rs = a->residual.row_stride;
    p.e.res_cs = a->residual.col_stride;
    p.e.pre = a->pre.data;
    p.e.pre_ld = a->pre.row_stride;
    p.e.y = a->y.data;
    p.e.y_ld = a->y.row_stride;
    p.e.vec = !p.e.res || p.e.res_cs == 1;
    const int planes = pl.slabs * pl.splits;
    const int dtype = planes > 1 ? MAG_F32 : a->dtype;
    for (int i = 0; i < pl.slabs; ++i) {
        const int64_t from = i * pl.slab;
        p.K = std::min(pl.slab, K - from);
        p.a = pl.pack_x ? pl.x : pl.x + from;
        p.b = pl.pack_w ? pl.w : pl.w + from;
        p.sa = scales(a->x_scale);
        p.sb = scales(a->weight_scale);
        p.sa.p += from / MAG_FP8_BLOCK * p.sa.cs;
        p.sb.p += from / MAG_FP8_BLOCK * p.sb.cs;
        if (planes > 1) p.partial = pl.partial + (int64_t)i * pl.splits * M * p.partial_ld;
        if (K > 0 && pl.pack_x) TRY(pack(a->x, from, p.K, pl.x, pl.ld_x, stream));
        if (K > 0 && pl.pack_w) TRY(pack(a->weight, from, p.K, pl.w, pl.ld_w, stream));
        if (pl.skinny) {
            if (K > 0) p.K = std::max<int64_t>(K, 16);
            TRY_HIP(mag::launch_skinny8(p, a->dtype, stream), "linear_fp8 launch");
            return MAG_OK;
        }
        TRY_HIP(pl.tile == mag::TILE_256   ? mag::launch_mm8_256(p, dtype, stream)
                : pl.tile == mag::TILE_128 ? mag::launch_mm8_128(p, dtype, stream)
                                           : mag::launch_mm8_64(p, dtype, stream),
                "linear_fp8 launch");
    }
    if (planes > 1) {
        mag::Mm j{};
        j.R = M;
        j.S = N;
        j.K = K;
        j.batch = 1;
        j.splits = planes;
        j.partial = pl.partial;
        j.partial_ld = up8(N);
        j.e = p.e;
        TRY_HIP(mag::launch_mm_join(j, a->dtype, stream), "linear_fp8 launch");
    }
    return MAG_OK;
}

}  // extern "C"
