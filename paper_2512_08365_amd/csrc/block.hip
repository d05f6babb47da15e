// block.hip -- host side of the feed-forward block's operators: argument
// checks, plans, workspace carving and launch sequences.  See
// include/magneton.h.

#include "block.hpp"

#include <math.h>

#include <algorithm>

using mag::clear_error;
using mag::set_error;
using mag::set_hip_error;

namespace {

constexpr int64_t MAX_DIM = MAG_MAX_EXTENT;
constexpr int64_t MOST_SPAN = 1LL << 60;   // elements from an array's first to its last: bytes fit 63 bits

size_t element(int dtype) { return dtype == MAG_F32 ? 4 : 2; }
bool known_dtype(int d) { return d == MAG_F32 || d == MAG_F16 || d == MAG_BF16; }
bool known_act(int a) { return a >= MAG_ACT_NONE && a <= MAG_ACT_SILU; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// sequential carving of one workspace (base NULL: only the size)
struct Carve {
    char* base;
    size_t off = 0;
    template <class T = void>
    T* take(size_t bytes)
    {
        char* p = base ? base + off : nullptr;
        off += round_up(bytes, 256);
        return reinterpret_cast<T*>(p);
    }
};

// sizes and strides of a matrix; out: one that is written
int check_shape(const mag_matrix& m, bool out)
{
    if (m.rows < 0 || m.cols < 0 || m.rows > MAX_DIM || m.cols > MAX_DIM)
        return set_error(MAG_E_SIZE, "a matrix extent is negative or exceeds MAG_MAX_EXTENT");
    if (m.rows == 0 || m.cols == 0) return MAG_OK;
    if ((m.rows > 1 && (m.row_stride < 0 || m.row_stride > (1LL << 32))) ||
        (m.cols > 1 && (m.col_stride < 0 || m.col_stride > (1LL << 32))))
        return set_error(MAG_E_SIZE, "a matrix stride is negative or exceeds 2^32 elements");
    const uint64_t last = (m.rows > 1 ? (uint64_t)((m.rows - 1) * m.row_stride) : 0) +
                          (m.cols > 1 ? (uint64_t)((m.cols - 1) * m.col_stride) : 0);
    if (last >= (uint64_t)MOST_SPAN) return set_error(MAG_E_SIZE, "a matrix spans 2^60 elements or more");
    if (out && ((m.cols > 1 && m.col_stride != 1) || (m.rows > 1 && m.row_stride < m.cols)))
        return set_error(MAG_E_SIZE, "an output matrix needs col_stride 1 and rows that do not overlap");
    return MAG_OK;
}

int check_data(const mag_matrix& m, int dtype)
{
    if (m.rows == 0 || m.cols == 0) return MAG_OK;
    if (!m.data) return set_error(MAG_E_NULL, "a matrix's data is NULL");
    if (!aligned(m.data, element(dtype)))
        return set_error(MAG_E_ALIGN, "a matrix is not aligned to its elements");
    return MAG_OK;
}

int check_vector(const void* p, int dtype)
{
    if (p && !aligned(p, element(dtype)))
        return set_error(MAG_E_ALIGN, "a vector is not aligned to its elements");
    return MAG_OK;
}

int check_workspace(const void* ws, size_t have, size_t need)
{
    if (need == 0) return MAG_OK;
    if (!ws) return set_error(MAG_E_NULL, "workspace is NULL");
    if (!aligned(ws, 256)) return set_error(MAG_E_WORKSPACE, "workspace must be 256-byte aligned");
    if (have < need) return set_error(MAG_E_WORKSPACE, "workspace too small");
    return MAG_OK;
}

bool same_shape(const mag_matrix& m, int64_t rows, int64_t cols)
{
    return m.rows == rows && m.cols == cols;
}

#define TRY(expr)                    \
    do {                             \
        const int rc_ = (expr);      \
        if (rc_ != MAG_OK) return rc_; \
    } while (0)
#define TRY_HIP(expr, where)                                      \
    do {                                                          \
        const hipError_t e_ = (expr);                             \
        if (e_ != hipSuccess) return set_hip_error(e_, where);    \
    } while (0)

// ----------------------------------------------------------------- operands

int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
// bytes of an element of a product's operand (kind: MM_*), elements of a packed
// row of n: whole lines of 128 bytes, but for narrow ones (a step's 128 bytes of a
// row are then one line in L2: gradients of 1,000 x 777 by 2,050 half 34.7 us with
// rows of whole 16 bytes, 29.5 us so)
size_t part_size(int kind) { return kind == mag::MM_F32 ? 4 : 2; }
int64_t packed_ld(int64_t n, int kind)
{
    if (kind == mag::MM_F32_PARTS) return n > 32 ? (n + 63) / 64 * 192 : 96;
    const int64_t line = 128 / (int64_t)part_size(kind);
    return n > line ? (n + line - 1) / line * line : up8(n);
}

// The largest ld of an operand (kind: MM_*): a tile's loads have 31 bits for a
// byte's offset from the tile's first one, and reach over a step of the reduction
// (across: its elements are lines) or over the rows of the kind's largest tile.
int64_t most_ld(int kind, bool across)
{
    const bool two_bytes = kind == mag::MM_BF16 || kind == mag::MM_F16;
    const int64_t lines = across ? (two_bytes ? 64 : 32)
                                 : mag::TILE_SIDE[kind == mag::MM_F32         ? mag::TILE_64
                                                  : kind == mag::MM_F32_PARTS ? mag::TILE_128
                                                                              : mag::TILE_256];
    return (1LL << 31) / (lines * (int64_t)part_size(kind));
}

// How a product reads a matrix: where it lies, or as rows packed into the
// workspace (what is cut into parts, and strides, alignments and widths that the
// 16-byte loads do not take).
struct Operand {
    bool packed;
    bool by_cols;      // packed: the matrix's columns are the rows
    size_t bytes;      // of the packed rows
    mag::MmOperand op; // p NULL while packed rows have no place yet
};

// along: the reduction runs along the matrix's columns (else along its rows)
Operand operand(const mag_matrix& m, int kind, bool along)
{
    Operand o{};
    if (kind != mag::MM_F32_PARTS && aligned(m.data, 16)) {
        const int64_t per = 16 / (int64_t)part_size(kind);
        const bool by_rows = (m.cols <= 1 || m.col_stride == 1) && m.cols % per == 0 &&
                             (m.rows <= 1 || (m.row_stride % per == 0 && m.row_stride <= most_ld(kind, !along)));
        const bool by_cols = m.row_stride == 1 && m.rows % per == 0 && m.rows > 1 &&
                             (m.cols <= 1 || (m.col_stride % per == 0 && m.col_stride <= most_ld(kind, along)));
        if (by_rows || by_cols) {
            o.op.p = m.data;
            o.op.ld = by_rows ? (m.rows <= 1 ? 0 : m.row_stride) : (m.cols <= 1 ? 0 : m.col_stride);
            o.op.mc = by_rows != along;
            return o;
        }
    }
    // (packed as it lies: by columns if these are what is contiguous, unless there are
    // too many rows; by rows ld follows from a layer's features and is never too large)
    o.packed = true;
    o.by_cols = m.rows > 1 && m.row_stride == 1 && m.col_stride != 1 &&
                packed_ld(m.rows, kind) <= most_ld(kind, along);
    o.op.ld = packed_ld(o.by_cols ? m.rows : m.cols, kind);
    o.op.mc = o.by_cols == along;
    o.bytes = (size_t)((o.by_cols ? m.cols : m.rows) * o.op.ld) * part_size(kind);
    return o;
}

mag::PackParams packing(const Operand& o, const mag_matrix& m)
{
    mag::PackParams p{};
    p.src = m.data;
    p.rs = o.by_cols ? m.col_stride : m.row_stride;
    p.cs = o.by_cols ? m.row_stride : m.col_stride;
    p.rows = o.by_cols ? m.cols : m.rows;
    p.cols = o.by_cols ? m.rows : m.cols;
    p.dst = const_cast<void*>(o.op.p);
    p.ld = o.op.ld;
    return p;
}

// Tile and splits of R x S x K.
struct Shape {
    int tile;
    int splits;
    double cost;   // estimated, in us
};

// What a workgroup's step, its tile beside the steps, and the call cost, in us:
// alone on a CU, and with a second one (0: there is no room for one).  bfloat16 and
// half are fitted to 148 products of sides 256 to 4,096 by 512 to 8,192 (most within
// 6 %), the others to 256 and 512 workgroups over reductions of 512 and 4,096.
struct TileCost {
    double alone, shared, tile;
};
constexpr double CALL_COST = 2.5;
constexpr double JOIN_COST = 3.5;           // a split product's second launch
constexpr double PARTIAL_BYTES = 4.5e6;     // of partial sums a us, written or read
const TileCost TILE_COST[mag::MM_KINDS][mag::TILES] = {
    // 64 (four steps in LDS), 128, 256
    {{0.165, 0.33, 1.7}, {0.52, 0.77, 4.4}, {1.15, 0.0, 10.0}},   // bfloat16: 64 k a step
    {{0.165, 0.33, 1.7}, {0.52, 0.77, 4.4}, {1.15, 0.0, 10.0}},   // half
    {{0.53, 1.00, 1.8}, {0.0, 0.0, 0.0}, {0.0, 0.0, 0.0}},       // fp32: 32 k
    {{0.35, 0.0, 3.6}, {1.20, 0.0, 10.5}, {0.0, 0.0, 0.0}},      // three parts: 32 k, six products
    {{0.22, 0.36, 1.8}, {0.58, 1.19, 6.5}, {2.13, 0.0, 10.5}},   // two parts: 32 k, three products
};
// (fp32 as it lies is bound by its instruction and gains nothing from a larger
// tile; three parts cost six products of bfloat16 and a pass to cut them, and win
// from some 10 GFLOP on: 2,048 x 1,024 by 4,096 97 to 110 us, as it lies 136 us; 256 x
// 2,048 by 512 21.6 and 14.5 us.)

// The tile and split of the reduction that these costs make fastest: large tiles
// move the least data where there are enough of them for the 256 CUs, small ones
// and splits fill the CUs otherwise (1,024 cubed in bfloat16: 7 us with 64, 12 us
// with 128; 4,096 cubed: 101 us with 256, 113 us with 128).  kind: MM_BF16 ...
Shape choose(int64_t R, int64_t S, int64_t K, int kind, int64_t batch, bool symmetric)
{
    constexpr int64_t CUS = 256;
    const int64_t step = kind == mag::MM_BF16 || kind == mag::MM_F16 ? 64 : 32;
    const int64_t steps = std::max<int64_t>(1, (K + step - 1) / step);
    Shape best{mag::TILE_64, 1, 1e300};
    for (int t = 0; t < mag::TILES; ++t) {
        const TileCost& c = TILE_COST[kind][t];
        if (c.alone == 0.0) continue;
        const int64_t side = mag::TILE_SIDE[t], tr = (R + side - 1) / side;
        const int64_t tiles = (symmetric ? tr * (tr + 1) / 2 : tr * ((S + side - 1) / side)) * batch;
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (t == mag::TILE_256 || steps < 2 * s)) break;
            const int64_t wgs = tiles * s;
            // rounds of two a CU where there is room, then a last one of what is left
            const int64_t pairs = c.shared == 0.0 ? 0 : (wgs + CUS - 1) / (2 * CUS);
            const int64_t single = (std::max<int64_t>(wgs - pairs * 2 * CUS, 0) + CUS - 1) / CUS;
            const double each = (double)((steps + s - 1) / s);
            double cost = CALL_COST + (double)pairs * (each * c.shared + c.tile) +
                          (double)single * (each * c.alone + c.tile);
            if (s > 1) cost += JOIN_COST + 2.0 * (double)s * (double)R * (double)S * (double)batch * 4.0 / PARTIAL_BYTES;
            if (cost < best.cost) best = Shape{t, s, cost};
        }
    }
    return best;
}

// Two products side by side in one launch, in 64 tiles: the workgroups that fit
// are dealt to them so that the slower one is done as early as may be.
struct Together {
    int wgs_dx, wgs_dw;
    double cost;
};
Together choose_two(int64_t M, int64_t N, int64_t K, int kind)
{
    const TileCost& c = TILE_COST[kind][mag::TILE_64];
    const int64_t step = kind == mag::MM_BF16 || kind == mag::MM_F16 ? 64 : 32;
    auto tiles = [](int64_t r, int64_t s) { return (double)((r + 63) / 64) * (double)((s + 63) / 64); };
    const double dx = tiles(M, K), dw = tiles(N, K), slots = c.shared > 0.0 ? 512 : 256;
    const double per_step = dx + dw > 256 && c.shared > 0.0 ? c.shared : c.alone;
    const double one_dx = (double)((N + step - 1) / step) * per_step + c.tile;
    const double one_dw = (double)((M + step - 1) / step) * per_step + c.tile;
    Together best{0, 0, 1e300};
    if (dx + dw <= slots) return Together{(int)dx, (int)dw, CALL_COST + std::max(one_dx, one_dw)};
    for (int w = 8; w < slots; w += 8) {   // (in eights: an XCD keeps its run)
        const double cost = CALL_COST + std::max(ceil(dx / w) * one_dx, ceil(dw / (slots - w)) * one_dw);
        if (cost < best.cost)
            best = Together{(int)std::min<double>(w, dx), (int)std::min<double>(slots - w, dw), cost};
    }
    return best;
}

// The products' kind without parts.
int kind_of(int dtype)
{
    return dtype == MAG_F32 ? mag::MM_F32 : dtype == MAG_F16 ? mag::MM_F16 : mag::MM_BF16;
}

// What packing `n` elements costs, in us: a launch and its bytes (read, and
// written whole or as three parts of two bytes).
double packing_cost(int64_t n, int kind)
{
    if (n == 0) return 0.0;
    return 3.0 + (double)n * (kind == mag::MM_F32_PARTS ? 10.0 : 8.0) / 6.5e6;
}

int launch_linear(const mag::Mm& p, int kind, int tile, hipStream_t stream)
{
    if (p.splits > 1) {
        TRY_HIP(mag::launch_mm_partial(p, kind, tile, stream), "product launch");
        TRY_HIP(mag::launch_mm_join(p, kind == mag::MM_F16 ? MAG_F16 : kind == mag::MM_BF16 ? MAG_BF16 : MAG_F32,
                                    stream),
                "join launch");
        return MAG_OK;
    }
    TRY_HIP(kind == mag::MM_F32_PARTS ? mag::launch_mm_f32_parts(p, tile, stream)
            : kind == mag::MM_F32     ? mag::launch_mm_f32(p, stream)
            : kind == mag::MM_F16     ? mag::launch_mm_f16(p, tile, stream)
                                      : mag::launch_mm_bf16(p, tile, stream),
            "product launch");
    return MAG_OK;
}

int launch_orth(const mag::Mm& p, int tile, hipStream_t stream)
{
    if (p.splits > 1) {
        TRY_HIP(mag::launch_mm_partial(p, mag::MM_HALVES, tile, stream), "product launch");
        TRY_HIP(mag::launch_orth_join(p, stream), "join launch");
        return MAG_OK;
    }
    TRY_HIP(mag::launch_mm_orth(p, tile, stream), "product launch");
    return MAG_OK;
}

size_t partial_bytes(int64_t R, int64_t S, const Shape& s, int64_t batch = 1)
{
    return s.splits > 1 ? (size_t)(batch * s.splits * R * up8(S) * 4) : 0;
}

// ------------------------------------------------------------------- linear

int check_linear(const mag_linear_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    TRY(check_shape(a->x, false));
    TRY(check_shape(a->weight, false));
    if (a->x.cols != a->weight.cols)
        return set_error(MAG_E_SIZE, "x and weight differ in their columns");
    if (a->weight.rows > MAG_MAX_FEATURES || a->weight.cols > MAG_MAX_FEATURES)
        return set_error(MAG_E_SIZE, "in or out exceeds MAG_MAX_FEATURES");
    return MAG_OK;
}

struct LinearPlan {
    int kind;          // MM_*
    bool skinny;       // few rows: operands as they lie, one launch, no workspace
    bool across;       // the weight lies input by output
    Operand x, w;
    Shape shape;
    float* partial;
};

size_t plan_linear(const mag_linear_args* a, void* ws, LinearPlan& pl)
{
    const bool along = a->weight.col_stride == 1 || a->weight.cols <= 1;
    pl.across = !along;
    pl.skinny = a->x.rows <= mag::SKINNY_ROWS && (a->x.col_stride == 1 || a->x.cols <= 1) &&
                (along || a->weight.row_stride == 1 || a->weight.rows <= 1);
    if (pl.skinny) return 0;
    double least = 1e300;
    for (int kind : {kind_of(a->dtype), (int)mag::MM_F32_PARTS}) {
        if (kind == mag::MM_F32_PARTS && a->dtype != MAG_F32) break;
        const Operand x = operand(a->x, kind, true), w = operand(a->weight, kind, true);
        const Shape s = choose(a->x.rows, a->weight.rows, a->x.cols, kind, 1, false);
        const double cost = s.cost + packing_cost((x.packed ? a->x.rows * a->x.cols : 0) +
                                                  (w.packed ? a->weight.rows * a->weight.cols : 0), kind);
        if (cost >= least) break;
        least = cost;
        pl.kind = kind;
        pl.x = x;
        pl.w = w;
        pl.shape = s;
    }
    Carve c{static_cast<char*>(ws)};
    for (Operand* o : {&pl.x, &pl.w})
        if (o->packed) o->op.p = c.take(o->bytes);
    pl.partial = c.take<float>(partial_bytes(a->x.rows, a->weight.rows, pl.shape));
    return c.off;
}

// ------------------------------------------------------------------ backward

struct BackwardPlan {
    int kind;         // MM_*
    bool skinny;      // few rows: dx as a layer of few rows whose weight is the transpose
    bool across;      // ... which lies row by row
    Operand x, w, dy;
    bool own_dz;      // dz in the workspace (else dy is dz)
    mag::MmOperand dz;
    Shape dx, dw;
    Together two;     // both at once, if that costs less
    float* partial;
    float* column_part;
};

size_t plan_backward(const mag_linear_backward_args* a, void* ws, BackwardPlan& pl)
{
    const int64_t M = a->x.rows, N = a->weight.rows, K = a->x.cols;
    pl.across = a->weight.row_stride != 1 && a->weight.rows > 1;
    pl.skinny = M <= mag::SKINNY_ROWS && (!pl.across || a->weight.col_stride == 1 || K <= 1);
    double least = 1e300;
    for (int kind : {kind_of(a->dtype), (int)mag::MM_F32_PARTS}) {
        if (kind == mag::MM_F32_PARTS && (a->dtype != MAG_F32 || pl.skinny)) break;
        // x and weight are both read across the reduction of the product they enter
        const Operand x = operand(a->x, kind, false), w = operand(a->weight, kind, false);
        const Shape dx = choose(M, K, N, kind, 1, false), dw = choose(N, K, M, kind, 1, false);
        Together two = choose_two(M, N, K, kind);
        if (two.cost > dx.cost + dw.cost || pl.skinny || !x.op.mc || !w.op.mc) two.cost = 0.0;
        const double cost = (two.cost > 0.0 ? two.cost : dx.cost + dw.cost) +
                            packing_cost((x.packed ? M * K : 0) + (w.packed ? N * K : 0), kind);
        if (cost >= least) break;
        least = cost;
        pl.kind = kind;
        pl.x = x;
        pl.w = w;
        pl.dx = dx;
        pl.dw = dw;
        pl.two = two;
    }
    pl.dy = operand(a->dy, pl.kind, true);
    // (as for the sizes: room for dz whether or not dy can stand in for it; dz is read
    // along the reduction by one product and across it by the other)
    pl.own_dz = a->activation != MAG_ACT_NONE || pl.dy.packed || !a->dy.data || (pl.skinny && pl.dy.op.mc) ||
                pl.dy.op.ld > most_ld(pl.kind, false);
    if (pl.own_dz) {
        pl.dz = mag::MmOperand{};
        pl.dz.ld = packed_ld(N, pl.kind);
    } else {
        pl.dz = pl.dy.op;
    }
    if (pl.dz.mc) pl.two.cost = 0.0;
    Carve c{static_cast<char*>(ws)};
    if (pl.skinny) {
        pl.w.packed = false;
        pl.dx.splits = 1;
    }
    for (Operand* o : {&pl.x, &pl.w})
        if (o->packed) o->op.p = c.take(o->bytes);
    void* dz = c.take((size_t)(M * packed_ld(N, pl.kind)) * part_size(pl.kind));
    if (pl.own_dz) pl.dz.p = dz;
    pl.column_part = c.take<float>((size_t)(mag::slope_chunks(M, N) * N * 4));
    pl.partial = c.take<float>(std::max(partial_bytes(M, K, pl.dx), partial_bytes(N, K, pl.dw)));
    return c.off;
}

int check_backward(const mag_linear_backward_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    TRY(check_shape(a->x, false));
    TRY(check_shape(a->weight, false));
    if (a->x.cols != a->weight.cols)
        return set_error(MAG_E_SIZE, "x and weight differ in their columns");
    if (a->weight.rows > MAG_MAX_FEATURES || a->weight.cols > MAG_MAX_FEATURES)
        return set_error(MAG_E_SIZE, "in or out exceeds MAG_MAX_FEATURES");
    return MAG_OK;
}

// ---------------------------------------------------------------- layer norm

int check_norm(const mag_norm_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    if (a->weight_dtype != a->dtype && a->weight_dtype != MAG_F32)
        return set_error(MAG_E_SIZE, "weight_dtype must be dtype or MAG_F32");
    TRY(check_shape(a->x, false));
    if (a->x.cols < 1 || a->x.cols > MAG_MAX_FEATURES)
        return set_error(MAG_E_SIZE, "width out of [1, MAG_MAX_FEATURES]");
    return MAG_OK;
}

size_t norm_bytes(const mag_norm_args* a)
{
    return (size_t)mag::norm_parts(a->x.rows, a->x.cols, a->dtype) * 2 * (size_t)a->x.cols * 4;
}

// ------------------------------------------------------------- orthogonalize

// g's orientation is kept: X is g or its transpose, read either way
struct OrthPlan {
    int64_t m, n;       // sides of X, m <= n
    int64_t ld, lda;    // of g's rows and of A's and B's, two parts each
    Shape gram, square, whole;  // of A = X X^T, A A and B X
    float* partial;
    int chunks;         // sums of squares of a matrix
    double* part;
    mag::f16* X[2];
    mag::f16* side[4];  // of m x m: A, and what the steps on that side need
    bool grouped;       // several steps on that side are less work than one by one
};

size_t plan_orth(const mag_orthogonalize_args* a, void* ws, OrthPlan& pl)
{
    pl.m = std::min(a->g.rows, a->g.cols);
    pl.n = std::max(a->g.rows, a->g.cols);
    pl.ld = (a->g.cols + 31) / 32 * 64;
    pl.lda = (pl.m + 31) / 32 * 64;
    pl.gram = choose(pl.m, pl.m, pl.n, mag::MM_HALVES, a->batch, true);
    pl.square = choose(pl.m, pl.m, pl.m, mag::MM_HALVES, a->batch, true);
    pl.whole = choose(a->g.rows, a->g.cols, pl.m, mag::MM_HALVES, a->batch, false);
    Carve c{static_cast<char*>(ws)};
    // (8,192 elements each, 1,024 in all the batch: a few rounds of the device)
    const int64_t most = std::max<int64_t>(1, 1024 / std::max<int64_t>(a->batch, 1));
    pl.chunks = (int)std::min<int64_t>(most, (a->g.rows * a->g.cols + 8191) / 8192);
    pl.chunks = std::max(pl.chunks, 1);
    pl.part = c.take<double>((size_t)(a->batch * pl.chunks * 8));
    for (auto& x : pl.X) x = c.take<mag::f16>((size_t)(a->batch * a->g.rows * pl.ld * 2));
    // (a step more on that side takes four products there, on its own one and the
    // two long ones)
    pl.grouped = a->dtype != MAG_F32 && pl.gram.cost + pl.whole.cost > 3.0 * pl.square.cost;
    for (int i = 0; i < 4; ++i)
        pl.side[i] = i < 2 || pl.grouped ? c.take<mag::f16>((size_t)(a->batch * pl.m * pl.lda * 2)) : nullptr;
    pl.partial = c.take<float>(std::max({partial_bytes(pl.m, pl.m, pl.gram, a->batch),
                                         partial_bytes(pl.m, pl.m, pl.square, a->batch),
                                         partial_bytes(a->g.rows, a->g.cols, pl.whole, a->batch)}));
    return c.off;
}

int check_orth(const mag_orthogonalize_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    if (a->batch < 0 || a->batch > 65535) return set_error(MAG_E_SIZE, "batch out of [0, 65535]");
    if (a->steps < 0 || a->steps > MAG_ORTH_MAX_STEPS)
        return set_error(MAG_E_SIZE, "steps out of [0, MAG_ORTH_MAX_STEPS]");
    TRY(check_shape(a->g, false));
    if (a->g.rows > MAG_MAX_FEATURES || a->g.cols > MAG_MAX_FEATURES)
        return set_error(MAG_E_SIZE, "a side exceeds MAG_MAX_FEATURES");
    if (a->g_batch_stride < 0 || a->g_batch_stride > MOST_SPAN / std::max<int64_t>(a->batch, 1))
        return set_error(MAG_E_SIZE, "g_batch_stride out of range");
    return MAG_OK;
}

// the largest |a s + b s^3 + c s^5| over 0 <= s <= u (at an end, or where the
// slope a + 3 b s^2 + 5 c s^4 is zero)
double most_of_polynomial(double a, double b, double c, double u)
{
    auto f = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    double top = f(u);
    const double disc = 9.0 * b * b - 20.0 * a * c;
    const double q = -0.5 * (3.0 * b + (b < 0.0 ? -1.0 : 1.0) * sqrt(std::max(disc, 0.0)));
    if (disc >= 0.0)
        for (double t : {q / (5.0 * c), a / q})
            if (t > 0.0 && t < u * u) top = std::max(top, f(sqrt(t)));
    return top;
}

// How many steps from step i on are done on the short side.  With Q the product of
// their U = a I + b A + c A A, X <- Q X is all that is as long as X, and the next
// A is U A U: of 2,048 x 8,192, three steps and two are 40 products of a side
// cubed where five single ones are 65 (1,660 and 1,190 us).  What an A so made
// costs is accuracy: its rounding, 2^-21 of the largest eigenvalue, grows by the
// slope of one step's map of eigenvalues, l (a + b l + c l l)^2, from step to step
// and enters U times the slope of that.  A quarter of the result's own rounding is
// let through (bfloat16: three steps by the usual coefficients, half: two; fp32
// results go one by one).
int orth_group(const mag_orthogonalize_args* a, const OrthPlan& pl, int i, const double* most)
{
    if (!pl.grouped) return 1;
    const double allowed = a->dtype == MAG_BF16 ? 0x1p-11 : 0x1p-14;
    double error = 0x1p-21, bound = 1.0;
    int group = 1;
    for (int j = i; j < a->steps; ++j) {
        const double u2 = most[j] * most[j];
        double slope = 0.0, growth = 1.0;
        for (int k = 0; k <= 128; ++k) {
            const double l = u2 * k / 128.0, q = a->a + l * (a->b + l * a->c), dq = a->b + 2.0 * a->c * l;
            slope = std::max(slope, fabs(dq));
            growth = std::max(growth, fabs(q * (q + 2.0 * l * dq)));
        }
        bound *= fabs(a->a) + fabs(a->b) * u2 + fabs(a->c) * u2 * u2;
        if (j > i && (error * slope > allowed || bound > 0x1p40)) break;
        group = j - i + 1;
        error *= 1.05 * growth;
    }
    return group;
}

}  // namespace

extern "C" {

int mag_linear_workspace_size(const mag_linear_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_linear(args));
    LinearPlan pl;
    *bytes = plan_linear(args, nullptr, pl);
    return MAG_OK;
}

int mag_linear(const mag_linear_args* a, void* workspace, size_t workspace_bytes,
               hipStream_t stream)
{
    clear_error();
    TRY(check_linear(a));
    if (!known_act(a->activation)) return set_error(MAG_E_SIZE, "unknown activation");
    const int64_t M = a->x.rows, N = a->weight.rows, K = a->x.cols;
    if (!same_shape(a->y, M, N)) return set_error(MAG_E_SIZE, "y must be [rows, out]");
    TRY(check_shape(a->y, true));
    if (a->residual.data) {
        if (!same_shape(a->residual, M, N))
            return set_error(MAG_E_SIZE, "residual must be [rows, out]");
        TRY(check_shape(a->residual, false));
        TRY(check_data(a->residual, a->dtype));
    }
    if (a->pre.data) {
        if (!same_shape(a->pre, M, N)) return set_error(MAG_E_SIZE, "pre must be [rows, out]");
        TRY(check_shape(a->pre, true));
        TRY(check_data(a->pre, a->dtype));
    }
    TRY(check_data(a->x, a->dtype));
    TRY(check_data(a->weight, a->dtype));
    TRY(check_data(a->y, a->dtype));
    TRY(check_vector(a->bias, a->dtype));
    LinearPlan pl;
    TRY(check_workspace(workspace, workspace_bytes, plan_linear(a, nullptr, pl)));
    if (M == 0 || N == 0) return MAG_OK;
    plan_linear(a, workspace, pl);
    mag::Epilogue e{};
    e.bias = a->bias;
    e.act = a->activation;
    e.res = a->residual.data;
    e.res_rs = a->residual.row_stride;
    e.res_cs = a->residual.col_stride;
    e.pre = a->pre.data;
    e.pre_ld = a->pre.row_stride;
    e.y = a->y.data;
    e.y_ld = a->y.row_stride;
    if (pl.skinny) {
        mag::SkinnyParams s{};
        s.x = a->x.data;
        s.x_ld = a->x.row_stride;
        s.w = a->weight.data;
        s.w_ld = pl.across ? a->weight.col_stride : a->weight.row_stride;
        s.across = pl.across;
        s.M = M;
        s.N = N;
        s.K = K;
        s.e = e;
        TRY_HIP(mag::launch_skinny(s, a->dtype, stream), "linear launch");
        return MAG_OK;
    }
    const mag::PackParams px = packing(pl.x, a->x), pw = packing(pl.w, a->weight);
    TRY_HIP(mag::launch_prepare(pl.x.packed ? &px : nullptr, pl.w.packed ? &pw : nullptr, nullptr,
                                pl.kind, stream),
            "linear launch");
    mag::Mm p{};
    p.in_parts = pl.kind == mag::MM_F32_PARTS;
    p.a = pl.x.op;
    p.b = pl.w.op;
    p.R = M;
    p.S = N;
    p.K = K;
    p.batch = 1;
    p.splits = pl.shape.splits;
    p.partial = pl.partial;
    p.partial_ld = up8(N);
    p.e = e;
    p.e.vec = !e.res || e.res_cs == 1;
    return launch_linear(p, pl.kind, pl.shape.tile, stream);
}

int mag_linear_backward_workspace_size(const mag_linear_backward_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_backward(args));
    BackwardPlan pl;
    *bytes = plan_backward(args, nullptr, pl);
    return MAG_OK;
}

int mag_linear_backward(const mag_linear_backward_args* a, void* workspace, size_t workspace_bytes,
                        hipStream_t stream)
{
    clear_error();
    TRY(check_backward(a));
    if (!known_act(a->activation)) return set_error(MAG_E_SIZE, "unknown activation");
    const int64_t M = a->x.rows, N = a->weight.rows, K = a->x.cols;
    if (!same_shape(a->dy, M, N)) return set_error(MAG_E_SIZE, "dy must be [rows, out]");
    TRY(check_shape(a->dy, false));
    TRY(check_data(a->dy, a->dtype));
    if (a->activation != MAG_ACT_NONE) {
        if (!same_shape(a->pre, M, N)) return set_error(MAG_E_SIZE, "pre must be [rows, out]");
        TRY(check_shape(a->pre, false));
        TRY(check_data(a->pre, a->dtype));
    }
    if (a->dx.data) {
        if (!same_shape(a->dx, M, K)) return set_error(MAG_E_SIZE, "dx must be [rows, in]");
        TRY(check_shape(a->dx, true));
        TRY(check_data(a->dx, a->dtype));
        TRY(check_data(a->weight, a->dtype));
    }
    if (a->dweight.data) {
        if (!same_shape(a->dweight, N, K)) return set_error(MAG_E_SIZE, "dweight must be [out, in]");
        TRY(check_shape(a->dweight, true));
        TRY(check_data(a->dweight, a->dtype));
        TRY(check_data(a->x, a->dtype));
    }
    TRY(check_vector(a->dbias, a->dtype));
    BackwardPlan pl;
    TRY(check_workspace(workspace, workspace_bytes, plan_backward(a, nullptr, pl)));
    if (N == 0 && !a->dx.data) return MAG_OK;
    plan_backward(a, workspace, pl);
    if (pl.own_dz || a->dbias) {
        mag::SlopeParams s{};
        s.dy = a->dy.data;
        s.dy_rs = a->dy.row_stride;
        s.dy_cs = a->dy.col_stride;
        s.pre = a->pre.data;
        s.pre_rs = a->pre.row_stride;
        s.pre_cs = a->pre.col_stride;
        s.M = M;
        s.N = N;
        s.act = a->activation;
        s.dz = pl.own_dz && (a->dx.data || a->dweight.data) ? const_cast<void*>(pl.dz.p) : nullptr;
        s.ldz = pl.dz.ld;
        s.dbias = a->dbias;
        s.part = pl.column_part;
        TRY_HIP(mag::launch_slope(s, pl.kind, stream), "linear_backward launch");
    }
    const bool dx = a->dx.data && M > 0 && K > 0, dw = a->dweight.data && N > 0 && K > 0;
    const mag::PackParams px = packing(pl.x, a->x), pw = packing(pl.w, a->weight);
    const mag::ColumnSums sums{pl.column_part, mag::slope_chunks(M, N), N, a->dbias};
    TRY_HIP(mag::launch_prepare(dw && pl.x.packed ? &px : nullptr, dx && pl.w.packed ? &pw : nullptr,
                                a->dbias ? &sums : nullptr, pl.kind, stream),
            "linear_backward launch");
    mag::Mm p{};
    p.in_parts = pl.kind == mag::MM_F32_PARTS;
    p.batch = p.splits = 1;
    p.partial = pl.partial;
    p.partial_ld = up8(K);
    p.S = K;
    p.e.vec = 1;
    mag::Mm q = p;
    p.a = q.a = pl.dz;
    q.a.mc = !pl.dz.mc;
    p.b = pl.w.op;
    p.R = M;
    p.K = N;
    p.e.y = a->dx.data;
    p.e.y_ld = a->dx.row_stride;
    q.b = pl.x.op;
    q.R = N;
    q.K = M;
    q.e.y = a->dweight.data;
    q.e.y_ld = a->dweight.row_stride;
    if (dx && dw && pl.two.cost > 0.0) {
        TRY_HIP(mag::launch_mm_two(p, q, pl.kind, pl.two.wgs_dx, pl.two.wgs_dw, stream),
                "linear_backward launch");
        return MAG_OK;
    }
    if (dx && pl.skinny) {
        mag::SkinnyParams s{};
        s.x = pl.dz.p;
        s.x_ld = pl.dz.ld;
        s.w = a->weight.data;
        s.w_ld = pl.across ? a->weight.row_stride : a->weight.col_stride;
        s.across = pl.across;
        s.M = M;
        s.N = K;
        s.K = N;
        s.e.y = a->dx.data;
        s.e.y_ld = a->dx.row_stride;
        TRY_HIP(mag::launch_skinny(s, a->dtype, stream), "linear_backward launch");
    } else if (dx) {
        p.splits = pl.dx.splits;
        TRY(launch_linear(p, pl.kind, pl.dx.tile, stream));
    }
    if (dw) {
        q.splits = pl.dw.splits;
        TRY(launch_linear(q, pl.kind, pl.dw.tile, stream));
    }
    return MAG_OK;
}

int mag_layer_norm(const mag_norm_args* a, hipStream_t stream)
{
    clear_error();
    TRY(check_norm(a));
    const int64_t M = a->x.rows, N = a->x.cols;
    if (!same_shape(a->y, M, N)) return set_error(MAG_E_SIZE, "y must be [rows, width]");
    TRY(check_shape(a->y, true));
    if (!(a->eps >= 0.0) || isinf(a->eps)) return set_error(MAG_E_SIZE, "eps must be finite and >= 0");
    TRY(check_data(a->x, a->dtype));
    TRY(check_data(a->y, a->dtype));
    TRY(check_vector(a->weight, a->weight_dtype));
    TRY(check_vector(a->bias, a->weight_dtype));
    TRY(check_vector(a->mean, MAG_F32));
    TRY(check_vector(a->rstd, MAG_F32));
    mag::NormParams p{};
    p.x = a->x.data;
    p.x_rs = a->x.row_stride;
    p.x_cs = a->x.col_stride;
    p.y = a->y.data;
    p.y_ld = a->y.row_stride;
    p.M = M;
    p.N = N;
    p.weight = a->weight;
    p.bias = a->bias;
    p.mean = a->mean;
    p.rstd = a->rstd;
    p.eps = (float)a->eps;
    TRY_HIP(mag::launch_norm(p, a->dtype, a->weight_dtype, stream), "layer_norm launch");
    return MAG_OK;
}

int mag_layer_norm_backward_workspace_size(const mag_norm_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_norm(args));
    *bytes = norm_bytes(args);
    return MAG_OK;
}

int mag_layer_norm_backward(const mag_norm_args* a, void* workspace, size_t workspace_bytes,
                            hipStream_t stream)
{
    clear_error();
    TRY(check_norm(a));
    const int64_t M = a->x.rows, N = a->x.cols;
    if (!same_shape(a->dy, M, N)) return set_error(MAG_E_SIZE, "dy must be [rows, width]");
    TRY(check_shape(a->dy, false));
    TRY(check_data(a->x, a->dtype));
    TRY(check_data(a->dy, a->dtype));
    if (a->dx.data) {
        if (!same_shape(a->dx, M, N)) return set_error(MAG_E_SIZE, "dx must be [rows, width]");
        TRY(check_shape(a->dx, true));
        TRY(check_data(a->dx, a->dtype));
    }
    if (M > 0 && (!a->mean || !a->rstd)) return set_error(MAG_E_NULL, "mean and rstd are needed");
    TRY(check_vector(a->weight, a->weight_dtype));
    TRY(check_vector(a->dweight, a->weight_dtype));
    TRY(check_vector(a->dbias, a->weight_dtype));
    TRY(check_vector(a->mean, MAG_F32));
    TRY(check_vector(a->rstd, MAG_F32));
    TRY(check_workspace(workspace, workspace_bytes, norm_bytes(a)));
    mag::NormParams p{};
    p.part = static_cast<float*>(workspace);
    p.x = a->x.data;
    p.x_rs = a->x.row_stride;
    p.x_cs = a->x.col_stride;
    p.dy = a->dy.data;
    p.dy_rs = a->dy.row_stride;
    p.dy_cs = a->dy.col_stride;
    p.y = a->dx.data;
    p.y_ld = a->dx.row_stride;
    p.M = M;
    p.N = N;
    p.weight = a->weight;
    p.mean = a->mean;
    p.rstd = a->rstd;
    p.dweight = a->dweight;
    p.dbias = a->dbias;
    TRY_HIP(mag::launch_norm_backward(p, a->dtype, a->weight_dtype, stream),
            "layer_norm_backward launch");
    return MAG_OK;
}

int mag_orthogonalize_workspace_size(const mag_orthogonalize_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_orth(args));
    OrthPlan pl;
    *bytes = plan_orth(args, nullptr, pl);
    return MAG_OK;
}

int mag_orthogonalize(const mag_orthogonalize_args* a, void* workspace, size_t workspace_bytes,
                      hipStream_t stream)
{
    clear_error();
    TRY(check_orth(a));
    if (!same_shape(a->out, a->g.rows, a->g.cols)) return set_error(MAG_E_SIZE, "out must be [rows, cols]");
    TRY(check_shape(a->out, true));
    if (a->batch > 1 && a->out_batch_stride <
                            (a->out.rows - 1) * (a->out.rows > 1 ? a->out.row_stride : 0) + a->out.cols)
        return set_error(MAG_E_SIZE, "the matrices of out overlap");
    if (a->batch > 1 && a->out_batch_stride > MOST_SPAN / a->batch)
        return set_error(MAG_E_SIZE, "out_batch_stride out of range");
    if (!isfinite(a->a) || !isfinite(a->b) || !isfinite(a->c) || !(a->eps >= 0.0) || isinf(a->eps))
        return set_error(MAG_E_SIZE, "coefficients must be finite and eps finite and >= 0");
    // bounds of X's singular values step by step, and with them of its elements
    double most[MAG_ORTH_MAX_STEPS + 1] = {1.001};
    for (int i = 0; i < a->steps; ++i) {
        most[i + 1] = 1.001 * most_of_polynomial(a->a, a->b, a->c, most[i]);
        const double u2 = most[i] * most[i];
        if (!(most[i + 1] < 0x1p60 && fabs(a->b) * u2 + fabs(a->c) * u2 * u2 < 0x1p60))
            return set_error(MAG_E_SIZE, "the polynomial grows past 2^60 over these steps");
    }
    if (a->batch == 0 || a->g.rows == 0 || a->g.cols == 0) return MAG_OK;
    TRY(check_data(a->g, a->dtype));
    TRY(check_data(a->out, a->dtype));
    OrthPlan pl;
    TRY(check_workspace(workspace, workspace_bytes, plan_orth(a, nullptr, pl)));
    plan_orth(a, workspace, pl);
    const bool tall = a->g.rows > a->g.cols;
    const int64_t m = pl.m, n = pl.n;
    const int64_t x_batch = a->g.rows * pl.ld;
    const int64_t a_batch = m * pl.lda;
    // halves hold a value times a power of two that takes its bound near 2^15 (bounds
    // from 2^-100 on: a polynomial that contracts takes them to zero)
    auto scale_for = [](double bound) { return ldexp(1.0, 15 - ilogb(std::max(bound, 0x1p-100)) - 1); };

    mag::OrthParams o{};
    o.g = a->g.data;
    o.g_batch = a->g_batch_stride;
    o.g_rs = a->g.row_stride;
    o.g_cs = a->g.col_stride;
    o.batch = a->batch;
    o.rows = a->g.rows;
    o.cols = a->g.cols;
    o.eps = a->eps;
    o.part = pl.part;
    o.chunks = pl.chunks;
    double sx = scale_for(most[0]);
    if (a->steps > 0) {
        o.scale = (float)sx;
        o.z = pl.X[0];
        o.z_ld = pl.ld;
        o.z_batch = x_batch;
    } else {
        o.scale = 1.0f;
        o.out = a->out.data;
        o.out_ld = a->out.row_stride;
        o.out_batch = a->out_batch_stride;
    }
    TRY_HIP(mag::launch_orth_begin(o, a->dtype, stream), "orthogonalize launch");
    const mag::MmOperand side[4] = {{pl.side[0], pl.lda, a_batch, 0}, {pl.side[1], pl.lda, a_batch, 0},
                                    {pl.side[2], pl.lda, a_batch, 0}, {pl.side[3], pl.lda, a_batch, 0}};
    mag::Mm p{};
    p.batch = (int)a->batch;
    p.partial = pl.partial;
    auto symmetric = [&](const mag::MmOperand& x, const mag::MmOperand& y, int64_t k, double scale, int z,
                         const Shape& shape) {
        p.a = x;
        p.b = y;
        p.R = p.S = m;
        p.K = k;
        p.symmetric = 1;
        p.partial_ld = up8(m);
        p.splits = shape.splits;
        p.o.scale = (float)scale;
        p.o.z = pl.side[z];
        p.o.z_ld = pl.lda;
        p.o.z_batch = a_batch;
        const int rc = launch_orth(p, shape.tile, stream);
        p.o.m = nullptr;
        p.o.diagonal = 0.0f;
        return rc;
    };
    auto mixed = [&](const mag::MmOperand& x, double mix) {
        p.o.m = static_cast<const mag::f16*>(x.p);
        p.o.m_ld = x.ld;
        p.o.m_batch = x.batch;
        p.o.mix = (float)mix;
    };
    constexpr int A = 0;
    for (int i = 0, from = 0; i < a->steps; from ^= 1) {
        const int group = orth_group(a, pl, i, most);
        mag::MmOperand X{pl.X[from], pl.ld, x_batch, 0};
        // A = X X^T
        X.mc = tall;
        double sa = scale_for(1.01 * most[i] * most[i]);
        TRY(symmetric(X, X, n, sa / (sx * sx), A, pl.gram));
        // Q: what X is multiplied by, without `rest` I
        int q = 1;
        double sq = 0.0, rest = a->a, bound = 1.0;
        for (int j = i; j < i + group; ++j) {
            const double u2 = most[j] * most[j];
            const double of_u = fabs(a->b) * u2 + fabs(a->c) * u2 * u2 + (group > 1 ? fabs(a->a) : 0.0);
            const double su = scale_for(1.01 * of_u);
            // U = b A + c A A, of a group a I + b A + c A A
            const int u = j == i ? 1 : q % 3 + 1;
            mixed(side[A], a->b * su / sa);
            if (group > 1) p.o.diagonal = (float)(a->a * su);
            TRY(symmetric(side[A], side[A], m, a->c * su / (sa * sa), u, pl.square));
            const int other = 6 - q - u;   // (of 1, 2 and 3, where q and u differ)
            bound *= of_u;
            if (j == i) {
                sq = su;
            } else {
                // Q <- U Q
                const double next = scale_for(1.01 * bound);
                TRY(symmetric(side[u], side[q], m, next / (su * sq), other, pl.square));
                sq = next;
                q = other;
            }
            if (j + 1 < i + group) {
                // A <- U A U
                const int t = u == q ? u % 3 + 1 : 6 - q - u;
                const double st = scale_for(1.01 * most[j] * most[j + 1]);
                const double next = scale_for(1.01 * most[j + 1] * most[j + 1]);
                TRY(symmetric(side[u], side[A], m, st / (su * sa), t, pl.square));
                TRY(symmetric(side[u], side[t], m, next / (su * st), A, pl.square));
                sa = next;
            }
        }
        if (group > 1) rest = 0.0;
        i += group;
        // X <- rest X + Q X, or its transpose <- rest X^T + X^T Q (Q symmetric)
        const bool last = i == a->steps;
        const double next = scale_for(most[i]), out = last ? 1.0 : next;
        X.mc = 0;
        if (rest != 0.0) mixed(X, rest * out / sx);
        p.symmetric = 0;
        p.a = tall ? X : side[q];
        p.b = tall ? side[q] : X;
        p.b.mc = !tall;
        p.R = a->g.rows;
        p.S = a->g.cols;
        p.K = m;
        p.partial_ld = up8(a->g.cols);
        p.splits = pl.whole.splits;
        p.o.scale = (float)(out / (sq * sx));
        p.o.z = last ? nullptr : pl.X[from ^ 1];
        p.o.z_ld = pl.ld;
        p.o.z_batch = x_batch;
        p.o.out = a->out.data;
        p.o.out_ld = a->out.row_stride;
        p.o.out_batch = a->out_batch_stride;
        p.o.dtype = a->dtype;
        TRY(launch_orth(p, pl.whole.tile, stream));
        p.o.m = nullptr;
        sx = next;
    }
    return MAG_OK;
}

}  // extern "C"
