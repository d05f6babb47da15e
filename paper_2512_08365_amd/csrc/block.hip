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
    // (the last element's offset stays far inside 63 bits)
    if ((m.rows > 1 && (m.row_stride < 0 || m.row_stride > (1LL << 32))) ||
        (m.cols > 1 && (m.col_stride < 0 || m.col_stride > (1LL << 32))))
        return set_error(MAG_E_SIZE, "a matrix stride is negative or exceeds 2^32 elements");
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

// ------------------------------------------------------------------- linear

int check_linear(const mag_linear_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    TRY(check_shape(a->x, false));
    TRY(check_shape(a->weight, false));
    if (a->x.cols != a->weight.cols)
        return set_error(MAG_E_SIZE, "x and weight differ in their columns");
    return MAG_OK;
}

// ------------------------------------------------------------------ backward

struct BackwardWorkspace {
    void* dz;
};

size_t carve_backward(const mag_linear_backward_args* a, void* ws, BackwardWorkspace& w)
{
    Carve c{static_cast<char*>(ws)};
    w.dz = c.take((size_t)a->x.rows * a->weight.rows * element(a->dtype));
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
    if (a->x.cols < 1) return set_error(MAG_E_SIZE, "width must be >= 1");
    return MAG_OK;
}

// ------------------------------------------------------------- orthogonalize

struct OrthWorkspace {
    float* X[2];
    float* A;
    float* B;
};

size_t carve_orth(const mag_orthogonalize_args* a, void* ws, OrthWorkspace& w)
{
    const size_t m = (size_t)std::min(a->g.rows, a->g.cols), n = (size_t)std::max(a->g.rows, a->g.cols);
    Carve c{static_cast<char*>(ws)};
    for (auto& x : w.X) x = c.take<float>((size_t)a->batch * m * n * 4);
    w.A = c.take<float>((size_t)a->batch * m * m * 4);
    w.B = c.take<float>((size_t)a->batch * m * m * 4);
    return c.off;
}

int check_orth(const mag_orthogonalize_args* a)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (!known_dtype(a->dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    if (a->batch < 0 || a->batch > MAX_DIM) return set_error(MAG_E_SIZE, "batch out of range");
    if (a->steps < 0 || a->steps > MAG_ORTH_MAX_STEPS)
        return set_error(MAG_E_SIZE, "steps out of [0, MAG_ORTH_MAX_STEPS]");
    TRY(check_shape(a->g, false));
    if (a->g_batch_stride < 0 || a->g_batch_stride > (1LL << 62) / std::max<int64_t>(a->batch, 1))
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

}  // namespace

extern "C" {

int mag_linear_workspace_size(const mag_linear_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_linear(args));
    *bytes = 0;
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
    (void)workspace;
    (void)workspace_bytes;
    mag::Product p{};
    p.a = a->x.data;
    p.b = a->weight.data;
    p.R = M;
    p.S = N;
    p.K = K;
    p.batch = 1;
    p.a_rs = a->x.row_stride;
    p.a_ks = a->x.col_stride;
    p.b_ss = a->weight.row_stride;
    p.b_ks = a->weight.col_stride;
    p.e.scale = 1.0f;
    p.e.bias = a->bias;
    p.e.act = a->activation;
    p.e.res = a->residual.data;
    p.e.res_rs = a->residual.row_stride;
    p.e.res_cs = a->residual.col_stride;
    p.e.pre = a->pre.data;
    p.e.pre_ld = a->pre.row_stride;
    p.e.y = a->y.data;
    p.e.y_ld = a->y.row_stride;
    TRY_HIP(mag::launch_product(p, a->dtype, stream), "linear launch");
    return MAG_OK;
}

int mag_linear_backward_workspace_size(const mag_linear_backward_args* args, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_backward(args));
    BackwardWorkspace w;
    *bytes = carve_backward(args, nullptr, w);
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
    BackwardWorkspace w;
    TRY(check_workspace(workspace, workspace_bytes, carve_backward(a, nullptr, w)));
    carve_backward(a, workspace, w);
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
    s.dz = w.dz;
    s.ldz = N;
    s.dbias = a->dbias;
    TRY_HIP(mag::launch_slope(s, a->dtype, stream), "linear_backward launch");
    mag::Product p{};
    p.batch = 1;
    p.e.scale = 1.0f;
    p.a = w.dz;
    if (a->dx.data) {
        p.R = M;
        p.S = K;
        p.K = N;
        p.a_rs = N;
        p.a_ks = 1;
        p.b = a->weight.data;
        p.b_ss = a->weight.col_stride;
        p.b_ks = a->weight.row_stride;
        p.e.y = a->dx.data;
        p.e.y_ld = a->dx.row_stride;
        TRY_HIP(mag::launch_product(p, a->dtype, stream), "linear_backward launch");
    }
    if (a->dweight.data) {
        p.R = N;
        p.S = K;
        p.K = M;
        p.a_rs = 1;
        p.a_ks = N;
        p.b = a->x.data;
        p.b_ss = a->x.col_stride;
        p.b_ks = a->x.row_stride;
        p.e.y = a->dweight.data;
        p.e.y_ld = a->dweight.row_stride;
        TRY_HIP(mag::launch_product(p, a->dtype, stream), "linear_backward launch");
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
    *bytes = 0;
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
    (void)workspace;
    (void)workspace_bytes;
    mag::NormParams p{};
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
    OrthWorkspace w;
    *bytes = carve_orth(args, nullptr, w);
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
    if (!isfinite(a->a) || !isfinite(a->b) || !isfinite(a->c) || !(a->eps >= 0.0) || isinf(a->eps))
        return set_error(MAG_E_SIZE, "coefficients must be finite and eps finite and >= 0");
    double most = 1.0;  // bounds X's singular values, and with them its elements
    for (int i = 0; i < a->steps; ++i) {
        most = 1.001 * most_of_polynomial(a->a, a->b, a->c, most);
        if (!(most < 0x1p60)) return set_error(MAG_E_SIZE, "the polynomial grows past 2^60 over these steps");
    }
    if (a->batch == 0 || a->g.rows == 0 || a->g.cols == 0) return MAG_OK;
    TRY(check_data(a->g, a->dtype));
    TRY(check_data(a->out, a->dtype));
    OrthWorkspace w;
    TRY(check_workspace(workspace, workspace_bytes, carve_orth(a, nullptr, w)));
    carve_orth(a, workspace, w);
    const bool tall = a->g.rows > a->g.cols;
    const int64_t m = std::min(a->g.rows, a->g.cols), n = std::max(a->g.rows, a->g.cols);
    mag::OrthParams o{};
    o.g = a->g.data;
    o.g_batch = a->g_batch_stride;
    o.g_rs = tall ? a->g.col_stride : a->g.row_stride;
    o.g_cs = tall ? a->g.row_stride : a->g.col_stride;
    o.out = a->out.data;
    o.out_batch = a->out_batch_stride;
    o.out_rs = tall ? 1 : a->out.row_stride;
    o.out_cs = tall ? a->out.row_stride : 1;
    o.batch = a->batch;
    o.m = m;
    o.n = n;
    o.eps = a->eps;
    o.X = w.X[0];
    TRY_HIP(mag::launch_orth_begin(o, a->dtype, stream), "orthogonalize launch");
    for (int i = 0; i < a->steps; ++i) {
        float* X = w.X[i & 1];
        mag::Product p{};
        p.batch = a->batch;
        p.a_rs = p.b_ss = n;
        p.a_ks = p.b_ks = 1;
        p.a = p.b = X;
        p.a_batch = p.b_batch = m * n;
        p.R = p.S = m;
        p.K = n;
        p.y_batch = p.mixed_batch = m * m;
        p.e.scale = 1.0f;
        p.e.y = w.A;
        p.e.y_ld = m;
        TRY_HIP(mag::launch_product(p, MAG_F32, stream), "orthogonalize launch");
        p.a = p.b = w.A;
        p.a_rs = p.b_ss = m;
        p.a_batch = p.b_batch = m * m;
        p.K = m;
        p.e.scale = (float)a->c;
        p.e.mix = (float)a->b;
        p.e.mixed = w.A;
        p.e.mixed_ld = m;
        p.e.y = w.B;
        TRY_HIP(mag::launch_product(p, MAG_F32, stream), "orthogonalize launch");
        p.a = w.B;
        p.b = X;
        p.b_ss = 1;
        p.b_ks = n;
        p.b_batch = m * n;
        p.S = n;
        p.e.scale = 1.0f;
        p.e.mix = (float)a->a;
        p.e.mixed = X;
        p.e.mixed_ld = n;
        p.mixed_batch = p.y_batch = m * n;
        p.e.y = o.X = w.X[(i + 1) & 1];
        p.e.y_ld = n;
        TRY_HIP(mag::launch_product(p, MAG_F32, stream), "orthogonalize launch");
    }
    TRY_HIP(mag::launch_orth_end(o, a->dtype, stream), "orthogonalize launch");
    return MAG_OK;
}

}  // extern "C"
