// step.hip -- host side of the norms around a block and of clipped gradients: argument
// checks, workspace carving and launch sequences.  See include/magneton.h.

#include "step.hpp"

#include <float.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "block_host.hpp"

namespace {

// ------------------------------------------------------------- residual norms

mag::Strided strided(const mag_matrix& m) { return {m.data, m.rows > 1 ? m.row_stride : 0, m.cols > 1 ? m.col_stride : 1}; }

// what both passes have: types, sizes, the gate
int check_residual_norm(int dtype, int weight_dtype, int gate_dtype, int kind, int post, const mag_matrix& x,
                        const mag_matrix& gate)
{
    if (!known_dtype(dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
    if (weight_dtype != dtype && weight_dtype != MAG_F32)
        return set_error(MAG_E_SIZE, "weight_dtype must be dtype or MAG_F32");
    if (kind != MAG_NORM_LAYER && kind != MAG_NORM_RMS) return set_error(MAG_E_SIZE, "unknown kind of norm");
    if (post != 0 && post != 1) return set_error(MAG_E_SIZE, "post must be 0 or 1");
    TRY(check_shape(x, false));
    if (x.cols < 1 || x.cols > MAG_MAX_FEATURES) return set_error(MAG_E_SIZE, "width out of [1, MAG_MAX_FEATURES]");
    if (!gate.data) return MAG_OK;
    if (gate_dtype != dtype && gate_dtype != MAG_F32) return set_error(MAG_E_SIZE, "gate_dtype must be dtype or MAG_F32");
    TRY(check_shape(gate, false));
    if (gate.cols != x.cols || gate.rows < 1) return set_error(MAG_E_SIZE, "gate must be [groups, width]");
    if (x.rows % gate.rows) return set_error(MAG_E_SIZE, "the rows are no whole number of the gate's groups");
    if (gate.cols > 1 && gate.col_stride != 1) return set_error(MAG_E_SIZE, "the gate's columns must be neighbours");
    return check_data(gate, gate_dtype);
}

int check_same(const mag_matrix& m, const mag_matrix& x, bool out, int dtype)
{
    if (!same_shape(m, x.rows, x.cols)) return set_error(MAG_E_SIZE, "matrices must be [rows, width]");
    TRY(check_shape(m, out));
    return check_data(m, dtype);
}

int check_scale(double scale)
{
    if (!(fabs(scale) <= FLT_MAX)) return set_error(MAG_E_SIZE, "scale must be finite in fp32");
    return MAG_OK;
}

// (two outputs that begin together; where they overlap otherwise is not looked at)
int check_apart(const mag_matrix& a, const mag_matrix& b)
{
    if (a.data && a.data == b.data && a.rows > 0 && a.cols > 0)
        return set_error(MAG_E_SIZE, "two outputs are the same memory");
    return MAG_OK;
}

void take_gate(mag::ResidualNorm& p, const mag_matrix& gate, int gate_dtype)
{
    p.gate = gate.data;
    p.gate_ld = gate.rows > 1 ? gate.row_stride : 0;
    p.gate_f32 = gate_dtype == MAG_F32;
    p.groups = gate.data ? gate.rows : 1;
    p.length = p.M / p.groups;
}

// of a backward pass over rows of any strides
size_t backward_bytes(const mag_matrix& x, const mag_matrix& gate)
{
    mag::ResidualNorm p{};
    p.M = x.rows;
    p.N = x.cols;
    take_gate(p, gate, MAG_F32);
    p.h = p.y = p.dn = p.dr = {&p, 0, 1};
    const int held = mag::residual_norm_parts(p).parts;
    p.h.cs = 2;
    const int wide = mag::residual_norm_parts(p).parts;
    return round_up((size_t)std::max(held, wide) * 5 * (size_t)p.N * 4, 256) + (size_t)p.M * 16;
}

// -------------------------------------------------------------------- clipping

struct Range {
    int64_t from, to;             // bytes: of the first row's begin and the last one's end
    int64_t rows, pitch, width;   // bytes
    bool out;
};

Range range_of(const void* p, int64_t count, int64_t cols, int64_t ld, size_t size, bool out)
{
    const int64_t at = (int64_t)reinterpret_cast<uintptr_t>(p), e = (int64_t)size;
    if (!cols || count <= cols || ld == cols) return {at, at + count * e, 1, 0, count * e, out};
    const int64_t rows = count / cols;
    return {at, at + ((rows - 1) * ld + cols) * e, rows, ld * e, cols * e, out};
}

// The least x >= 0 with l <= a x mod m <= r, of 0 < l <= r < m and 0 <= a < m, or -1.
// Where no multiple of a lies in [l, r] itself, a x - m y in [l, r] is m y mod a in
// [-r, -l] mod a: the same with a and at most half of it, as Euclid's algorithm.
__int128 first_within(__int128 a, __int128 m, __int128 l, __int128 r)
{
    if (a == 0) return -1;
    if (2 * a > m) return first_within(m - a, m, m - r, m - l);
    const __int128 x = (l + a - 1) / a;
    if (a * x <= r) return x;
    const __int128 y = first_within((a - m % a) % a, a, l % a, r % a);
    return y < 0 ? y : (l + m * y + a - 1) / a;
}

int64_t modulo(int64_t a, int64_t m) { return (a % m + m) % m; }

// whether two tensors share a byte
bool meet(const Range& a, const Range& b)
{
    if (a.to <= b.from || b.to <= a.from) return false;
    if (a.rows == 1 && b.rows > 1) return meet(b, a);
    // a's rows that reach into the stretch from b's first byte to its last one
    const int64_t d = a.from - b.from, span = b.to - b.from;
    int64_t first = 0, last = a.rows - 1;
    if (a.rows > 1) {
        if (d + a.width <= 0) first = -(d + a.width) / a.pitch + 1;
        last = std::min(last, (span - 1 - d) / a.pitch);
    }
    if (first > last) return false;
    if (b.rows == 1 || d + first * a.pitch < 0 || d + last * a.pitch >= span - b.width) return true;
    // each of them begins in a row of b, ends in the next one, or lies between the two
    const int64_t free = b.pitch - a.width - b.width;
    if (free < 0) return true;
    const int64_t at = modulo(d + first * a.pitch - b.width, b.pitch);   // (of the first, behind a row's end)
    const int64_t l = modulo(free + 1 - at, b.pitch), r = modulo(b.pitch - 1 - at, b.pitch);
    if (l > r || l == 0) return true;
    const __int128 x = first_within(a.pitch % b.pitch, b.pitch, l, r);
    return x >= 0 && x <= last - first;
}

int check_list(const mag_tensors_args* a, bool scaled)
{
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    if (a->n < 0 || a->n > MAG_MAX_TENSORS) return set_error(MAG_E_SIZE, "n out of [0, MAG_MAX_TENSORS]");
    if (a->n > 0 && !a->tensors) return set_error(MAG_E_NULL, "tensors is NULL");
    if (a->kind != MAG_NORM_TWO && a->kind != MAG_NORM_INF) return set_error(MAG_E_SIZE, "unknown kind of norm");
    for (int64_t i = 0; i < a->n; ++i) {
        const mag_tensor_ref& t = a->tensors[i];
        if (!known_dtype(t.dtype)) return set_error(MAG_E_SIZE, "unknown dtype");
        if (t.count < 0 || t.count > (1LL << 36)) return set_error(MAG_E_SIZE, "a tensor's count is out of [0, 2^36]");
        if (t.count == 0) continue;
        if (t.cols < 0 || (t.cols && t.count % t.cols)) return set_error(MAG_E_SIZE, "a tensor is no whole number of rows");
        for (int64_t ld : {t.in_stride, t.out_stride})
            if (t.cols && t.count > t.cols && (ld < t.cols || ld > (1LL << 32)))
                return set_error(MAG_E_SIZE, "a tensor's rows overlap or are more than 2^32 elements apart");
        for (int64_t ld : {t.in_stride, t.out_stride})
            if (t.cols && t.count > t.cols && t.count / t.cols - 1 >= (MOST_SPAN - t.cols) / ld)
                return set_error(MAG_E_SIZE, "a tensor spans 2^60 elements or more");
        if (!t.in || (scaled && !t.out)) return set_error(MAG_E_NULL, "a tensor's data is NULL");
        if (!aligned(t.in, element(t.dtype)) || (scaled && !aligned(t.out, element(t.dtype))))
            return set_error(MAG_E_ALIGN, "a tensor is not aligned to its elements");
    }
    return MAG_OK;
}

// What is written may be its own tensor, and meets nothing else.
int check_overlap(const mag_tensors_args* a)
{
    std::vector<Range> r;
    r.reserve((size_t)a->n * 2);
    for (int64_t i = 0; i < a->n; ++i) {
        const mag_tensor_ref& t = a->tensors[i];
        if (t.count == 0) continue;
        const size_t size = element(t.dtype);
        r.push_back(range_of(t.out, t.count, t.cols, t.out_stride, size, true));
        if (t.in != t.out || (t.cols && t.count > t.cols && t.in_stride != t.out_stride))
            r.push_back(range_of(t.in, t.count, t.cols, t.in_stride, size, false));
    }
    std::sort(r.begin(), r.end(), [](const Range& x, const Range& y) { return x.from < y.from; });
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = i + 1; j < r.size() && r[j].from < r[i].to; ++j)
            if ((r[i].out || r[j].out) && meet(r[i], r[j]))
                return set_error(MAG_E_SIZE, "an output overlaps another tensor of the list");
    return MAG_OK;
}

// The list as launches' arguments: f(spans) for every 64 tensors that have elements.
template <class F>
int each_launch(const mag_tensors_args* a, F f)
{
    mag::Spans s;
    s.n = 0;
    s.chunks = 0;
    for (int64_t i = 0; i <= a->n; ++i) {
        if (s.n == mag::SPANS || (i == a->n && s.n > 0)) {
            TRY(f(s));
            s.n = 0;
            s.chunks = 0;
        }
        if (i == a->n) break;
        const mag_tensor_ref& t = a->tensors[i];
        if (t.count == 0) continue;
        const int64_t chunks = (t.count + mag::CHUNK - 1) / mag::CHUNK;
        mag::Span& p = s.span[s.n++];
        const bool apart = t.cols && t.count > t.cols && (t.in_stride != t.cols || t.out_stride != t.cols);
        p.in = t.in;
        p.out = t.out;
        p.count = t.count;
        p.cols = apart ? t.cols : 0;
        p.in_ld = t.in_stride;
        p.out_ld = t.out_stride;
        p.dtype = t.dtype;
        p.first = s.chunks;
        s.chunks += (uint32_t)chunks;   // (at most 64 times 2^23)
    }
    return MAG_OK;
}

int wgs_of(uint32_t chunks) { return (int)std::min<uint32_t>(chunks, mag::CLIP_WGS); }

size_t parts_of(const mag_tensors_args* a)
{
    size_t parts = 0;
    (void)each_launch(a, [&](const mag::Spans& s) { return parts += (size_t)wgs_of(s.chunks), MAG_OK; });
    return parts;
}

int run_list(const mag_tensors_args* a, bool scaled, void* workspace, size_t bytes, hipStream_t stream)
{
    TRY(check_list(a, scaled));
    if (scaled && !(a->max_norm >= 0.0 && isfinite(a->max_norm) && a->eps >= 0.0 && isfinite(a->eps)))
        return set_error(MAG_E_SIZE, "max_norm and eps must be finite and >= 0");
    if (!a->norm && !scaled) return set_error(MAG_E_NULL, "norm is NULL");
    TRY(check_vector(a->norm, MAG_F32));
    if (scaled) try {
            TRY(check_overlap(a));
        } catch (const std::bad_alloc&) {
            return set_error(MAG_E_SIZE, "no host memory to compare the tensors' places");
        }
    const size_t parts = parts_of(a);
    TRY(check_workspace(workspace, bytes, parts * 8));
    double* part = static_cast<double*>(workspace);
    const bool inf = a->kind == MAG_NORM_INF;
    size_t at = 0;
    TRY(each_launch(a, [&](const mag::Spans& s) {
        TRY_HIP(mag::launch_clip_norm(s, part + at, wgs_of(s.chunks), inf, stream), "norm launch");
        at += (size_t)wgs_of(s.chunks);
        return MAG_OK;
    }));
    if (!scaled || parts == 0) {
        mag::Spans none;
        none.n = 0;
        none.chunks = 0;
        if (a->norm)
            TRY_HIP(mag::launch_clip_scale(none, part, (int)parts, 1, inf, 0.0, 0.0, a->norm, stream), "norm launch");
        return MAG_OK;
    }
    bool first = true;
    return each_launch(a, [&](const mag::Spans& s) {
        TRY_HIP(mag::launch_clip_scale(s, part, (int)parts, wgs_of(s.chunks), inf, a->max_norm, a->eps,
                                       first ? a->norm : nullptr, stream),
                "clip_gradients launch");
        first = false;
        return MAG_OK;
    });
}

}  // namespace

extern "C" {

int mag_residual_norm(const mag_residual_norm_args* a, hipStream_t stream)
{
    clear_error();
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    TRY(check_residual_norm(a->dtype, a->weight_dtype, a->gate_dtype, a->kind, a->post, a->residual, a->gate));
    TRY(check_data(a->residual, a->dtype));
    TRY(check_same(a->branch, a->residual, false, a->dtype));
    TRY(check_same(a->out, a->residual, true, a->dtype));
    TRY(check_same(a->normed, a->residual, true, a->dtype));
    TRY(check_apart(a->out, a->normed));
    if (!(a->eps >= 0.0 && a->eps <= FLT_MAX)) return set_error(MAG_E_SIZE, "eps must be >= 0 and finite in fp32");
    TRY(check_scale(a->scale));
    if (!a->post && (a->post_weight || a->post_bias))
        return set_error(MAG_E_SIZE, "post_weight and post_bias belong to a norm of the branch");
    for (const void* v : {a->weight, a->bias, a->post_weight, a->post_bias}) TRY(check_vector(v, a->weight_dtype));
    for (const float* v : {a->mean, a->rstd, a->post_mean, a->post_rstd}) TRY(check_vector(v, MAG_F32));
    mag::ResidualNorm p{};
    p.h = strided(a->residual);
    p.y = strided(a->branch);
    p.out = a->out.data;
    p.out_ld = a->out.row_stride;
    p.normed = a->normed.data;
    p.normed_ld = a->normed.row_stride;
    p.M = a->residual.rows;
    p.N = a->residual.cols;
    take_gate(p, a->gate, a->gate_dtype);
    p.rms = a->kind == MAG_NORM_RMS;
    p.post = a->post;
    p.weight_f32 = a->weight_dtype == MAG_F32;
    p.weight = a->weight;
    p.bias = a->bias;
    p.post_weight = a->post_weight;
    p.post_bias = a->post_bias;
    p.mean = a->mean;
    p.rstd = a->rstd;
    p.post_mean = a->post_mean;
    p.post_rstd = a->post_rstd;
    p.scale = (float)a->scale;
    p.eps = (float)a->eps;
    TRY_HIP(mag::launch_residual_norm(p, a->dtype, stream), "residual_norm launch");
    return MAG_OK;
}

int mag_residual_norm_backward_workspace_size(const mag_residual_norm_backward_args* a, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    TRY(check_residual_norm(a->dtype, a->weight_dtype, a->gate_dtype, a->kind, a->post, a->residual, a->gate));
    *bytes = backward_bytes(a->residual, a->gate);
    return MAG_OK;
}

int mag_residual_norm_backward(const mag_residual_norm_backward_args* a, void* workspace, size_t workspace_bytes,
                               hipStream_t stream)
{
    clear_error();
    if (!a) return set_error(MAG_E_NULL, "args is NULL");
    TRY(check_residual_norm(a->dtype, a->weight_dtype, a->gate_dtype, a->kind, a->post, a->residual, a->gate));
    const mag_matrix& x = a->residual;
    TRY(check_data(x, a->dtype));
    TRY(check_same(a->branch, x, false, a->dtype));
    TRY(check_same(a->d_normed, x, false, a->dtype));
    if (a->d_out.data) TRY(check_same(a->d_out, x, false, a->dtype));
    if (a->d_residual.data) TRY(check_same(a->d_residual, x, true, a->dtype));
    if (a->d_branch.data) TRY(check_same(a->d_branch, x, true, a->dtype));
    TRY(check_apart(a->d_residual, a->d_branch));
    TRY(check_scale(a->scale));
    const bool layer = a->kind == MAG_NORM_LAYER;
    if (x.rows > 0 && (!a->rstd || (layer && !a->mean) || (a->post && (!a->post_rstd || (layer && !a->post_mean)))))
        return set_error(MAG_E_NULL, "the norms' statistics are needed");
    if (!a->post && (a->post_weight || a->post_bias || a->dpost_weight || a->dpost_bias))
        return set_error(MAG_E_SIZE, "post_weight and post_bias belong to a norm of the branch");
    for (const void* v : {a->weight, a->post_weight, a->post_bias, (const void*)a->dweight, (const void*)a->dbias,
                          (const void*)a->dpost_weight, (const void*)a->dpost_bias})
        TRY(check_vector(v, a->weight_dtype));
    for (const float* v : {a->mean, a->rstd, a->post_mean, a->post_rstd}) TRY(check_vector(v, MAG_F32));
    if (a->d_gate.data) {
        if (!a->gate.data) return set_error(MAG_E_SIZE, "d_gate without a gate");
        if (!same_shape(a->d_gate, a->gate.rows, a->gate.cols)) return set_error(MAG_E_SIZE, "d_gate must be [groups, width]");
        TRY(check_shape(a->d_gate, true));
        TRY(check_data(a->d_gate, a->gate_dtype));
    }
    TRY(check_workspace(workspace, workspace_bytes, backward_bytes(x, a->gate)));
    mag::ResidualNorm p{};
    p.h = strided(x);
    p.y = strided(a->branch);
    p.dn = strided(a->d_normed);
    if (a->d_out.data) p.dr = strided(a->d_out);
    p.out = a->d_residual.data;
    p.out_ld = a->d_residual.row_stride;
    p.normed = a->d_branch.data;
    p.normed_ld = a->d_branch.row_stride;
    p.M = x.rows;
    p.N = x.cols;
    take_gate(p, a->gate, a->gate_dtype);
    p.rms = !layer;
    p.post = a->post;
    p.weight_f32 = a->weight_dtype == MAG_F32;
    p.weight = a->weight;
    p.post_weight = a->post_weight;
    p.post_bias = a->post_bias;
    p.mean = const_cast<float*>(a->mean);
    p.rstd = const_cast<float*>(a->rstd);
    p.post_mean = const_cast<float*>(a->post_mean);
    p.post_rstd = const_cast<float*>(a->post_rstd);
    p.scale = (float)a->scale;
    p.d_gate = a->d_gate.data;
    p.d_gate_ld = a->d_gate.row_stride;
    p.dweight = a->dweight;
    p.dbias = a->dbias;
    p.dpost_weight = a->dpost_weight;
    p.dpost_bias = a->dpost_bias;
    const mag::RowParts parts = mag::residual_norm_parts(p);
    p.parts = parts.parts;
    p.chunks = parts.chunks;
    Carve c{static_cast<char*>(workspace)};
    p.part = c.take<float>((size_t)p.parts * 5 * (size_t)p.N * 4);
    p.rows = c.take<float>((size_t)p.M * 16);
    TRY_HIP(mag::launch_residual_norm_backward(p, a->dtype, stream), "residual_norm_backward launch");
    return MAG_OK;
}

int mag_clip_gradients_workspace_size(const mag_tensors_args* a, size_t* bytes)
{
    clear_error();
    if (!bytes) return set_error(MAG_E_NULL, "bytes is NULL");
    TRY(check_list(a, false));
    *bytes = parts_of(a) * 8;
    return MAG_OK;
}

int mag_gradient_norm(const mag_tensors_args* a, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    clear_error();
    return run_list(a, false, workspace, workspace_bytes, stream);
}

int mag_clip_gradients(const mag_tensors_args* a, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    clear_error();
    return run_list(a, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
