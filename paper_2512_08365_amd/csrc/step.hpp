// step.hpp -- shared definitions of what a training step adds around a block: norms
// fused with its gate, residual scale and addition, and clipped gradients.
#pragma once

#include "block.hpp"

namespace mag {

struct Strided {
    const void* p;
    int64_t rs, cs;
};

// a = post ? N(y) pw + pb : y; out = h + scale gate a; normed = N(out) w + b
struct ResidualNorm {
    Strided h, y;          // backward: out and y
    Strided dn, dr;        // backward: gradients of normed and (or p NULL) of out
    void *out, *normed;    // backward: gradients of h and y, each or NULL
    int64_t out_ld, normed_ld;
    const void* gate;      // [groups][gate_ld], or NULL: ones
    int64_t gate_ld;
    int32_t gate_f32, weight_f32;   // gate, weights and biases are fp32, else of the rows' type
    int32_t rms, post;
    int64_t M, N, groups, length;   // rows, width; groups of `length` rows
    const void *weight, *bias, *post_weight, *post_bias;   // or NULL
    float *mean, *rstd, *post_mean, *post_rstd;            // mean, post_mean: not of an rms norm
    float scale, eps;
    // backward
    void* d_gate;
    int64_t d_gate_ld;
    void *dweight, *dbias, *dpost_weight, *dpost_bias;
    float* part;           // [parts][5][N]: of the four vectors and, with chunks, the gate
    int32_t parts, chunks; // chunks: workgroups a group; 0: whole groups a workgroup
    float* rows;           // [M][4], of rows that no registers hold
};
// how the backward pass deals out its rows
struct RowParts {
    int parts, chunks;
};
RowParts residual_norm_parts(const ResidualNorm& p);
hipError_t launch_residual_norm(const ResidualNorm& p, int dtype, hipStream_t stream);
hipError_t launch_residual_norm_backward(const ResidualNorm& p, int dtype, hipStream_t stream);

// A tensor of a list: `count` elements from `in` to `out`, in rows of `cols` that are
// ld apart (cols 0: neighbours all).
struct Span {
    const void* in;
    void* out;
    int64_t count, cols, in_ld, out_ld;
    int32_t dtype;
    uint32_t first;        // of its chunks, in the launch
};
constexpr int SPANS = 64;          // a launch
constexpr int64_t CHUNK = 8192;    // elements
struct Spans {
    Span span[SPANS];
    int32_t n;
    uint32_t chunks;       // in all
};
constexpr int CLIP_WGS = 1024;
// partial sums (inf: largest magnitudes) of a launch, one a workgroup
hipError_t launch_clip_norm(const Spans& s, double* part, int wgs, bool inf, hipStream_t stream);
// the norm from `parts` of them, and (n > 0) out = in min(1, most / (norm + eps))
hipError_t launch_clip_scale(const Spans& s, const double* part, int parts, int wgs, bool inf, double most,
                             double eps, float* norm, hipStream_t stream);

}  // namespace mag
