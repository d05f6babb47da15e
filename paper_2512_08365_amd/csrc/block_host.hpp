// block_host.hpp -- argument checks and workspace carving that the host sides of the
// block's operators share.
#pragma once

#include "block.hpp"

using mag::clear_error;
using mag::set_error;
using mag::set_hip_error;

namespace {

constexpr int64_t MAX_DIM = MAG_MAX_EXTENT;
constexpr int64_t MOST_SPAN = 1LL << 60;   // elements from an array's first to its last: bytes fit 63 bits

inline size_t element(int dtype) { return dtype == MAG_F32 ? 4 : 2; }
inline bool known_dtype(int d) { return d == MAG_F32 || d == MAG_F16 || d == MAG_BF16; }
inline bool known_act(int a) { return a >= MAG_ACT_NONE && a <= MAG_ACT_SILU; }
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

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
inline int check_shape(const mag_matrix& m, bool out)
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

inline int check_data(const mag_matrix& m, int dtype)
{
    if (m.rows == 0 || m.cols == 0) return MAG_OK;
    if (!m.data) return set_error(MAG_E_NULL, "a matrix's data is NULL");
    if (!aligned(m.data, element(dtype)))
        return set_error(MAG_E_ALIGN, "a matrix is not aligned to its elements");
    return MAG_OK;
}

inline int check_vector(const void* p, int dtype)
{
    if (p && !aligned(p, element(dtype)))
        return set_error(MAG_E_ALIGN, "a vector is not aligned to its elements");
    return MAG_OK;
}

inline int check_workspace(const void* ws, size_t have, size_t need)
{
    if (need == 0) return MAG_OK;
    if (!ws) return set_error(MAG_E_NULL, "workspace is NULL");
    if (!aligned(ws, 256)) return set_error(MAG_E_WORKSPACE, "workspace must be 256-byte aligned");
    if (have < need) return set_error(MAG_E_WORKSPACE, "workspace too small");
    return MAG_OK;
}

inline bool same_shape(const mag_matrix& m, int64_t rows, int64_t cols)
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

inline int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }

}  // namespace
