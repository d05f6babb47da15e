// fp8.hpp -- shared definitions of the 8-bit operands' quantization and product.
#pragma once

#include "block.hpp"

namespace mag {

constexpr int FP8_BLOCK = MAG_FP8_BLOCK;

// scales: element (row, block) at row * rs + block * cs
struct Scales {
    float* p;
    int64_t rs, cs;
};

struct QuantizeParams {
    const void* x;
    int64_t rs, cs;
    int64_t rows, cols;
    uint8_t* q;         // [rows][q_ld], or NULL
    int64_t q_ld;
    Scales scale;
    uint8_t* qt;        // [cols][qt_ld], or NULL
    int64_t qt_ld;
    Scales scale_t;
};
// square: blocks of 128 x 128; else of 128 neighbours of a row (of qt: of a column)
hipError_t launch_quantize(const QuantizeParams& p, int dtype, int format, bool square, hipStream_t stream);

// out[r][s] = sum over blocks of sa[r] sb[s] sum over the block's k of a(r, k) b(s, k);
// rows along k, at multiples of 16 bytes and (tiles) at most 2^23 apart
struct Mm8 {
    const uint8_t *a, *b;
    int64_t lda, ldb;
    int64_t R, S, K;
    Scales sa, sb;
    int32_t by_row;       // sb has a scale for each s, else for each 128 of them
    int32_t fa, fb;       // MAG_E4M3 / MAG_E5M2
    int32_t splits;       // of the blocks, each with its own sums in `partial`
    float* partial;       // [splits][R][partial_ld]
    int64_t partial_ld;
    Epilogue e;
};
// tile: TILE_*; dtype: of y, MAG_F32 for partial sums
hipError_t launch_mm8_64(const Mm8& p, int dtype, hipStream_t stream);
hipError_t launch_mm8_128(const Mm8& p, int dtype, hipStream_t stream);
hipError_t launch_mm8_256(const Mm8& p, int dtype, hipStream_t stream);
// at most SKINNY_ROWS rows, operands at any alignment and distance, K 0 or at least 16
hipError_t launch_skinny8(const Mm8& p, int dtype, hipStream_t stream);

// rows x cols bytes of any strides as rows of ld bytes
struct Pack8Params {
    const uint8_t* src;
    int64_t rs, cs;
    int64_t rows, cols;
    uint8_t* dst;
    int64_t ld;
};
hipError_t launch_pack8(const Pack8Params& p, hipStream_t stream);

}  // namespace mag
