// mm_f32.hip -- products of fp32 operands: as they are, and in three bfloat16 parts
// each.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_f32(const Mm& p, hipStream_t stream)
{
    return launch_mm_tile<float, float, MM_LINEAR, 64, 4, 1>(p, stream);
}

hipError_t launch_mm_f32_parts(const Mm& p, int tile, hipStream_t stream)
{
    if (tile == TILE_128) return launch_mm_tile<bf16, float, MM_LINEAR, 128, 2, 3>(p, stream);
    return launch_mm_tile<bf16, float, MM_LINEAR, 64, 4, 3>(p, stream);
}

}  // namespace mag
