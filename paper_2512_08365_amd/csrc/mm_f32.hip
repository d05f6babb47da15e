// mm_f32.hip -- products of fp32 operands in three bfloat16 parts each.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_f32(const Mm& p, int tile, hipStream_t stream)
{
    if (tile == TILE_128) return launch_mm_tile<bf16, float, MM_LINEAR, 128, 2, 3>(p, stream);
    return launch_mm_tile<bf16, float, MM_LINEAR, 64, 4, 3>(p, stream);
}

}  // namespace mag
