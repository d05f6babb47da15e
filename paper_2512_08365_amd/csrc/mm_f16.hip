// mm_f16.hip -- products of half operands.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_f16(const Mm& p, int tile, hipStream_t stream)
{
    if (tile == TILE_256) return launch_mm_tile<f16, f16, MM_LINEAR, 256, 2, 1>(p, stream);
    if (tile == TILE_128) return launch_mm_128<f16, f16, MM_LINEAR, 1>(p, stream);
    return launch_mm_tile<f16, f16, MM_LINEAR, 64, 4, 1>(p, stream);
}

}  // namespace mag
