// mm_orth.hip -- products of an update's iteration, operands in two half parts each.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_orth(const Mm& p, int tile, hipStream_t stream)
{
    if (tile == TILE_256) return launch_mm_tile<f16, f16, MM_ORTH, 256, 2, 2>(p, stream);
    if (tile == TILE_128) return launch_mm_128<f16, f16, MM_ORTH, 2>(p, stream);
    return launch_mm_tile<f16, f16, MM_ORTH, 64, 4, 2>(p, stream);
}

}  // namespace mag
