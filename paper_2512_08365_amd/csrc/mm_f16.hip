// mm_f16.hip -- products of half operands.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_f16(const Mm& p, int tile, hipStream_t stream)
{
    switch (tile) {
    case TILE_256: return launch_mm_tile<f16, f16, MM_LINEAR, 256>(p, stream);
    case TILE_128: return launch_mm_tile<f16, f16, MM_LINEAR, 128>(p, stream);
    default: return launch_mm_tile<f16, f16, MM_LINEAR, 64>(p, stream);
    }
}

}  // namespace mag
