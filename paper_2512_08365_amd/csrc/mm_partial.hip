// mm_partial.hip -- products split along the reduction, into sums of their own.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_partial(const Mm& p, int type, int tile, hipStream_t stream)
{
    if (type == MAG_F16) {
        switch (tile) {
        case TILE_256: return launch_mm_tile<f16, f16, MM_PARTIAL, 256>(p, stream);
        case TILE_128: return launch_mm_tile<f16, f16, MM_PARTIAL, 128>(p, stream);
        default: return launch_mm_tile<f16, f16, MM_PARTIAL, 64>(p, stream);
        }
    }
    switch (tile) {
    case TILE_256: return launch_mm_tile<bf16, bf16, MM_PARTIAL, 256>(p, stream);
    case TILE_128: return launch_mm_tile<bf16, bf16, MM_PARTIAL, 128>(p, stream);
    default: return launch_mm_tile<bf16, bf16, MM_PARTIAL, 64>(p, stream);
    }
}

}  // namespace mag
