// mm_partial.hip -- products split along the reduction, into sums of their own.
#include "mm.hpp"

namespace mag {

template <class T, int P>
static hipError_t launch(const Mm& p, int tile, hipStream_t stream)
{
    if (tile == TILE_128) return launch_mm_tile<T, T, MM_PARTIAL, 128, 2, P>(p, stream);
    return launch_mm_tile<T, T, MM_PARTIAL, 64, 4, P>(p, stream);
}

hipError_t launch_mm_partial(const Mm& p, int kind, int tile, hipStream_t stream)
{
    switch (kind) {
    case MM_BF16: return launch<bf16, 1>(p, tile, stream);
    case MM_F16: return launch<f16, 1>(p, tile, stream);
    case MM_F32: return launch_mm_tile<float, float, MM_PARTIAL, 64, 4, 1>(p, stream);
    case MM_F32_PARTS: return launch<bf16, 3>(p, tile, stream);
    default: return launch<f16, 2>(p, tile, stream);
    }
}

}  // namespace mag
