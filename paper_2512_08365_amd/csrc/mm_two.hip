// mm_two.hip -- a small layer's two gradients in one launch.
#include "mm.hpp"

namespace mag {

hipError_t launch_mm_two(const Mm& dx, const Mm& dw, int kind, int wgs_dx, int wgs_dw, hipStream_t stream)
{
    switch (kind) {
    case MM_BF16: return launch_mm_two_tiles<bf16, bf16, 1>(dx, dw, wgs_dx, wgs_dw, stream);
    case MM_F16: return launch_mm_two_tiles<f16, f16, 1>(dx, dw, wgs_dx, wgs_dw, stream);
    case MM_F32: return launch_mm_two_tiles<float, float, 1>(dx, dw, wgs_dx, wgs_dw, stream);
    default: return launch_mm_two_tiles<bf16, float, 3>(dx, dw, wgs_dx, wgs_dw, stream);
    }
}

}  // namespace mag
