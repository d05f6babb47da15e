// mm_fp8_256.hip -- the 8-bit product's tiles of 256.
#include "mm_fp8.hpp"

namespace mag {

hipError_t launch_mm8_256(const Mm8& p, int dtype, hipStream_t stream)
{
    return launch_mm8<Shape8<256, 2, 4>>(p, dtype, stream);
}

}  // namespace mag
