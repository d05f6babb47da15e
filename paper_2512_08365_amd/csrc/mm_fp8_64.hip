// mm_fp8_64.hip -- the 8-bit product's tiles of 64.
#include "mm_fp8.hpp"

namespace mag {

hipError_t launch_mm8_64(const Mm8& p, int dtype, hipStream_t stream)
{
    return launch_mm8<Shape8<64, 2, 2>>(p, dtype, stream);
}

}  // namespace mag
