// 256x128 tiles of the product of 8-bit operands (see nvfp4_e4m3_gemm.h).
#include "nvfp4_e4m3_gemm.h"

namespace nvfp4 {

hipError_t launch_e4m3_256x128(int kind, const E4m3GemmArgs &g, hipStream_t s)
{
    return g.fast ? launch_e4m3_kind<256, 128, true>(kind, g, s) : hipErrorInvalidValue;           // (exact sums: two rounds of 128 x 128 take less)
}

}  // namespace nvfp4
