// 256x256 tiles of the product of 8-bit operands (see nvfp4_e4m3_gemm.h).
#include "nvfp4_e4m3_gemm.h"

namespace nvfp4 {

hipError_t launch_e4m3_256x256(int kind, const E4m3GemmArgs &g, hipStream_t s)
{
    return g.fast ? launch_e4m3_kind<256, 256, true>(kind, g, s) : launch_e4m3_kind<256, 256, false>(kind, g, s);
}

}  // namespace nvfp4
