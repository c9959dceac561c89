// proj_tile_pair.cu -- the gated operator's kernels of proj_tile.cuh.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_pair(int finish, int act, int f32)
{
    TileKernel k = nullptr;
#define DPDR_CALL(A)                                                              \
    k = f32 ? tile_kernel<true, kValue, A, true>                                 \
            : finish == kSlope ? tile_kernel<true, kSlope, A, false> : tile_kernel<true, kValue, A, false>
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return k;
}

}  // namespace proj
}  // namespace dpdr
