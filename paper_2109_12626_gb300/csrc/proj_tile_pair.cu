// proj_tile_pair.cu -- the gated operator's kernels of proj_tile.cuh.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_pair(int finish, int act)
{
    TileKernel k = nullptr;
#define DPDR_CALL(A) k = finish == kSlope ? tile_kernel<true, kSlope, A> : tile_kernel<true, kValue, A>
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return k;
}

}  // namespace proj
}  // namespace dpdr
