// proj_tile_scaled.cu -- the kernel of proj_tile.cuh of whole numbers, their sums
// scaled by row and column.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_scaled() { return tile_kernel<false, kScaled, DPDR_ACT_NONE, true>; }

}  // namespace proj
}  // namespace dpdr
