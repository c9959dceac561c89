// proj_tile_pair.cu -- the gated operator's kernels of proj_tile.cuh.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_pair(int finish, int act) { return tile_kernel_of<true, false>(finish, act); }

}  // namespace proj
}  // namespace dpdr
