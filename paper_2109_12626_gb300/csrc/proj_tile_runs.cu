// proj_tile_runs.cu -- kernels of proj_tile.cuh of one product a tile and
// several runs a sum.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_single_runs(int finish, int act) { return tile_kernel_of<false, true>(finish, act); }

}  // namespace proj
}  // namespace dpdr
