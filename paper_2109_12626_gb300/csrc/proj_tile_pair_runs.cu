// proj_tile_pair_runs.cu -- the gated operator's kernels of proj_tile.cuh
// of several runs a sum.
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_pair_runs(int finish, int act) { return tile_kernel_of<true, true>(finish, act); }

}  // namespace proj
}  // namespace dpdr
