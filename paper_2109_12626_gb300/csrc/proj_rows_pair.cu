// proj_rows_pair.cu -- the gated operator's kernels of proj_rows.cuh.
#include "proj_rows.cuh"

namespace dpdr {
namespace proj {

RowKernel row_kernel_pair(int finish, int act, int split)
{
    return row_kernel_of<true>(finish, act, split);
}

}  // namespace proj
}  // namespace dpdr
