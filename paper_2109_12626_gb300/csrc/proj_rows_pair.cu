// proj_rows_pair.cu -- the gated operator's kernels of proj_rows.cuh.
#include "proj_rows.cuh"

namespace dpdr {
namespace proj {

RowKernel row_kernel_pair(int finish, int act)
{
    RowKernel k = nullptr;
#define DPDR_CALL(A) k = finish == kSlope ? row_kernel<true, kSlope, A> : row_kernel<true, kValue, A>
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return k;
}

}  // namespace proj
}  // namespace dpdr
