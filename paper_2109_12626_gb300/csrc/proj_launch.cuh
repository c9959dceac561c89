// proj_launch.cuh -- how the projections' kernels are launched: each is set up
// while the kernel before it in the stream drains, and waits there before it
// touches memory.
#pragma once

#include "proj.h"

namespace dpdr {
namespace proj {

// Before a kernel's first access to global memory, in every thread that makes
// one: the kernel before is complete and its writes are visible.  A kernel
// that has passed here has no predecessor running, so the order of calls in a
// stream is what it would be without.
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Lets the next kernel in the stream be set up from here on: asked for by the
// kernels of a few microseconds, whose CTAs leave room beside them (one row of
// 4096 x 4096 weights, back to back: 10.4 and 9.6 us; 24 rows of 8192 x 1024
// 8.5 and 7.8).  A kernel of one CTA an SM gains nothing by it.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;"); }

template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t s,
           const char* what, const Args&... args)
{
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = unsigned(cluster);
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c = {};
    c.gridDim = grid;
    c.blockDim = block;
    c.dynamicSmemBytes = smem;
    c.stream = s;
    c.attrs = at;
    c.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&c, kernel, args...);
    return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, what);
}

}  // namespace proj
}  // namespace dpdr
