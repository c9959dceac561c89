// proj_waits.cu -- the projections' bounded waits by themselves (test
// infrastructure only): one CTA whose warps wait for barriers that complete and
// for one that nothing arrives at.
#include "proj_ptx.cuh"

using namespace dpdr::proj;

namespace {

// answers[thread]; in ns how long warp 0 waited, warp 2 waited and the CTA
// settled
__global__ void __launch_bounds__(96) waits_kernel(uint64_t limit, uint32_t* err, int* answers, uint64_t* took)
{
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ uint32_t stop;
    const uint32_t never = smem_addr(&bars[0]), done = smem_addr(&bars[1]);
    if (threadIdx.x == 0) {
        stop = 0;
        bar_init(never, 1);
        bar_init(done, 1);
        bar_init_fence();
        bar_expect(done, 0);
    }
    __syncthreads();
    const Waits w{&stop, err};
    const int warp = warp_number();
    const uint64_t t0 = now_ns();
    bool ok;
    if (warp == 0) ok = bar_wait_warp(never, 0, w, limit);
    else if (warp == 1) ok = bar_wait_warp(done, 0, w, limit);
    else ok = bar_wait_warp(never, 0, w, 100 * limit);   // ended by warp 0's
    const uint64_t t = now_ns() - t0;
    answers[threadIdx.x] = ok;
    if (threadIdx.x == 0) took[0] = t;
    if (threadIdx.x == 64) took[1] = t;
    __syncthreads();
    if (stop) settle(2 * limit);
    if (threadIdx.x == 0) took[2] = now_ns() - t0 - t;
}

}  // namespace

// err, answers (96) and took (3) are in device memory; a CUDA error code
extern "C" int run_waits(uint64_t limit, uint32_t* err, int* answers, uint64_t* took)
{
    waits_kernel<<<1, 96>>>(limit, err, answers, took);
    const cudaError_t e = cudaGetLastError();
    return int(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
