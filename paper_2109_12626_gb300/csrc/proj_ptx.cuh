// proj_ptx.cuh -- the instructions that the projections' tensor-core kernels
// are made of: mbarriers with bounded waits, TMA tile loads, tcgen05.
#pragma once

#include <cuda.h>

#include <cstdint>

namespace dpdr {
namespace proj {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// the same shared-memory place in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync()
{
    cluster_arrive();
    cluster_wait();
}

__device__ __forceinline__ void cluster_load4(uint32_t addr, float (&v)[4])
{
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                 : "r"(addr)
                 : "memory");
}

// ------------------------------------------------------------- mbarriers

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void bar_init_fence()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// an arrival at a barrier of this CTA
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// An arrival at a barrier of any CTA of the cluster (address from in_cta).  It
// orders no memory: it tells that tensor memory has been read, which the
// fences of tcgen05 order, and as a release it waited for the results' stores
// to reach L2, 2 us a tile.
__device__ __forceinline__ void bar_arrive_at(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// The device-side state of a bounded wait: `stop` (shared memory) ends every
// wait of the CTA once one has run out, `err` is the plan's error word.
struct Waits {
    volatile uint32_t* stop;
    uint32_t* err;
};
constexpr uint64_t kWaitNs = 4000000000ull;

// Waits for the phase of that parity; false if it did not come in time or
// another wait of the CTA has already given up.  The answer is each lane's own:
// kernels ask with bar_wait_warp.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, const Waits& w, uint64_t limit = kWaitNs)
{
    if (bar_try(bar, parity)) return true;
    const uint64_t t0 = now_ns();
    for (uint32_t i = 1;; i++) {
        if (bar_try(bar, parity)) return true;
        if ((i & 15u) == 0u) {
            if (*w.stop) return false;
            if (now_ns() - t0 > limit) break;
        }
    }
    *w.stop = 1u;
    *reinterpret_cast<volatile uint32_t*>(w.err) = 1u;
    __threadfence_system();
    return false;
}

// The same for a whole warp, with one answer for it: what follows a wait, loads
// from tensor memory and barriers of the CTA, is for all lanes of a warp or for
// none.  The warps that issue loads and products stay together, and one lane of them issues: what those
// instructions take then stays in the registers that a warp shares.  A lone
// thread moved each operand there anew, which took 126 cycles a product.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, const Waits& w, uint64_t limit = kWaitNs)
{
    return __all_sync(0xFFFFFFFFu, bar_wait(bar, parity, w, limit));
}

// true in one lane of a warp that is together
__device__ __forceinline__ bool elected()
{
    uint32_t is;
    asm volatile(
        "{\n.reg .pred p;\n"
        "elect.sync _|p, 0xFFFFFFFF;\n"
        "selp.u32 %0, 1, 0, p;\n}"
        : "=r"(is));
    return is != 0;
}

// this thread's warp, as a value that the whole warp shares
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0); }

// For a CTA that leaves after a failed wait, once all its warps have ended: its
// loads that no wait stands for any more still write to its shared memory, and
// products still read it.  Both take microseconds, whichever barriers they
// count on; a second is ample.
__device__ __forceinline__ void settle(uint64_t ns = kWaitNs / 4)
{
    const uint64_t t0 = now_ns();
    while (now_ns() - t0 < ns) {
    }
}

// ------------------------------------------------------------------- TMA

// Tile of a two-dimensional tensor map into this CTA's shared memory; the
// bytes count on a barrier of either CTA of the pair (address from in_cta).
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}

// --------------------------------------------------------------- tcgen05

template <int G>
__device__ __forceinline__ void tmem_alloc(uint32_t dst, uint32_t cols)
{
    if (G == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}

template <int G>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t cols)
{
    if (G == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols));
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory matrix descriptor of a tile in TMA's 128-byte swizzle, whose
// patterns of 8 rows x 128 bytes start on 1024-byte boundaries.
//   summed index contiguous: a pattern holds 8 rows of 64 summed elements;
//     the next 8 rows follow 1024 bytes on (stride offset)
//   other index contiguous: a pattern holds 64 elements at 8 summed indices;
//     the next 8 summed indices follow 1024 bytes on (stride offset), the next
//     64 elements `lead` bytes on (leading offset)
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lead)
{
    return uint64_t((addr >> 4) & 0x3FFFu) | uint64_t((lead >> 4) & 0x3FFFu) << 16 | uint64_t(1024 >> 4) << 32 |
           uint64_t(1) << 46 | uint64_t(2) << 61;
}

// Instruction descriptor of kind::f16: float32 sums, operands both bfloat16
// or both float16, each with the summed index contiguous or not.
constexpr uint32_t mma_desc(int m, int n, int half, int a_mn, int b_mn)
{
    return 1u << 4 | uint32_t(half ? 0 : 1) << 7 | uint32_t(half ? 0 : 1) << 10 | uint32_t(a_mn) << 15 |
           uint32_t(b_mn) << 16 | uint32_t(n >> 3) << 17 | uint32_t(m >> 4) << 24;
}

template <int G>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add)
{
    if (G == 2)
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"(uint32_t(add))
            : "memory");
    else
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"(uint32_t(add))
            : "memory");
}

// arrives at the barrier once the products issued so far are done; the pair's
// form at the same place of both CTAs
__device__ __forceinline__ void mma_commit_pair(uint32_t bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"(uint16_t(3))
        : "memory");
}

__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// 16 columns of this warp's 32 lanes: v[i] is (lane, column + i)
__device__ __forceinline__ void tmem_load16(float* v, uint32_t at)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at));
}

// and 32 columns
__device__ __forceinline__ void tmem_load32(float (&v)[32], uint32_t at)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}

// The loads so far are complete; v passes through, so that nothing is done
// with it before.
__device__ __forceinline__ void tmem_load_wait(float (&v)[32])
{
    asm volatile(
        "tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
          "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
          "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
          "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
        :
        : "memory");
}

__device__ __forceinline__ void tmem_load_wait(float (&v)[16])
{
    asm volatile(
        "tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
          "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
        :
        : "memory");
}

__device__ __forceinline__ void tmem_load_wait(float (&v)[16], float (&w)[16])
{
    asm volatile(
        "tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
          "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(w[0]),
          "+f"(w[1]), "+f"(w[2]), "+f"(w[3]), "+f"(w[4]), "+f"(w[5]), "+f"(w[6]), "+f"(w[7]), "+f"(w[8]), "+f"(w[9]),
          "+f"(w[10]), "+f"(w[11]), "+f"(w[12]), "+f"(w[13]), "+f"(w[14]), "+f"(w[15])
        :
        : "memory");
}

// v[i] to (lane, column + i), and all such stores done
__device__ __forceinline__ void tmem_store16(const float (&v)[16], uint32_t at)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"f"(v[0]),
        "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
        "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

}  // namespace proj
}  // namespace dpdr
