// proj_rows.cuh -- the projections' products for few rows: the weights are
// read once, by as many CTAs as keep the memory busy.
//
// With M rows of a few (tokens being answered) the weights' bytes bound the
// product.  The tensor core's 128 rows are then 128 features (64 of each
// weight of a pair) and its N columns the M rows of x, so that one pass over a
// weight serves all of them; the sum over k is split over the S CTAs of a
// cluster, which each load their part through a ring of TMA stages (all of it
// in flight at once where it fits), leave their partial tile in shared memory
// and then add up the S partials of their share of the columns in the order
// of the CTAs: one launch, no atomics, the same bits every time.  A part longer
// than a run (proj.h) is summed in several, each in columns of tensor memory of
// its own, which are added up rounded at the end; or, where there are more runs
// than columns for them, in one or two sets of columns in turn, which four
// otherwise idle warps add to a total, in tensor memory too, while the next
// run's products are at work.
//
// Bound by the weights' bytes while there are some megabytes an SM, else by the
// chain of setting up, one trip to memory, the cluster's barriers and partials
// (3.7 us at 1024 x 1024): two rows of 8192 x 8192 in 24.4 us (5.5 TB/s, 0.82 of
// the measured copy), 48 rows of a pair of 2048 x 5120 in 12.4 (3.4 TB/s), 128
// rows of a pair of 8192 x 4096 in 28.4 (4.8 TB/s).  Loads asked into L2 before
// the kernel before has ended, or a smaller ring for more CTAs an SM, gained
// nothing.
#pragma once

#include "proj_common.cuh"
#include "proj_launch.cuh"
#include "proj_ptx.cuh"

namespace dpdr {
namespace proj {

constexpr int kRowStep = kSumStep;         // summed elements a stage
constexpr int kRowFeatures = 128;
constexpr int kRowMaxStages = 12;
constexpr int kRowThreads = 256;
constexpr int kRowSplits = 8;              // CTAs of a cluster, at most

struct RowArgs {
    CUtensorMap w[2], x[2];
    int w_mn, x_mn;
    int steps, segments;      // stages a segment, of all CTAs of a cluster
    int split;                // CTAs of a cluster
    int columns;              // rows of x a tile: a multiple of 16 up to 128
    int x_bytes;              // bytes of x a stage
    int stages;
    int runs;                 // of a CTA's part of the sum, each with its own columns,
    int turns;                // or, if not 0, in this many sets of columns in turn
    int apart;                // columns of tensor memory from one set to the next
    int held;                 // and in all, a power of two
    int width;                // features a tile: 128, of a pair 64
    int vec;                  // results and what else is read allow 4 elements at a time
    int64_t M, N;             // rows of x, features
    Epilogue e;
    uint32_t* err;
};

namespace {

// Four sums side by side from the partials of the cluster's CTAs, in their order
template <int SPLIT>
__device__ __forceinline__ void join(uint32_t at, int split, float (&z)[4])
{
    float p[SPLIT][4];
#pragma unroll
    for (int s = 0; s < SPLIT; s++) {
        p[s][0] = p[s][1] = p[s][2] = p[s][3] = 0.0f;
        if (s < split) cluster_load4(split > 1 ? in_cta(at, s) : at, p[s]);
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        z[i] = p[0][i];
#pragma unroll
        for (int s = 1; s < SPLIT; s++) z[i] += p[s][i];
    }
}

struct Barriers {
    uint32_t full, empty;   // by stage
    uint32_t ready;         // all products done
    uint32_t done, taken;   // of runs in turn, by set of columns
    __device__ __forceinline__ explicit Barriers(uint32_t at)
        : full(at), empty(full + 8 * kRowMaxStages), ready(empty + 8 * kRowMaxStages), done(ready + 8), taken(done + 16)
    {
    }
};

// The products of this CTA's part of the sum, by one warp
template <bool TURNS>
__device__ __forceinline__ void products(const RowArgs& t, uint32_t base, const Barriers& bar, uint32_t tmem, int k_first,
                                         int k_last, int stage_bytes, const Waits& waits)
{
    constexpr int kWBytes = kRowFeatures * kRowStep * 2;
    const uint32_t desc = mma_desc(kRowFeatures, t.columns, t.e.half, t.w_mn, t.x_mn);
    const uint64_t w_desc = tile_desc(base, t.w_mn ? kWBytes / 2 : 0),
                   x_desc = tile_desc(base + kWBytes, t.x_mn ? 64 * kRowStep * 2 : 0);
    const uint32_t w_step = (t.w_mn ? 2048 : 32) >> 4, x_step = (t.x_mn ? 2048 : 32) >> 4;   // 16 summed elements
    RunEnds ends(TURNS ? k_last - k_first : 0, TURNS ? t.runs : 1, k_first);
    int stage = 0, run = -1, next = k_first;   // `next`: the step that begins another run
    uint32_t phase = 0, turn = 0, use = 0;     // TURNS: the set of columns, behind the total
    for (int k = k_first; k < k_last; k++) {
        const bool begins = k == next;
        if (TURNS && begins) {
            next = ends.next();
            if (k > k_first && ++turn == uint32_t(t.turns)) turn = 0, use ^= 1;
            if (!bar_wait_warp(bar.taken + 8 * turn, use ^ 1, waits)) break;
        }
        if (!bar_wait_warp(bar.full + 8 * stage, phase, waits)) break;
        tc_fence_after();
        if (!TURNS && begins) next = k_first + (k_last - k_first) * (++run + 1) / t.runs;
        const uint32_t on = uint32_t(stage * (stage_bytes >> 4)), sums = tmem + (TURNS ? 1 + turn : run) * t.apart;
        const uint64_t w = w_desc + on, x = x_desc + on;
        if (elected()) {
#pragma unroll
            for (int j = 0; j < kRowStep / 16; j++)
                mma_f16<1>(sums, w + j * w_step, x + j * x_step, desc, !begins || j > 0);
            mma_commit(bar.empty + 8 * stage);
            if (TURNS && k + 1 == next) mma_commit(bar.done + 8 * turn);
        }
        if (++stage == t.stages) stage = 0, phase ^= 1;
    }
    if (elected()) mma_commit(bar.ready);
}

// Of runs in turn, not inline, like add_runs: most calls have no use for them, and
// in one loop with the others they cost those 0.1 to 0.2 us (two rows of 2048 x
// 2048 4.26 instead of 4.14).
__device__ __noinline__ void products_in_turns(const RowArgs& t, uint32_t base, const Barriers bar, uint32_t tmem,
                                               int k_first, int k_last, int stage_bytes, const Waits waits)
{
    products<true>(t, base, bar, tmem, k_first, k_last, stage_bytes, waits);
}

// Warps 4 to 7, the runs in turn: each added to the total, in tensor memory, 16
// columns of a thread's row at a time.
__device__ __noinline__ void add_runs(uint32_t tmem, uint32_t done, uint32_t taken, int runs, int turns, int columns,
                                      int apart, const Waits waits)
{
    const int warp = warp_number();
    const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);
    uint32_t turn = 0, use = 0;
    for (int run = 0; run < runs; run++) {
        if (!bar_wait_warp(done + 8 * turn, use, waits)) break;
        tc_fence_after();
        for (int c = 0; c < columns; c += 16) {
            float v[16], w[16] = {};
            tmem_load16(v, lanes + (1 + turn) * apart + c);
            if (run > 0) tmem_load16(w, lanes + c);
            tmem_load_wait(v, w);
#pragma unroll
            for (int i = 0; i < 16; i++) v[i] += w[i];
            tmem_store16(v, lanes + c);
        }
        tmem_store_wait();
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) bar_arrive(taken + 8 * turn);
        if (++turn == uint32_t(turns)) turn = 0, use ^= 1;
    }
}

template <bool PAIR, int FINISH, int ACT, int SPLIT>
__global__ void __launch_bounds__(kRowThreads) row_kernel(const __grid_constant__ RowArgs t)
{
    extern __shared__ char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kRowMaxStages + 5];
    __shared__ uint32_t tmem_at, stop;
    char* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const int rank = t.split > 1 ? int(cluster_rank()) : 0;
    const Barriers bar(smem_addr(bars));
    const Waits waits{&stop, t.err};
    const int64_t n0 = int64_t(blockIdx.x / t.split) * t.width, m0 = int64_t(blockIdx.y) * t.columns;
    const int cols = int(min(int64_t(t.columns), t.M - m0));
    constexpr int kWBytes = kRowFeatures * kRowStep * 2;
    const int stage_bytes = kWBytes + t.x_bytes;
    // this CTA's share of the steps
    const int steps = t.steps * t.segments;
    const int k_first = int(int64_t(steps) * rank / t.split), k_last = int(int64_t(steps) * (rank + 1) / t.split);

    if (threadIdx.x == 0) {
        stop = 0;
        for (int i = 0; i < t.stages; i++) {
            bar_init(bar.full + 8 * i, 1);
            bar_init(bar.empty + 8 * i, 1);
        }
        bar_init(bar.ready, 1);
        for (int i = 0; i < t.turns; i++) {
            bar_init(bar.done + 8 * i, 1);
            bar_init(bar.taken + 8 * i, 4);
        }
        bar_init_fence();
    }
    if (warp == 2) tmem_alloc<1>(smem_addr(&tmem_at), t.held);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    wait_previous();
    allow_next();

    if (warp == 0) {
        int stage = 0;
        uint32_t phase = 0;
        for (int k = k_first; k < k_last; k++) {
            if (!bar_wait_warp(bar.empty + 8 * stage, phase ^ 1, waits)) break;
            const int seg = k >= t.steps, k0 = (seg ? k - t.steps : k) * kRowStep;
            const uint32_t dst = smem_addr(base) + stage * stage_bytes, full = bar.full + 8 * stage;
            if (elected()) {
                bar_expect(full, stage_bytes);
                if (PAIR) {   // 64 features of either weight
                    const int a = int(n0);
                    if (t.w_mn) {
                        tma_load(dst, &t.w[0], a, k0, full);
                        tma_load(dst + kWBytes / 2, &t.w[1], a, k0, full);
                    } else {
                        tma_load(dst, &t.w[0], k0, a, full);
                        tma_load(dst + kWBytes / 2, &t.w[1], k0, a, full);
                    }
                } else if (t.w_mn) {
                    tma_load(dst, &t.w[seg], int(n0), k0, full);
                    tma_load(dst + kWBytes / 2, &t.w[seg], int(n0) + 64, k0, full);
                } else {
                    tma_load(dst, &t.w[seg], k0, int(n0), full);
                }
                if (t.x_mn) {
                    for (int c = 0; c < t.columns; c += 64)
                        tma_load(dst + kWBytes + c * kRowStep * 2, &t.x[seg], int(m0) + c, k0, full);
                } else {
                    tma_load(dst + kWBytes, &t.x[seg], k0, int(m0), full);
                }
            }
            if (++stage == t.stages) stage = 0, phase ^= 1;
        }
    } else if (warp == 1) {
        if (t.turns) products_in_turns(t, smem_addr(base), bar, tmem, k_first, k_last, stage_bytes, waits);
        else products<false>(t, smem_addr(base), bar, tmem, k_first, k_last, stage_bytes, waits);
    } else if (warp >= 4 && t.turns) {
        add_runs(tmem, bar.done, bar.taken, t.runs, t.turns, t.columns, t.apart, waits);
    }
    __syncwarp();
    // All products done (and with them every load): the stages' memory now
    // takes the partial tile, column by column.  Of runs in turn the warps that
    // add them know it, and the others wait for those at the barrier: a wait of
    // theirs would stand for a sum of any length.
    float* part = reinterpret_cast<float*>(base);
    bool ok = true;
    if (!t.turns || warp >= 4) ok = bar_wait_warp(bar.ready, 0, waits);
    tc_fence_before();
    ok = __syncthreads_and(ok && !stop);   // every role is done with the stages
    if (!ok) settle();
    tc_fence_after();
    if (ok) {
        const int quarter = warp & 3;
        for (int c0 = (warp >> 2) * 32; c0 < cols; c0 += 64) {
            float v[32], w[32];
            tmem_load32(v, tmem + c0 + (uint32_t(quarter) << 21));
            tmem_load_wait(v);
            for (int r = 1; r < t.runs && !t.turns; r++) {
                tmem_load32(w, tmem + r * t.apart + c0 + (uint32_t(quarter) << 21));
                tmem_load_wait(w);
#pragma unroll
                for (int i = 0; i < 32; i++) v[i] += w[i];
            }
#pragma unroll
            for (int i = 0; i < 32; i++)
                if (c0 + i < cols) part[(c0 + i) * kRowFeatures + quarter * 32 + lane] = v[i];
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (t.split > 1) cluster_arrive();
    if (warp == 2) tmem_free<1>(tmem, t.held);
    if (t.split > 1) cluster_wait();
    constexpr bool kSums = !PAIR && FINISH == kSlope;
    float down[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // dz's sums over this thread's rows of it
    if (ok) {
        // ------------------------------------------------ results
        // A thread takes four features of a column; the partials of all CTAs
        // are asked for before the first is added (one after the other, each a
        // trip to another SM, took 8 of the 12 us of 333 rows, 2500 to 1000).
        const Epilogue& e = t.e;
        constexpr int kAcross = (PAIR ? 64 : 128) / 4, kApart = kRowThreads / kAcross;
        constexpr int kBatch = SPLIT > 2 ? 1 : 2;   // columns whose partials are asked for together
        const int f = 4 * (int(threadIdx.x) % kAcross);
        const int64_t n = n0 + f;
        const bool four = t.vec && n + 3 < t.N;
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (e.bias) {
            if (four)
                load4(static_cast<const char*>(e.bias), n, 0, e.half, bias);
            else
                for (int i = 0; i < 4; i++)
                    if (n + i < t.N) bias[i] = load1(static_cast<const char*>(e.bias), n + i, 0, e.half);
        }
        if (n < t.N)
            for (int c = rank + t.split * int(threadIdx.x / kAcross); c < cols; c += kBatch * kApart * t.split) {
                float z[kBatch][4], u[kBatch][4], o[kBatch][4];
#pragma unroll
                for (int b = 0; b < kBatch; b++) {
                    // a batch's column past the last reads that one's partials
                    // again, and is dropped
                    const int at = c + b * kApart * t.split;
                    const uint32_t from = smem_addr(part + min(at, cols - 1) * kRowFeatures + f);
#pragma unroll
                    for (int i = 0; i < 4; i++) u[b][i] = o[b][i] = 0.0f;
                    if (four && e.other && at < cols)
                        load4(e.other, (m0 + at) * e.other_rs + n, e.other_f32, e.half, o[b]);
                    if (!four && at < cols)
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (n + i < t.N) o[b][i] = other1(e, m0 + at, n + i);
                    join<SPLIT>(from, t.split, z[b]);
                    if (PAIR) join<SPLIT>(from + 64 * 4, t.split, u[b]);
                }
#pragma unroll
                for (int b = 0; b < kBatch; b++) {
                    const int64_t m = m0 + c + b * kApart * t.split;
                    if (m >= m0 + cols) break;
                    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (four)
                        put4<PAIR, FINISH, ACT>(e, e.out, e.out_rs, m, n, z[b], u[b], bias, o[b], v);
                    else
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            if (n + i < t.N)
                                v[i] = put1<PAIR, FINISH, ACT>(e, e.out, e.out_rs, m, n + i, z[b][i], u[b][i], bias[i],
                                                               o[b][i]);
                    if (kSums)
#pragma unroll
                        for (int i = 0; i < 4; i++) down[i] += v[i];
                }
            }
    }
    __syncwarp();
    if (t.split > 1) cluster_sync();   // the others have read this CTA's partials
    if (kSums && t.e.sums && ok) {
        // over the warps, which had every eighth of this CTA's rows of dz, in their
        // order, where the partials were
        __syncthreads();
        *reinterpret_cast<float4*>(part + 4 * threadIdx.x) = make_float4(down[0], down[1], down[2], down[3]);
        __syncthreads();
        const int64_t at = n0 + threadIdx.x;
        if (threadIdx.x < kRowFeatures && at < t.N) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kRowThreads / 32; i++) sum += part[i * kRowFeatures + threadIdx.x];
            t.e.sums[(int64_t(blockIdx.y) * t.split + rank) * t.N + at] = sum;
        }
    }
}

}  // namespace

using RowKernel = void (*)(RowArgs);

// kernels for up to 2, 4 and 8 CTAs of a cluster: as many partials as are
// asked for at a time (with that for 8 alone, 256 rows of 4096 x 4096 in 15.6
// instead of 15.1 us, 1024 rows of 1024 x 1024 in 7.9 instead of 7.4)
inline int row_split_class(int split) { return split <= 2 ? 0 : split <= 4 ? 1 : 2; }

template <bool PAIR>
RowKernel row_kernel_of(int finish, int act, int split)
{
    const int c = row_split_class(split);
    RowKernel k = nullptr;
    // without an activation a single dz is dy, and no product is finished as one
#define DPDR_KERNELS(F, A) \
    c == 0 ? row_kernel<PAIR, F, A, 2> : c == 1 ? row_kernel<PAIR, F, A, 4> : row_kernel<PAIR, F, A, 8>
#define DPDR_CALL(A)                                                                       \
    if ((PAIR || A != DPDR_ACT_NONE) && finish == kSlope) {                                 \
        k = DPDR_KERNELS((PAIR || A != DPDR_ACT_NONE ? kSlope : kValue), A);                \
    } else {                                                                               \
        k = DPDR_KERNELS(kValue, A);                                                       \
    }
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
#undef DPDR_KERNELS
    return k;
}

}  // namespace proj
}  // namespace dpdr
