// proj_tile.cuh -- the projections' products on the tensor cores: pairs of CTAs
// on 256 x 256 tiles of the result.
//
// D[m][n] = sum_k A[m][k] B[n][k].  A persistent pair of CTAs (a cluster of
// two) takes one tile after another.  CTA r loads rows 128 r of A's 256 and of
// B's 256 (64 summed elements at a time, by TMA, into a ring of stages), one
// thread of CTA 0 issues the pair's products (256 x 256 x 16 each, cta_group::2),
// and CTA r holds the sums of its 128 rows in half of its tensor memory, so
// that the other half takes the next tile's sums while four warps finish this
// one's.  Each operand may have the summed index contiguous or the other one;
// the tile in shared memory is then laid out the other way and the
// instruction told so, so that the gradients' products read the same arrays
// as the forward product, nothing transposed.  For the gated operator B is the
// two weights' 128 rows of the same features, one weight a CTA: the pair g, u
// of an output ends in columns n and n + 128 of one thread's row.
#pragma once

#include "proj_common.cuh"
#include "proj_launch.cuh"
#include "proj_ptx.cuh"

namespace dpdr {
namespace proj {

namespace {

constexpr int kStages = 6;
constexpr int kStep = 64;                     // summed elements a stage
constexpr int kHalf = 128 * kStep * 2;        // bytes of one operand of a stage and CTA
constexpr int kStage = 2 * kHalf;
constexpr int kStaging = 4 * 32 * 64 * 4;     // 32 x 64 floats a finishing warp
constexpr int kSmem = 1024 + kStages * kStage + kStaging;
constexpr int kThreads = 256;                 // warps: load, product, tensor memory, -, 4 finishing

struct TileArgs {
    CUtensorMap a[2], b[2];
    int a_mn, b_mn;                // the other index is the contiguous one
    int kind, steps, segments;     // stages a segment
    int tiles_m, tiles_n, tiles;   // tiles_m of one of kTwin's products
    int width;                     // result columns a tile
    int vec;                       // results and what else is read allow 4 elements at a time
    int64_t M, N;
    Epilogue e;
    uint32_t* err;
};

// Tiles in bands of 8 rows of tiles, down each band's columns, so that the
// tiles in work at a time share their operands in L2.
__device__ __forceinline__ void tile_place(const TileArgs& t, int i, int& tm, int& tn)
{
    const int rows = t.tiles / t.tiles_n;
    const int band = 8 * t.tiles_n, b = i / band, first = 8 * b;
    const int high = min(8, rows - first), in = i - b * band;
    tm = first + in % high;
    tn = in / high;
}

// Finishes a warp's 32 rows of a tile.  The tensor memory hands each thread a
// row, the results want rows across threads: 64 columns at a time (of a pair 32
// and 32) go through shared memory, 16-byte chunk q of row r at q ^ (r & 7), so
// that neither way meets a bank twice.
template <bool PAIR, int FINISH, int ACT>
__device__ __forceinline__ void finish_rows(const TileArgs& t, uint32_t tmem, float* stage, int lane, int64_t m0,
                                            int64_t n0, char* out, int64_t out_rs)
{
    const Epilogue& e = t.e;
    constexpr int kCols = PAIR ? 32 : 64;    // result columns a round
    constexpr int kPer = kCols / 4;          // threads a row
    const int rows = int(min(int64_t(32), t.M - m0));
    const int cols = int(min(int64_t(t.width), t.N - n0));
    for (int c0 = 0; c0 < cols; c0 += kCols) {
        float v[32];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            tmem_load32(v, tmem + (PAIR ? h * 128 + c0 : c0 + h * 32));
            tmem_load_wait();
#pragma unroll
            for (int q = 0; q < 8; q++)
                *reinterpret_cast<float4*>(stage + lane * 64 + 4 * ((h * 8 + q) ^ (lane & 7))) =
                    make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
        __syncwarp();
        if (t.vec) {
            const int q = lane % kPer, c = c0 + 4 * q;
            const int64_t n = n0 + c;
            if (c + 3 < cols) {
                float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (e.bias) load4(static_cast<const char*>(e.bias), n, 0, e.half, bias);
                // eight rows' other values are asked for before the first
                // row's results are stored
                constexpr int kRows = 32 / kPer, kBatch = 8;
                for (int r0 = lane / kPer; r0 < rows; r0 += kRows * kBatch) {
                    float o[kBatch][4];
#pragma unroll
                    for (int b = 0; b < kBatch; b++) {
                        o[b][0] = o[b][1] = o[b][2] = o[b][3] = 0.0f;
                        if (e.other && r0 + b * kRows < rows)
                            load4(e.other, (m0 + r0 + b * kRows) * e.other_rs + n, e.other_f32, e.half, o[b]);
                    }
#pragma unroll
                    for (int b = 0; b < kBatch; b++) {
                        const int r = r0 + b * kRows;
                        if (r >= rows) break;
                        const float4 z4 = *reinterpret_cast<const float4*>(stage + r * 64 + 4 * (q ^ (r & 7)));
                        float z[4] = {z4.x, z4.y, z4.z, z4.w}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        if (PAIR) {
                            const float4 u4 = *reinterpret_cast<const float4*>(stage + r * 64 + 4 * ((8 + q) ^ (r & 7)));
                            u[0] = u4.x, u[1] = u4.y, u[2] = u4.z, u[3] = u4.w;
                        }
                        put4<PAIR, FINISH, ACT>(e, out, out_rs, m0 + r, n, z, u, bias, o[b]);
                    }
                }
            } else {
                for (int r = lane / kPer; r < rows; r += 32 / kPer)
                    for (int i = 0; i < 4 && c + i < cols; i++)
                        put1<PAIR, FINISH, ACT>(e, out, out_rs, m0 + r, n + i, stage[r * 64 + 4 * (q ^ (r & 7)) + i],
                                   PAIR ? stage[r * 64 + 4 * ((8 + q) ^ (r & 7)) + i] : 0.0f,
                                   e.bias ? load1(static_cast<const char*>(e.bias), n + i, 0, e.half) : 0.0f);
            }
        } else {
            for (int h = 0; h < kCols / 32; h++) {
                const int c = h * 32 + lane, q = c >> 2, i = c & 3;
                if (c0 + c >= cols) break;
                const int64_t n = n0 + c0 + c;
                const float bias = e.bias ? load1(static_cast<const char*>(e.bias), n, 0, e.half) : 0.0f;
#pragma unroll 4
                for (int r = 0; r < rows; r++)
                    put1<PAIR, FINISH, ACT>(e, out, out_rs, m0 + r, n, stage[r * 64 + 4 * (q ^ (r & 7)) + i],
                               PAIR ? stage[r * 64 + 4 * ((8 + q) ^ (r & 7)) + i] : 0.0f, bias);
            }
        }
        __syncwarp();
    }
}

template <bool PAIR, int FINISH, int ACT>
__global__ void __launch_bounds__(kThreads, 1) tile_kernel(const __grid_constant__ TileArgs t)
{
    extern __shared__ char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
    __shared__ uint32_t tmem_at, stop;
    char* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages,
                   taken = ready + 16, last = taken + 16;
    const Waits waits{&stop, t.err};
    const int pairs = gridDim.x >> 1, first = blockIdx.x >> 1;

    if (threadIdx.x == 0) {
        stop = 0;
        for (int i = 0; i < kStages; i++) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; i++) {
            bar_init(ready + 8 * i, 1);
            bar_init(taken + 8 * i, 8);   // four warps of each CTA
        }
        bar_init(last, 1);
        bar_init_fence();
    }
    if (warp == 2) tmem_alloc<2>(smem_addr(&tmem_at), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    const int steps = t.steps * t.segments;
    wait_previous();

    if (warp == 0 && lane == 0) {
        // ------------------------------------------------ loads
        int stage = 0, used = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int i = first; i < t.tiles && ok; i += pairs) {
            int tm, tn;
            tile_place(t, i, tm, tn);
            const int twin = tm >= t.tiles_m;
            const int m0 = (tm - twin * t.tiles_m) * 256 + int(rank) * 128;
            const int n0 = PAIR ? tn * 128 : tn * 256 + int(rank) * 128;
            for (int k = 0; k < steps; k++) {
                if (!(ok = bar_wait(empty + 8 * stage, phase ^ 1, waits))) break;
                const int seg = k >= t.steps, k0 = (seg ? k - t.steps : k) * kStep;
                const CUtensorMap* ma = &t.a[twin | seg];
                const CUtensorMap* mb = &t.b[PAIR ? int(rank) : seg];
                const uint32_t dst = smem_addr(base) + stage * kStage, bar = in_cta(full + 8 * stage, 0);
                if (rank == 0) bar_expect(full + 8 * stage, 2 * kStage);
                if (t.a_mn) {
                    tma_load_pair(dst, ma, m0, k0, bar);
                    tma_load_pair(dst + kHalf / 2, ma, m0 + 64, k0, bar);
                } else {
                    tma_load_pair(dst, ma, k0, m0, bar);
                }
                if (t.b_mn) {
                    tma_load_pair(dst + kHalf, mb, n0, k0, bar);
                    tma_load_pair(dst + kHalf + kHalf / 2, mb, n0 + 64, k0, bar);
                } else {
                    tma_load_pair(dst + kHalf, mb, k0, n0, bar);
                }
                used++;
                if (++stage == kStages) stage = 0, phase ^= 1;
            }
        }
        // Both CTAs' loads have landed once the products that take them are
        // issued; after a failed wait they are waited for here.
        if (!ok && rank == 0)
            for (int n = min(used, kStages); n > 0; n--) {
                if (--stage < 0) stage = kStages - 1, phase ^= 1;
                bar_drain(full + 8 * stage, phase);
            }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ------------------------------------------------ products
        const uint32_t desc = mma_desc(256, 256, t.e.half, t.a_mn, t.b_mn);
        const uint32_t a_lead = t.a_mn ? kHalf / 2 : 0, b_lead = t.b_mn ? kHalf / 2 : 0;
        const uint32_t a_step = t.a_mn ? 2048 : 32, b_step = t.b_mn ? 2048 : 32;   // bytes for 16 summed elements
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (int i = first; i < t.tiles && ok; i += pairs) {
            if (!(ok = bar_wait(taken + 8 * acc, acc_phase ^ 1, waits))) break;
            tc_fence_after();
            for (int k = 0; k < steps; k++) {
                if (!(ok = bar_wait(full + 8 * stage, phase, waits))) break;
                tc_fence_after();
                const uint32_t at = smem_addr(base) + stage * kStage;
#pragma unroll
                for (int j = 0; j < kStep / 16; j++)
                    mma_f16<2>(tmem + acc * 256, tile_desc(at + j * a_step, a_lead),
                               tile_desc(at + kHalf + j * b_step, b_lead), desc, (k | j) != 0);
                mma_commit_pair(empty + 8 * stage);
                if (++stage == kStages) stage = 0, phase ^= 1;
            }
            if (!ok) break;
            mma_commit_pair(ready + 8 * acc);
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
        if (!ok) {   // the products under way still read shared memory
            mma_commit_pair(last);
            bar_drain(last, 0);
        }
    } else if (warp >= 4) {
        // ------------------------------------------------ results
        float* stage = reinterpret_cast<float*>(base + kStages * kStage) + (warp - 4) * 32 * 64;
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int i = first; i < t.tiles; i += pairs) {
            int tm, tn;
            tile_place(t, i, tm, tn);
            const int twin = tm >= t.tiles_m;
            const int64_t m0 = int64_t(tm - twin * t.tiles_m) * 256 + int64_t(rank) * 128 + (warp - 4) * 32;
            if (!bar_wait(ready + 8 * acc, acc_phase, waits)) break;
            tc_fence_after();
            finish_rows<PAIR, FINISH, ACT>(t, tmem + acc * 256 + (uint32_t(warp - 4) << 21), stage, lane, m0, int64_t(tn) * t.width,
                              twin ? t.e.out2 : t.e.out, twin ? t.e.out2_rs : t.e.out_rs);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_at(in_cta(taken + 8 * acc, 0));
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    }
    __syncwarp();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    if (warp == 2) tmem_free<2>(tmem, 512);
}

}  // namespace

using TileKernel = void (*)(TileArgs);

}  // namespace proj
}  // namespace dpdr
