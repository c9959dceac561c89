// proj_tile.cuh -- the projections' products on the tensor cores: pairs of CTAs
// on 256 x 256 tiles of the result.
//
// D[m][n] = sum_k A[m][k] B[n][k].  A persistent pair of CTAs (a cluster of
// two) takes one tile after another.  CTA r loads rows 128 r of A's 256 and of
// B's 256 (64 summed elements at a time, by TMA, into a ring of stages), one
// thread of CTA 0 issues the pair's products (256 x 256 x 16 each, cta_group::2),
// and CTA r holds the sums of its 128 rows in half of its tensor memory, so
// that the other half takes the next tile's sums while eight warps finish this
// one's.  A pair reads 512 rows of operands for 256 x 256 results, half of what
// two CTAs of 128 x 256 would.  Each operand may have the summed index contiguous
// or the other one; the tile in shared memory is then laid out the other way and
// the instruction told so, so that the gradients' products read the same arrays
// as the forward product, nothing transposed.  For the gated operator B is the
// two weights' 128 rows of the same features, one weight a CTA: the pair g, u
// of an output ends in columns n and n + 128 of one thread's row.
//
// Bound by the tensor cores and, in a long loop, by the power limit: the gated
// operator 8192 x 4096 x 8192 in 632 to 652 us (1.69 to 1.74 PFLOP/s), in a burst of
// 24 calls 529; such bursts of 4096 x 4096 x 4096 in 72 us a call (1.91), of 8192 x
// 4096 x 8192 in 269.  Short sums are bound by finishing a tile (3.5 us) and by
// loads: 4096 x 1000 x 4096 in 32 us.  Tried and not kept: asking tiles into L2 ahead
// of their loads (every pair its own: 411 against 299 us; one pair for all: no
// faster), the last round's tiles summed by several pairs that join their sums (no
// faster, and 43 against 33 us for short sums).
//
// Sums longer than a run (proj.h) are taken in runs (RUNS), and the finishing
// warps add up the runs in registers, rounded, while the next run's products are
// at work: float32 results of 4096 x 4096 x 4096 in 79 us instead of 72.  No wait
// then stands for more than a run, so that none runs out over a sum of any length.
#pragma once

#include "proj_common.cuh"
#include "proj_launch.cuh"
#include "proj_ptx.cuh"

namespace dpdr {
namespace proj {

namespace {

constexpr int kStages = 6;
constexpr int kStep = kSumStep;               // summed elements a stage
constexpr int kHalf = 128 * kStep * 2;        // bytes of one operand of a stage and CTA
constexpr int kStage = 2 * kHalf;
constexpr int kFinishers = 8;                 // warps
constexpr int kStaging = kFinishers * 32 * 32 * 4;   // 32 x 32 floats each
constexpr int kSmem = 1024 + kStages * kStage + kStaging;
constexpr int kThreads = 96 + 32 * kFinishers;   // warps: load A, load B, product, finishing

struct TileArgs {
    CUtensorMap a[2], b[2], b_half[2];   // B's rows by 128 and by 64
    int a_mn, b_mn;                // the other index is the contiguous one
    int steps, segments;           // stages a segment
    int runs;                      // of a sum
    int tiles_m, tiles_n, tiles;   // tiles_m of one of kTwin's products
    // the first `whole` tiles are taken as they are, the rest in two halves of
    // their columns: `items` in all
    int whole, items;
    int vec;                       // results and what else is read allow 4 elements at a time
    int64_t M, N;
    Epilogue e;
    uint32_t* err;
};

// What item i is: its rows and columns of the result, which of kTwin's
// products, and how many columns of sums (of a pair, two for each result).
// Tiles lie in bands of 8 rows of tiles, down each band's columns, so that the
// tiles in work at a time share their operands in L2.
struct Item {
    int m, n, sums, twin;
};

template <bool PAIR>
__device__ __forceinline__ Item item_of(const TileArgs& t, int i)
{
    Item it;
    int part = 0;
    it.sums = 256;
    if (i >= t.whole) {
        part = (i - t.whole) & 1;
        i = t.whole + ((i - t.whole) >> 1);
        it.sums = 128;
    }
    const int rows = t.tiles / t.tiles_n;
    const int band = 8 * t.tiles_n, b = i / band, first = 8 * b;
    const int high = min(8, rows - first), in = i - b * band;
    const int tm = first + in % high, tn = in / high;
    it.twin = tm >= t.tiles_m;
    it.m = (tm - it.twin * t.tiles_m) * 256;
    it.n = PAIR ? tn * 128 + part * 64 : tn * 256 + part * 128;
    return it;
}

// Finishing a warp's 32 rows of an item: 32 columns of sums at a time (of a
// pair 16 and 16), every second such round, the other warp of its rows taking
// the rest.  The tensor memory hands each thread a row, the results want rows
// across threads: the round goes through shared memory, 16-byte chunk q of row
// r at q ^ (r & 7), so that neither way meets a bank twice.  What else a result
// needs (residual, dy) is asked into L2 while the item's products still run, and
// all of a round's together when the round comes: one row at a time, each a trip
// to memory, took 45 us a tile; registers filled a round ahead, between a round's
// stores, half as long again as this.
template <bool PAIR, int FINISH, int ACT, bool RUNS>
struct Finisher {
    static constexpr int kCols = PAIR ? 16 : 32;     // result columns a round
    static constexpr int kPer = kCols / 4;           // threads a row
    static constexpr int kRows = 32 / kPer;          // rows a step
    static constexpr int kSteps = 32 / kRows;

    const TileArgs& t;
    float* stage;
    int q, row;              // this thread's columns (4 q) and first row of a round
    int turn;                // which of the two warps of these rows
    // of the item
    int64_t m0, n0;
    int rows, cols;

    __device__ __forceinline__ Finisher(const TileArgs& args, float* st, int lane, int tu) : t(args), stage(st), turn(tu)
    {
        q = lane % kPer;
        // of a pair, eight threads on two rows four apart: no bank twice
        row = PAIR ? ((lane >> 2) & 1) * 4 + (lane >> 3) : lane / kPer;
    }

    // dz's column sums over a warp's rows, before they are rounded
    static constexpr bool kSums = !PAIR && FINISH == kSlope;

    // threads kPer apart have the same four columns
    __device__ __forceinline__ void put_sums(int c0, float (&down)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int d = kPer; d < 32; d *= 2) down[i] += __shfl_xor_sync(0xFFFFFFFFu, down[i], d);
        if (row == 0 && rows > 0)
#pragma unroll
            for (int i = 0; i < 4; i++) t.e.sums[m0 / 32 * t.N + n0 + c0 + 4 * q + i] = down[i];
    }

    // whether a round of fours starts at c0
    __device__ __forceinline__ bool fours(int c0) const { return t.vec && c0 + kCols <= cols; }

    __device__ __forceinline__ void start(int64_t m, int64_t n, int sums, int lane)
    {
        m0 = m, n0 = n;
        rows = int(max(int64_t(0), min(int64_t(32), t.M - m)));
        cols = int(min(int64_t(PAIR ? sums / 2 : sums), t.N - n));
        const Epilogue& e = t.e;
        if (!e.other || e.other_cs != 1 || cols <= 0) return;
        const int size = e.other_f32 ? 4 : 2;
        if (lane < rows) {   // a row a lane, every second line of it
            const char* p = e.other + ((m0 + lane) * e.other_rs + n0) * size;
            for (int at = 128 * turn; at < cols * size; at += 256) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + at));
        }
    }

    // the round's results in 16 bits, four columns a thread and step
    template <int HALF>
    __device__ __forceinline__ void by_four(int c0, char* out, int64_t out_rs)
    {
        const Epilogue& e = t.e;
        const int64_t n = n0 + c0 + 4 * q;
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (e.bias) load4(static_cast<const char*>(e.bias), n, 0, HALF, bias);
        const int64_t m = m0 + row;
        char* p = out + (m * out_rs + n) * 2;
        char* p2 = e.out2 + (m * e.out2_rs + n) * 2;
        float* pre = e.pre + (m * e.pre_rs + n);
        uint4 other[kSteps];
        if (e.other) {
            const int size = e.other_f32 ? 4 : 2;
            const char* at = e.other + (m * e.other_rs + n) * size;
            const int64_t apart = e.other_rs * kRows * size;
#pragma unroll
            for (int b = 0; b < kSteps; b++, at += apart)
                if (row + b * kRows < rows) {
                    if (e.other_f32) {
                        other[b] = *reinterpret_cast<const uint4*>(at);
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(at);
                        other[b].x = x.x, other[b].y = x.y;
                    }
                }
        }
        // all of the round's sums before the first result is stored: behind a store
        // whose place the compiler cannot tell from theirs, each would wait
        float z[kSteps][4], u[kSteps][4];
#pragma unroll
        for (int b = 0; b < kSteps; b++) {
            const int r = row + b * kRows;
            const float4 z4 = *reinterpret_cast<const float4*>(stage + r * 32 + 4 * (q ^ (r & 7)));
            z[b][0] = z4.x, z[b][1] = z4.y, z[b][2] = z4.z, z[b][3] = z4.w;
            if (PAIR) {
                const float4 u4 = *reinterpret_cast<const float4*>(stage + r * 32 + 4 * ((4 + q) ^ (r & 7)));
                u[b][0] = u4.x, u[b][1] = u4.y, u[b][2] = u4.z, u[b][3] = u4.w;
            }
        }
        const int64_t down = out_rs * kRows * 2, down2 = e.out2_rs * kRows * 2, down_pre = e.pre_rs * kRows;
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int b = 0; b < kSteps; b++) {
            const int r = row + b * kRows;
            if (r < rows) {
                float o[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4], w[4];
#pragma unroll
                for (int i = 0; i < 4; i++) z[b][i] += bias[i];
                if (e.pre) {
                    *reinterpret_cast<float4*>(pre) = make_float4(z[b][0], z[b][1], z[b][2], z[b][3]);
                    if (PAIR)
                        *reinterpret_cast<float4*>(pre + e.pre_up) = make_float4(u[b][0], u[b][1], u[b][2], u[b][3]);
                }
                if (e.other) widen4(other[b], e.other_f32, HALF, o);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    w[i] = 0.0f;
                    finish1<PAIR, FINISH, ACT>(z[b][i], PAIR ? u[b][i] : 0.0f, o[i], v[i], w[i]);
                }
                store4(p, 0, 0, HALF, v);
                if (PAIR && FINISH == kSlope) store4(p2, 0, 0, HALF, w);
                if (kSums)
#pragma unroll
                    for (int i = 0; i < 4; i++) sums[i] += v[i];
            }
            p += down, p2 += down2, pre += down_pre;
        }
        if (kSums && e.sums) put_sums(c0, sums);
    }

    // The same for sums in runs, whatever the results' type, in as few registers as
    // it can be: the other rounds' sums hold most of them.
    __device__ __forceinline__ void by_four_runs(int c0, char* out, int64_t out_rs)
    {
        const Epilogue& e = t.e;
        const int64_t n = n0 + c0 + 4 * q;
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (e.bias) load4(static_cast<const char*>(e.bias), n, 0, e.half, bias);
        float across[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // the columns' scales
        if (FINISH == kScaled) {
            load4(reinterpret_cast<const char*>(e.col_scale), n, 1, 0, across);
            if (e.bias32) load4(reinterpret_cast<const char*>(e.bias32), n, 1, 0, bias);
        }
        float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        auto step = [&](int b, const float (&o)[4]) {
            const int r = row + b * kRows;
            if (r >= rows) return;
            float u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[4];
            const float4 z4 = *reinterpret_cast<const float4*>(stage + r * 32 + 4 * (q ^ (r & 7)));
            float z[4] = {z4.x, z4.y, z4.z, z4.w};
            if (PAIR) {
                const float4 u4 = *reinterpret_cast<const float4*>(stage + r * 32 + 4 * ((4 + q) ^ (r & 7)));
                u[0] = u4.x, u[1] = u4.y, u[2] = u4.z, u[3] = u4.w;
            }
            if constexpr (FINISH == kScaled) {
                const float scale = e.row_scale[m0 + r];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = z[i] * (scale * across[i]) + bias[i] + o[i];
                store4(out, (m0 + r) * out_rs + n, e.out_f32, e.half, v);
            } else {
                put4<PAIR, FINISH, ACT>(e, out, out_rs, m0 + r, n, z, u, bias, o, v);
            }
            if (kSums)
#pragma unroll
                for (int i = 0; i < 4; i++) sums[i] += v[i];
        };
        if ((!PAIR || FINISH == kSlope) && e.other) {
            for (int b0 = 0; b0 < kSteps; b0 += 4) {
                float o[4][4];
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    const int r = row + (b0 + b) * kRows;
#pragma unroll
                    for (int i = 0; i < 4; i++) o[b][i] = 0.0f;
                    if (r < rows) load4(e.other, (m0 + r) * e.other_rs + n, e.other_f32, e.half, o[b]);
                }
#pragma unroll
                for (int b = 0; b < 4; b++) step(b0 + b, o[b]);
            }
            if (kSums && e.sums) put_sums(c0, sums);
            return;
        }
        const float none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
        for (int b = 0; b < kSteps; b++) step(b, none);
    }

    // One element a thread and step, for results that do not lie on fours; the sums
    // and other values of eight steps (of a pair 16) before the first is stored.
    __device__ __forceinline__ void by_one(int c0, int lane, char* out, int64_t out_rs, int half)
    {
        const Epilogue& e = t.e;
        constexpr int kDown = 32 / kCols;   // rows a step
        // one for dz of several runs, which only rows of many thousand elements take
        constexpr int kAsk = RUNS && FINISH == kSlope ? 1 : PAIR ? 16 : 8;
        const int f32 = RUNS && e.out_f32, size = f32 ? 4 : 2;
        const int c = lane % kCols, first = lane / kCols;
        if (c0 + c >= cols) return;
        const int64_t n = n0 + c0 + c, m = m0 + first;
        const float bias = e.bias ? load1(static_cast<const char*>(e.bias), n, 0, half) : 0.0f;
        char* at = out + (m * out_rs + n) * size;
        const int64_t down = out_rs * kDown * size;
        float total = 0.0f;   // of a column's dz, which one thread has
        const float across = FINISH == kScaled ? e.col_scale[n] : 0.0f;
        const float bias32 = FINISH == kScaled && e.bias32 ? e.bias32[n] : 0.0f;
        auto step = [&](int r, char* p, float z, float u, float o) {
            if constexpr (FINISH == kScaled) {
                store1(p, 0, z * (e.row_scale[m0 + r] * across) + bias32 + o, f32, half);
                return;
            }
            if (e.pre) {
                float* pre = e.pre + ((m0 + r) * e.pre_rs + n);
                *pre = z;
                if (PAIR) pre[e.pre_up] = u;
            }
            float v = 0.0f, w = 0.0f;
            finish1<PAIR, FINISH, ACT>(z, u, o, v, w);
            store1(p, 0, v, f32, half);
            if (kSums) total += v;
            if (PAIR && FINISH == kSlope) store1(e.out2, (m0 + r) * e.out2_rs + n, w, f32, half);
        };
        auto sum = [&](int r, int side) {
            return stage[r * 32 + 4 * ((4 * side + (c >> 2)) ^ (r & 7)) + (c & 3)];
        };
        if (!e.other) {
#pragma unroll 4
            for (int r = first; r < rows; r += kDown, at += down)
                step(r, at, sum(r, 0) + bias, PAIR ? sum(r, 1) : 0.0f, 0.0f);
            return;
        }
        for (int r0 = first; r0 < rows; r0 += kDown * kAsk, at += kAsk * down) {
            float z[kAsk], u[kAsk], o[kAsk];
#pragma unroll
            for (int b = 0; b < kAsk; b++) {
                const int r = r0 + b * kDown;
                o[b] = r < rows ? other1(e, m0 + r, n) : 0.0f;
                z[b] = sum(r & 31, 0) + bias;
                u[b] = PAIR ? sum(r & 31, 1) : 0.0f;
            }
#pragma unroll
            for (int b = 0; b < kAsk; b++)
                if (r0 + b * kDown < rows) step(r0 + b * kDown, at + b * down, z[b], u[b], o[b]);
        }
        if (kSums && e.sums && rows > 0) e.sums[m0 / 32 * t.N + n] = total;
    }

    // a round's sums (two halves of its columns), to its results
    __device__ __forceinline__ void put(const float (&v)[16], const float (&w)[16], int c0, int lane, char* out,
                                        int64_t out_rs)
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            *reinterpret_cast<float4*>(stage + lane * 32 + 4 * (i ^ (lane & 7))) =
                make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            *reinterpret_cast<float4*>(stage + lane * 32 + 4 * ((4 + i) ^ (lane & 7))) =
                make_float4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
        __syncwarp();
        if (!fours(c0)) {
            if (RUNS) by_one(c0, lane, out, out_rs, t.e.half);
            else if (t.e.half) by_one(c0, lane, out, out_rs, 1);
            else by_one(c0, lane, out, out_rs, 0);
        } else if (RUNS) {
            by_four_runs(c0, out, out_rs);
        } else if (t.e.half) {
            by_four<1>(c0, out, out_rs);
        } else {
            by_four<0>(c0, out, out_rs);
        }
        __syncwarp();
    }

    // `taken`: the barrier that tells the products' thread that this warp has
    // fetched its sums
    __device__ __forceinline__ void fetched(int lane, uint32_t taken)
    {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_at(taken);
    }

    __device__ __forceinline__ void finish(uint32_t tmem, int sums, int lane, char* out, int64_t out_rs, uint32_t taken)
    {
        int c0 = turn * kCols;
        if (c0 >= cols) fetched(lane, taken);
        for (; c0 < cols; c0 += 2 * kCols) {
            float v[16], w[16];
            tmem_load16(v, tmem + c0);
            tmem_load16(w, tmem + c0 + (PAIR ? sums / 2 : 16));
            tmem_load_wait(v, w);
            if (c0 + 2 * kCols >= cols) fetched(lane, taken);
            put(v, w, c0, lane, out, out_rs);
        }
    }

    // RUNS: adds a run to this warp's sums so far, 16 columns each: half a round (of
    // a pair, one weight's), whether the result has them or not
    static __device__ __forceinline__ void add_run(float (&sum)[8][16], uint32_t tmem, int sums)
    {
#pragma unroll
        for (int r = 0; r < 8; r++) {
            float v[16];
            tmem_load16(v, tmem + (r >> 1) * 2 * kCols + (r & 1) * (PAIR ? sums / 2 : 16));
            tmem_load_wait(v);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                if (FINISH == kScaled) sum[r][i] = __int_as_float(__float_as_int(sum[r][i]) + __float2int_rn(v[i]));
                else sum[r][i] += v[i];
            }
        }
    }

    __device__ __forceinline__ void put_runs(float (&sum)[8][16], int lane, char* out, int64_t out_rs)
    {
        if (FINISH == kScaled)   // so far integers
#pragma unroll
            for (int r = 0; r < 8; r++)
#pragma unroll
                for (int i = 0; i < 16; i++) sum[r][i] = float(__float_as_int(sum[r][i]));
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int c0 = turn * kCols + r * 2 * kCols;
            if (c0 < cols) put(sum[2 * r], sum[2 * r + 1], c0, lane, out, out_rs);
        }
    }
};

template <bool PAIR, int FINISH, int ACT, bool RUNS>
__global__ void __launch_bounds__(kThreads, 1) tile_kernel(const __grid_constant__ TileArgs t)
{
    extern __shared__ char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 4];
    __shared__ uint32_t tmem_at, stop;
    char* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages,
                   taken = ready + 16;
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
            bar_init(taken + 8 * i, 2 * kFinishers);   // of both CTAs
        }
        bar_init_fence();
    }
    if (warp == 2) tmem_alloc<2>(smem_addr(&tmem_at), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    const int steps = t.steps * t.segments, runs = RUNS ? t.runs : 1;
    wait_previous();

    if (warp < 2) {
        // ------------------------------------------------ loads, a warp for each operand
        const bool b = warp == 1, mn = b ? t.b_mn : t.a_mn;
        const uint32_t to = smem_addr(base) + (b ? kHalf : 0), there = in_cta(full, 0);
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int i = first; i < t.items && ok; i += pairs) {
            const Item it = item_of<PAIR>(t, i);
            const bool two = mn && (!b || it.sums == 256);   // boxes of 64
            const int row = b ? it.n + (PAIR ? 0 : int(rank) * (it.sums / 2)) : it.m + int(rank) * 128;
            const int bytes = 2 * kHalf + it.sums * kStep * 2;
            for (int seg = 0, k = 0; seg < t.segments && ok; seg++) {
                const CUtensorMap* b_maps = it.sums == 256 ? t.b : t.b_half;
                const CUtensorMap* map = b ? &b_maps[PAIR ? int(rank) : seg] : &t.a[it.twin | seg];
                const int k_last = (seg + 1) * t.steps;
                for (int at = 0; k < k_last; k++, at += kStep) {
                    if (!(ok = bar_wait_warp(empty + 8 * stage, phase ^ 1, waits))) break;
                    if (elected()) {
                        if (!b && rank == 0) bar_expect(full + 8 * stage, bytes);
                        const uint32_t dst = to + stage * kStage, bar = there + 8 * stage;
                        tma_load_pair(dst, map, mn ? row : at, mn ? at : row, bar);
                        if (two) tma_load_pair(dst + kHalf / 2, map, row + 64, at, bar);
                    }
                    if (++stage == kStages) stage = 0, phase ^= 1;
                }
            }
        }
    } else if (warp == 2 && rank == 0) {
        // ------------------------------------------------ products
        const uint64_t a_desc = tile_desc(smem_addr(base), t.a_mn ? kHalf / 2 : 0),
                       b_desc = tile_desc(smem_addr(base) + kHalf, t.b_mn ? kHalf / 2 : 0);
        const uint32_t a_step = (t.a_mn ? 2048 : 32) >> 4, b_step = (t.b_mn ? 2048 : 32) >> 4;   // 16 summed elements
        int stage = 0, acc = 0;
        uint32_t phase = 0, acc_phase = 0;
        bool ok = true;
        for (int i = first; i < t.items && ok; i += pairs) {
            const uint32_t desc = mma_desc(256, i < t.whole ? 256 : 128, t.e.half, t.a_mn, t.b_mn);
            RunEnds ends(steps, runs);
            for (int run = 0, k = 0; run < runs && ok; run++) {
                const int k_last = RUNS ? ends.next() : steps;
                bool add = false;
                if (!(ok = bar_wait_warp(taken + 8 * acc, acc_phase ^ 1, waits))) break;
                tc_fence_after();
                for (; k < k_last; k++) {
                    if (!(ok = bar_wait_warp(full + 8 * stage, phase, waits))) break;
                    tc_fence_after();
                    // addresses stay below 2^18, so the descriptors' fields do not run over
                    const uint32_t on = uint32_t(stage * (kStage >> 4));
                    const uint64_t a = a_desc + on, b = b_desc + on;
                    if (elected()) {
#pragma unroll
                        for (int j = 0; j < kStep / 16; j++)
                            mma_f16<2>(tmem + acc * 256, a + j * a_step, b + j * b_step, desc, add || j > 0);
                        mma_commit_pair(empty + 8 * stage);
                    }
                    add = true;
                    if (++stage == kStages) stage = 0, phase ^= 1;
                }
                if (!ok) break;
                if (elected()) mma_commit_pair(ready + 8 * acc);
                if (++acc == 2) acc = 0, acc_phase ^= 1;
            }
        }
    } else if (warp >= 3) {
        // ------------------------------------------------ results
        const int mine = warp - 3, quarter = warp & 3;   // a warp reaches the 32 lanes of its number's quarter
        Finisher<PAIR, FINISH, ACT, RUNS> f(t, reinterpret_cast<float*>(base + kStages * kStage) + mine * 32 * 32, lane,
                                           mine >> 2);
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int i = first; i < t.items; i += pairs) {
            const Item it = item_of<PAIR>(t, i);
            f.start(int64_t(it.m) + int(rank) * 128 + quarter * 32, it.n, it.sums, lane);
            char* out = it.twin ? t.e.out2 : t.e.out;
            const int64_t out_rs = it.twin ? t.e.out2_rs : t.e.out_rs;
            const uint32_t lanes = tmem + (uint32_t(quarter) << 21);
            if (RUNS) {
                float sum[8][16] = {};
                bool ok = true;
                for (int run = 0; run < runs; run++) {
                    if (!(ok = bar_wait_warp(ready + 8 * acc, acc_phase, waits))) break;
                    tc_fence_after();
                    f.add_run(sum, lanes + acc * 256 + (mine >> 2) * f.kCols, it.sums);
                    f.fetched(lane, in_cta(taken + 8 * acc, 0));
                    if (++acc == 2) acc = 0, acc_phase ^= 1;
                }
                if (!ok) break;
                f.put_runs(sum, lane, out, out_rs);
            } else {
                if (!bar_wait_warp(ready + 8 * acc, acc_phase, waits)) break;
                tc_fence_after();
                f.finish(lanes + acc * 256, it.sums, lane, out, out_rs, in_cta(taken + 8 * acc, 0));
                if (++acc == 2) acc = 0, acc_phase ^= 1;
            }
        }
    }
    // Where all waits of this CTA ended well, the last sums were ready, and so the
    // products and both CTAs' loads that they are made of are done.
    __syncwarp();
    __syncthreads();
    if (stop) settle();
    cluster_sync();
    tc_fence_after();
    if (warp == 2) tmem_free<2>(tmem, 512);
}

}  // namespace

using TileKernel = void (*)(TileArgs);

template <bool PAIR, bool RUNS>
TileKernel tile_kernel_of(int finish, int act)
{
    TileKernel k = nullptr;
    // without an activation a single dz is dy, and no product is finished as one
#define DPDR_CALL(A)                                                                        \
    if ((PAIR || A != DPDR_ACT_NONE) && finish == kSlope) {                                  \
        k = tile_kernel<PAIR, (PAIR || A != DPDR_ACT_NONE ? kSlope : kValue), A, RUNS>;      \
    } else {                                                                                \
        k = tile_kernel<PAIR, kValue, A, RUNS>;                                              \
    }
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return k;
}

}  // namespace proj
}  // namespace dpdr
