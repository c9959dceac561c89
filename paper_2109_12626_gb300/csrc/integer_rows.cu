// integer_rows.cu -- products of 8-bit integers for some rows on the tensor cores,
// both operands widened on the way from memory to shared memory.
//
// Between the rows that streaming the weights past them serves (integer.cu) and
// those whose products keep the tiles of proj_tile.cuh busy, widened copies of the
// weights cost more than the product: 5 bytes moved for each of their bytes.  Here
// sixteen warps load 32 bytes of either operand a thread, two steps ahead, widen
// them to float16 and write them where the tensor core reads them (rows of 64 values
// in the 128-byte swizzle); one more warp issues the products, 128 features by up to
// 128 rows of x.  The sum is split over the CTAs of a cluster, which join their whole
// numbers through its shared memory.
//
// float16 holds 8-bit integers exactly, and float32 sums of 1024 of their products
// too (below 2^24): each run of 8 steps has columns of tensor memory of its own, and
// the runs are added up as integers.
//
// Bound by shared memory: a step's operands come through L1, are written once in 16
// bits and read once by the tensor core (about 1300 cycles for 128 features by 128 rows
// by 128 values, of which the products are 512).  4096 x 4096 weights: 32 rows 10.6 us,
// 128 rows 13.9, 256 rows 20.1 (two tiles of columns), where widened copies and the
// tiles take 26.  From where tiles leave no SMs for parts of the sum these are faster:
// 512 rows 27.5 and 32.7 us.  Features past some thousand go that way too from 65 rows on (128
// rows of 8192 to 28,672 210 us, of which the bytes take 35); this kernel unsplit is not
// measured there.
#include "integer.h"
#include "proj_common.cuh"
#include "proj_launch.cuh"
#include "proj_ptx.cuh"
#include "stream.cuh"

namespace dpdr {
namespace integer {

using namespace proj;

namespace {

constexpr int kFeatures = 128;
constexpr int kHalf = 64;                  // values of a row that lie together for the tensor core
constexpr int kStep = 2 * kHalf;           // and of a stage
constexpr int kRunSteps = kScaledRunSteps * kSumStep / kStep;
constexpr int kWideners = 16;              // warps
constexpr int kThreads = 32 * kWideners + 32;
constexpr int kAhead = 2;                  // steps whose loads are under way; three gained nothing
constexpr int kMostStages = 3;
// CTAs of a cluster.  Clusters of eight do not all find a place at a time: 48 rows of
// 5120 x 2048 17.8 us with them, 12.0 with four
constexpr int kMostSplit = 4;
constexpr int kWBytes = kFeatures * kStep * 2;

struct WideArgs {
    int64_t m, n;
    int k, columns, stages, split, steps, sets, held;   // sets of columns of tensor memory, and all of them
    const char *x, *w;
    int64_t x_rs, w_rs;
    Finish f;
    int vec;
    uint32_t* err;
};

// What a thread holds of a row until it is widened: 16 bytes, or the aligned 16 that
// they begin in and the next.  The row is there as a whole.
template <bool ALIGNED>
struct Held {
    uint4 v[ALIGNED ? 1 : 2];

    __device__ __forceinline__ void load(const char* p, int o)
    {
        const uint4* q = reinterpret_cast<const uint4*>(p - o);
        v[0] = q[0];
        if (!ALIGNED) v[1] = q[1];
    }
    // of the 16 bytes the first `left` are there; none is read of aligned 16 that
    // hold none of them
    __device__ __forceinline__ void load_some(const char* p, int o, int left)
    {
        const uint4* q = reinterpret_cast<const uint4*>(p - o);
        v[0] = make_uint4(0, 0, 0, 0);
        if (left > 0) v[0] = q[0];
        if (!ALIGNED) v[1] = left > 16 - o ? q[1] : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ uint4 bytes(int o) const { return ALIGNED ? v[0] : stream::shifted(v[0], v[1], o); }
    __device__ __forceinline__ uint4 some_bytes(int o, int left) const
    {
        uint4 w = bytes(o);
        auto some = [&](uint32_t x, int n) { return n >= 4 ? x : n <= 0 ? 0u : x & ((1u << 8 * n) - 1); };
        return make_uint4(some(w.x, left), some(w.y, left - 4), some(w.z, left - 8), some(w.w, left - 12));
    }
};

// 16 values as float16 to two places
__device__ __forceinline__ void put_wide(char* first, char* second, const uint4& v)
{
    uint32_t h[8];
    stream::bytes_to_f16(v.x, h[0], h[1]);
    stream::bytes_to_f16(v.y, h[2], h[3]);
    stream::bytes_to_f16(v.z, h[4], h[5]);
    stream::bytes_to_f16(v.w, h[6], h[7]);
    *reinterpret_cast<uint4*>(first) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(second) = make_uint4(h[4], h[5], h[6], h[7]);
}

template <bool ALIGNED>
__global__ void __launch_bounds__(kThreads, 1) wide_kernel(const __grid_constant__ WideArgs a)
{
    extern __shared__ char raw[];
    __shared__ __align__(8) uint64_t bars[2 * kMostStages + 1];
    __shared__ uint32_t tmem_at, stop;
    char* base = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023);
    const int warp = warp_number(), lane = threadIdx.x & 31;
    const int rank = a.split > 1 ? int(cluster_rank()) : 0;
    const uint32_t full = smem_addr(bars), empty = full + 8 * kMostStages, ready = empty + 8 * kMostStages;
    const Waits waits{&stop, a.err};
    const int64_t n0 = int64_t(blockIdx.x / a.split) * kFeatures, m0 = int64_t(blockIdx.y) * a.columns;
    const int cols = int(min(int64_t(a.columns), a.m - m0));
    const int stage_bytes = kWBytes + a.columns * kStep * 2;
    const int k_first = int(int64_t(a.steps) * rank / a.split), k_last = int(int64_t(a.steps) * (rank + 1) / a.split);
    const int apart = a.held / a.sets;

    if (threadIdx.x == 0) {
        stop = 0;
        for (int i = 0; i < a.stages; i++) {
            bar_init(full + 8 * i, kWideners);
            bar_init(empty + 8 * i, 1);
        }
        bar_init(ready, 1);
        bar_init_fence();
    }
    if (warp == kWideners) tmem_alloc<1>(smem_addr(&tmem_at), a.held);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    wait_previous();
    allow_next();

    bool ok = true;
    if (warp < kWideners) {
        // ------------------------------------------------ operands
        // A thread takes 16 values of either half of a row, of w and of x.  Rows that there
        // are not repeat the last, for nothing that is stored.
        const int r = threadIdx.x / 4, quarter = threadIdx.x & 3;
        const char* w = a.w + min(n0 + r, a.n - 1) * a.w_rs + 16 * quarter;
        const char* x = a.x + (m0 + min(r, cols - 1)) * a.x_rs + 16 * quarter;
        const int ow = ALIGNED ? 0 : int(reinterpret_cast<uintptr_t>(w) & 15),
                  ox = ALIGNED ? 0 : int(reinterpret_cast<uintptr_t>(x) & 15);
        const bool room = r < a.columns;
        const int x_half = a.columns * kHalf * 2;
        // steps that lie inside every row, with what is read beside them
        const int whole = (a.k - (ALIGNED ? 0 : 16)) / kStep;
        char* const first = base + r * 128 + 16 * ((2 * quarter) ^ (r & 7));
        char* const second = base + r * 128 + 16 * ((2 * quarter + 1) ^ (r & 7));
        Held<ALIGNED> hw[kAhead][2], hx[kAhead][2];
        auto load = [&](int s, int k) {
            const char *pw = w + k * kStep, *px = x + k * kStep;
            if (k < whole) {
#pragma unroll
                for (int j = 0; j < 2; j++) hw[s][j].load(pw + kHalf * j, ow), hx[s][j].load(px + kHalf * j, ox);
            } else {
                const int left = k < k_last ? a.k - k * kStep - 16 * quarter : 0;
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    hw[s][j].load_some(pw + kHalf * j, ow, left - kHalf * j);
                    hx[s][j].load_some(px + kHalf * j, ox, left - kHalf * j);
                }
            }
        };
#pragma unroll
        for (int s = 0; s < kAhead; s++) load(s, k_first + s);
        int stage = 0;
        uint32_t phase = 0;
        for (int k0 = k_first; k0 < k_last && ok; k0 += kAhead) {
#pragma unroll
            for (int s = 0; s < kAhead; s++) {
                const int k = k0 + s, at = stage * stage_bytes;
                if (k >= k_last) break;
                if (!(ok = bar_wait_warp(empty + 8 * stage, phase ^ 1, waits))) break;
                const int left = a.k - k * kStep - 16 * quarter;
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const int to = at + j * (kWBytes / 2);
                    put_wide(first + to, second + to,
                             k < whole ? hw[s][j].bytes(ow) : hw[s][j].some_bytes(ow, left - kHalf * j));
                }
                if (room)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const int to = at + kWBytes + j * x_half;
                        put_wide(first + to, second + to,
                                 k < whole ? hx[s][j].bytes(ox) : hx[s][j].some_bytes(ox, left - kHalf * j));
                    }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(full + 8 * stage);
                load(s, k + kAhead);
                if (++stage == a.stages) stage = 0, phase ^= 1;
            }
        }
        if (ok) ok = bar_wait_warp(ready, 0, waits);
    } else {
        // ------------------------------------------------ products
        const uint32_t desc = mma_desc(kFeatures, a.columns, 1, 0, 0);
        const uint64_t w_desc = tile_desc(smem_addr(base), 0), x_desc = tile_desc(smem_addr(base) + kWBytes, 0);
        int stage = 0;
        uint32_t phase = 0;
        for (int k = k_first; k < k_last; k++) {
            if (!(ok = bar_wait_warp(full + 8 * stage, phase, waits))) break;
            tc_fence_after();
            const int step = k - k_first;
            const uint32_t on = uint32_t(stage * (stage_bytes >> 4)), sums = tmem + step / kRunSteps * apart;
            if (elected()) {
#pragma unroll
                for (int j = 0; j < kStep / 16; j++) {
                    const uint32_t w_on = on + (j / 4) * (kWBytes / 2 >> 4) + 2 * (j % 4),
                                   x_on = on + (j / 4) * (a.columns * kHalf * 2 >> 4) + 2 * (j % 4);
                    mma_f16<1>(sums, w_desc + w_on, x_desc + x_on, desc, step % kRunSteps != 0 || j > 0);
                }
                mma_commit(empty + 8 * stage);
            }
            if (++stage == a.stages) stage = 0, phase ^= 1;
        }
        if (elected()) mma_commit(ready);
    }
    __syncwarp();
    // The products are done: the stages' memory takes the sums, column by column
    int* part = reinterpret_cast<int*>(base);
    tc_fence_before();
    ok = __syncthreads_and(ok && !stop);
    if (!ok) settle();
    tc_fence_after();
    if (ok && warp < kWideners) {
        const int quarter = warp & 3, runs = (k_last - k_first + kRunSteps - 1) / kRunSteps;
        for (int c0 = (warp >> 2) * 16; c0 < cols; c0 += 4 * kWideners) {
            int sum[16] = {};
            for (int run = 0; run < runs; run++) {
                float t[16];
                tmem_load16(t, tmem + run * apart + c0 + (uint32_t(quarter) << 21));
                tmem_load_wait(t);
#pragma unroll
                for (int i = 0; i < 16; i++) sum[i] += __float2int_rn(t[i]);
            }
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (c0 + i < cols) part[(c0 + i) * kFeatures + quarter * 32 + lane] = sum[i];
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (a.split > 1) cluster_arrive();
    if (warp == kWideners) tmem_free<1>(tmem, a.held);
    if (a.split > 1) cluster_wait();
    if (ok && warp < kWideners) {
        // ------------------------------------------------ results: four features of a column a thread
        const Finish& f = a.f;
        const int at = 4 * lane;
        const int64_t n = n0 + at;
        const bool four = a.vec && n + 3 < a.n;
        float scale[4] = {0.0f, 0.0f, 0.0f, 0.0f}, bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (n + i < a.n) {
                scale[i] = f.w_scale[n + i];
                if (f.bias) bias[i] = f.bias[n + i];
            }
        for (int c = rank + a.split * warp; c < cols && n < a.n; c += a.split * kWideners) {
            const uint32_t from = smem_addr(part + c * kFeatures + at);
            int sum[4] = {0, 0, 0, 0};
            float p[kMostSplit][4];   // of the CTAs, asked for together
#pragma unroll
            for (int s = 0; s < kMostSplit; s++)
                if (s < a.split) cluster_load4(a.split > 1 ? in_cta(from, s) : from, p[s]);
#pragma unroll
            for (int s = 0; s < kMostSplit; s++)
                if (s < a.split)
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[i] += __float_as_int(p[s][i]);
            const int64_t m = m0 + c;
            const float by = f.x_scale[m];
            float o[4] = {0.0f, 0.0f, 0.0f, 0.0f}, y[4];
            if (f.residual) {
                const int64_t at_m = m * f.residual_rs;
                if (four) load4(f.residual, at_m + n, f.out_f32, f.half, o);
                else
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (n + i < a.n) o[i] = load1(f.residual, at_m + (n + i) * f.residual_cs, f.out_f32, f.half);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) y[i] = float(sum[i]) * (by * scale[i]) + bias[i] + o[i];
            if (four) store4(f.y, m * f.y_rs + n, f.out_f32, f.half, y);
            else
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (n + i < a.n) store1(f.y, m * f.y_rs + n + i, y[i], f.out_f32, f.half);
        }
    }
    __syncwarp();
    if (a.split > 1) cluster_sync();   // the others have read this CTA's sums
}

}  // namespace

namespace {

// How a product is cut: column tiles of equal height, a multiple of 16, parts of the
// sum, as many as there are SMs for, each of two steps at least, and sets of columns of
// tensor memory, one a run
struct Cut {
    int64_t across, down;
    int columns, steps, split, sets, held;
};
Cut cut_of(int64_t rows, int64_t n, int64_t k, int num_sms)
{
    Cut c;
    c.down = (rows + 127) / 128;
    c.across = (n + kFeatures - 1) / kFeatures;
    c.columns = int(((rows + c.down - 1) / c.down + 15) / 16 * 16);
    c.steps = int((k + kStep - 1) / kStep);
    c.split = 1;
    while (c.split < kMostSplit && 2 * c.split * c.across * c.down <= num_sms && c.steps >= 4 * c.split) c.split *= 2;
    const int runs = ((c.steps + c.split - 1) / c.split + kRunSteps - 1) / kRunSteps;
    c.sets = 1;
    while (c.sets < runs) c.sets *= 2;
    int apart = 32;
    while (apart < c.columns) apart *= 2;
    c.held = apart * c.sets;
    return c;
}

}  // namespace

bool wide_takes(int64_t rows, int64_t n, int64_t k, int num_sms)
{
    if (n > int64_t(num_sms) * kFeatures || rows > int64_t(num_sms) * 128) return false;
    const Cut c = cut_of(rows, n, k, num_sms);
    return c.split > 1 && c.held <= 512;
}

int wide_launch(const Wide& q, int num_sms, cudaStream_t s)
{
    WideArgs a;
    a.m = q.rows;
    a.n = q.n;
    a.k = q.k;
    a.x = q.x;
    a.w = q.w;
    a.x_rs = q.x_rs;
    a.w_rs = q.w_rs;
    a.f = q.f;
    a.err = q.err;
    const Cut c = cut_of(q.rows, q.n, q.k, num_sms);
    a.columns = c.columns;
    a.steps = c.steps;
    a.split = c.split;
    a.sets = c.sets;
    a.held = c.held;
    const int stage = kWBytes + a.columns * kStep * 2;
    // 128 rows of 4096 x 4096 with 2 and 3 stages 13.9 and 14.2 us, 32 rows 10.8 and 10.6
    a.stages = a.columns > 64 ? 2 : kMostStages;
    auto fits = [](const void* p, int64_t rs, int unit) {
        return reinterpret_cast<uintptr_t>(p) % unit == 0 && rs % unit == 0;
    };
    const int os = q.f.out_f32 ? 4 : 2;
    a.vec = fits(q.f.y, q.f.y_rs * os, 4 * os) &&
            (!q.f.residual || (q.f.residual_cs == 1 && fits(q.f.residual, q.f.residual_rs * os, 4 * os)));
    const bool aligned = fits(q.x, q.rows > 1 ? q.x_rs : 0, 16) && fits(q.w, q.n > 1 ? q.w_rs : 0, 16);
    auto* kernel = aligned ? wide_kernel<true> : wide_kernel<false>;
    const int bytes = 1024 + kMostStages * (kWBytes + 64 * kStep * 2);
    static_assert(kMostStages * (kWBytes + 64 * kStep * 2) >= 2 * (kWBytes + 128 * kStep * 2),
                  "either number of stages fits");
    if (!q.set[aligned]) {
        const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return cuda_fail_c(e, "integer wide kernel");
        q.set[aligned] = true;
    }
    return launch(kernel, dim3(unsigned(c.across * a.split), unsigned(c.down)), dim3(kThreads),
                  size_t(1024 + a.stages * stage), a.split, s, "integer wide kernel", a);
}

}  // namespace integer
}  // namespace dpdr
