// proj_rows.cu -- which kernel of proj_rows.cuh a product takes, how it is
// split, its tensor maps and launch.
#include <algorithm>

#include "proj_rows.cuh"

namespace dpdr {
namespace proj {

RowKernel row_kernel_single(int finish, int act, int split)
{
    return row_kernel_of<false>(finish, act, split);
}

RowKernel row_kernel_pair(int finish, int act, int split);   // proj_rows_pair.cu

int row_launch(Proj* P, const Product& p, cudaStream_t s)
{
    const bool pair = p.kind == kPair, two_x = p.kind == kChain, two_w = pair || two_x;
    RowArgs t;
    t.w_mn = p.b[0].ks != 1;
    t.x_mn = p.a[0].ks != 1;
    t.segments = two_x ? 2 : 1;
    t.steps = int((p.K + kRowStep - 1) / kRowStep);
    t.width = pair ? 64 : kRowFeatures;
    // Tiles of 64 rows where 128 would leave SMs without one, unless the sum is
    // long and four CTAs a tile fill the SMs, when the fewer bytes of larger
    // tiles count: 128 rows of 4096 x 4096 12.5 against 14.9 us, 1024 rows of 1024 x
    // 1024 8.3 against 9.4; 128 rows of 8192 x 8192, 31.8 against 29.4.  With more
    // tiles than SMs, 512 rows of 4096 x 4096, 25.3 against 21.1.
    const int64_t across = (p.N + t.width - 1) / t.width;
    const int steps = t.steps * t.segments;
    t.columns = p.M <= 16 ? 16 : p.M <= 32 ? 32 : p.M <= 64 ? 64 : 128;
    if (t.columns == 128 && (p.M + 63) / 64 * across <= P->num_sms &&
        (steps <= 64 || (p.M + 127) / 128 * across * 4 < P->num_sms))
        t.columns = 64;
    // as many tiles, but of equal height: 130 rows as three of 48
    const int64_t down = (p.M + t.columns - 1) / t.columns;
    if (down > 1) t.columns = int((p.M + down - 1) / down + 15) / 16 * 16;
    t.x_bytes = (t.x_mn ? (t.columns + 63) / 64 * 64 : t.columns) * kRowStep * 2;
    t.M = p.M;
    t.N = p.N;
    t.e = p.e;
    t.vec = by_fours(p.e);
    t.err = P->err;
    const int64_t tiles = across * down;
    // As many CTAs of a cluster as fit beside each other, two an SM, while each
    // still has four stages to load: two rows of 4096 x 4096 with 1, 2, 4 and 8
    // CTAs 15.4, 10.6, 8.6 and 8.5 us; eight rows of a pair of 8192 x 4096 24.0,
    // 23.3, 26.2 and 33.0 (more than two an SM).
    // Clusters leave SMs of their group of SMs unused, and one that finds no
    // place waits for another's whole time, so room is counted for 19/20 of the
    // CTAs with three and four a cluster (16 rows of 4096 x 9728, 76 tiles, 3 and 4:
    // 16.6 and 21.9 us; a pair of 4096 x 2048 and 145 rows, 96 tiles, 2 and 3: 14.7
    // and 13.0) and for 7/8 with more (64 rows of 8192 x 4864, 38 tiles, 6 and 8:
    // 18.6 and 25.6).  Beyond 32 columns, where the partials that the CTAs send
    // each other weigh more, more than four CTAs only with eight stages each: 128
    // rows of 8192 x 1024 with 4 and 8 13.0 and 10.2 us, 333 of 2504 x 1000 with 4
    // and 5 10.3 and 9.5; 2 rows of 2048 x 2048 with 4 and 8 5.3 and 5.1.
    constexpr int kRoom = 110 * 1024;
    int split = 1;
    for (int next = 2; next <= kRowSplits; next++) {
        const int64_t room = int64_t(2 * P->num_sms) * (next > 4 ? 35 : next > 2 ? 38 : 40) / 40;
        if (tiles * next > room || steps < (next > 4 && t.columns > 32 ? 8 : 4) * next) break;
        split = next;
    }
    t.split = split;
    const int stage = kRowFeatures * kRowStep * 2 + t.x_bytes, mine = (steps + split - 1) / split;
    // Runs with columns of their own, for float32 results of 512 products where two
    // CTAs an SM have tensor memory for them (256 columns each): a power of two, no
    // more than the shortest part's steps.  Where those would be longer than a run
    // may be, as many runs as it takes, in turn; a fifth more is let pass (384 rows
    // of 4096 x 4096, 704 products a run, 17.2 against 18.7 us in turn).  The
    // rounding of most 16-bit results hides what one run loses.
    t.apart = 32;
    while (t.apart < t.columns) t.apart *= 2;
    t.runs = 1;
    while (p.e.out_f32 && 2 * t.runs * t.apart <= 256 && t.runs * 8 < mine && 2 * t.runs <= steps / split) t.runs *= 2;
    t.held = t.runs * t.apart;
    t.turns = 0;
    const int most = most_run_steps(p.e.out_f32, p.e.half);
    if (5 * ((mine + t.runs - 1) / t.runs) > 6 * most) {
        t.runs = (mine + most - 1) / most;
        t.turns = 3 * t.apart <= 256 ? 2 : 1;
        t.held = t.turns == 2 ? 4 * t.apart : 256;
    }
    t.stages = std::max(2, std::min({mine, kRoom / stage, kRowMaxStages}));
    const int smem = 1024 + std::max(t.stages * stage, kRowFeatures * t.columns * 4);
    int rc = tensor_map(&t.w[0], p.b[0], p.N, p.K, p.e.half, pair ? 64 : 128, kRowStep);
    if (!rc && two_w) rc = tensor_map(&t.w[1], p.b[1], p.N, p.K, p.e.half, pair ? 64 : 128, kRowStep);
    if (!rc) rc = tensor_map(&t.x[0], p.a[0], p.M, p.K, p.e.half, t.columns, kRowStep);
    if (!rc && two_x) rc = tensor_map(&t.x[1], p.a[1], p.M, p.K, p.e.half, t.columns, kRowStep);
    if (rc) return rc;
    const RowKernel kernel = (pair ? row_kernel_pair : row_kernel_single)(p.e.finish, p.e.act, split);
    bool& set = P->row_set[pair][p.e.finish][p.e.act != DPDR_ACT_NONE][row_split_class(split)];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
        if (e != cudaSuccess) return cuda_fail_c(e, "projection row kernel");
        set = true;
    }
    if (p.sum_parts) *p.sum_parts = down * split;
    return launch(kernel, dim3(unsigned(across * split), unsigned(down)), dim3(kRowThreads), size_t(smem), split, s,
                  "projection row kernel", t);
}

}  // namespace proj
}  // namespace dpdr
