// proj_tile.cu -- which kernel of proj_tile.cuh a product takes, its tensor
// maps and launch; the kernels of one product a tile and one run a sum
// (proj_tile_pair.cu holds the gated operator's, proj_tile_runs.cu and
// proj_tile_pair_runs.cu those of several runs, proj_tile_scaled.cu the one of
// scaled whole numbers, compiled beside them).
#include "proj_tile.cuh"

namespace dpdr {
namespace proj {

TileKernel tile_kernel_single(int finish, int act) { return tile_kernel_of<false, false>(finish, act); }
TileKernel tile_kernel_single_runs(int finish, int act);   // proj_tile_runs.cu
TileKernel tile_kernel_pair(int finish, int act);          // proj_tile_pair.cu
TileKernel tile_kernel_pair_runs(int finish, int act);     // proj_tile_pair_runs.cu
TileKernel tile_kernel_scaled();                           // proj_tile_scaled.cu

int tile_launch(Proj* P, const Product& p, cudaStream_t s)
{
    TileArgs t;
    t.a_mn = p.a[0].ks != 1;
    t.b_mn = p.b[0].ks != 1;
    t.segments = p.kind == kChain ? 2 : 1;
    t.steps = int((p.K + kStep - 1) / kStep);
    const bool scaled = p.e.finish == kScaled;
    const int most = scaled ? kScaledRunSteps : most_run_steps(p.e.out_f32, p.e.half);
    t.runs = (t.steps * t.segments + most - 1) / most;
    const bool runs = scaled || p.e.out_f32 || t.runs > 1;
    const int width = p.kind == kPair ? 128 : 256;
    t.tiles_m = int((p.M + 255) / 256);
    t.tiles_n = int((p.N + width - 1) / width);
    const int64_t tiles = int64_t(t.tiles_m) * t.tiles_n * (p.kind == kTwin ? 2 : 1);
    if (tiles > (int64_t(1) << 30)) return fail_c(DPDR_ERR_INVALID, "projection: more than 2^30 tiles");
    t.tiles = int(tiles);
    // A last round of tiles that fills at most half of the pairs is taken in
    // halves: 4096 x 4096 x 4096 (256 tiles on 76 pairs) with bias and gelu_tanh 97
    // against 109 us, 4096 x 1024 x 4096 28 against 32.
    const int pairs_all = P->num_sms / 2, left = t.tiles % pairs_all;
    t.whole = 2 * left <= pairs_all ? t.tiles - left : t.tiles;
    t.items = t.whole + 2 * (t.tiles - t.whole);
    t.vec = by_fours(p.e);
    t.M = p.M;
    t.N = p.N;
    t.e = p.e;
    t.err = P->err;
    const bool two_a = p.kind == kChain || p.kind == kTwin, two_b = p.kind == kChain || p.kind == kPair;
    int rc = tensor_map(&t.a[0], p.a[0], p.M, p.K, p.e.half, 128, kStep);
    if (!rc && two_a) rc = tensor_map(&t.a[1], p.a[1], p.M, p.K, p.e.half, 128, kStep);
    if (!rc) rc = tensor_map(&t.b[0], p.b[0], p.N, p.K, p.e.half, 128, kStep);
    if (!rc && two_b) rc = tensor_map(&t.b[1], p.b[1], p.N, p.K, p.e.half, 128, kStep);
    if (t.whole < t.tiles) {
        if (!rc) rc = tensor_map(&t.b_half[0], p.b[0], p.N, p.K, p.e.half, 64, kStep);
        if (!rc && two_b) rc = tensor_map(&t.b_half[1], p.b[1], p.N, p.K, p.e.half, 64, kStep);
    }
    if (rc) return rc;
    const TileKernel kernel =
        scaled            ? tile_kernel_scaled()
        : p.kind == kPair ? (runs ? tile_kernel_pair_runs : tile_kernel_pair)(p.e.finish, p.e.act)
                          : (runs ? tile_kernel_single_runs : tile_kernel_single)(p.e.finish, p.e.act);
    // a plan's activation is fixed, but its gradients' products have none
    bool& set = P->tile_set[p.kind == kPair][p.e.finish][p.e.act != DPDR_ACT_NONE][runs];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return cuda_fail_c(e, "projection tile kernel");
        set = true;
    }
    if (p.sum_parts) *p.sum_parts = (p.M + 31) / 32;
    const int pairs = t.items < pairs_all ? t.items : pairs_all;
    return launch(kernel, dim3(unsigned(2 * pairs)), dim3(kThreads), kSmem, 2, s, "projection tile kernel", t);
}

}  // namespace proj
}  // namespace dpdr
