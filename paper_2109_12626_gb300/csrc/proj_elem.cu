// proj_elem.cu -- the projections' element-wise and reducing kernels: dz from
// kept projections, column sums, copies of operands.
#include "proj_common.cuh"
#include "proj_launch.cuh"

namespace dpdr {
namespace proj {

namespace {

template <bool PAIR, int ACT>
__global__ void __launch_bounds__(256) slope_kernel(const Epilogue e, int64_t rows, int64_t cols)
{
    wait_previous();
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y) {
        const float g = e.pre ? e.pre[m * e.pre_rs + n] : 0.0f;
        const float u = PAIR ? e.pre[m * e.pre_rs + e.pre_up + n] : 0.0f;
        const float o = load1(e.other, m * e.other_rs + n * e.other_cs, e.other_f32, e.half);
        float v = 0.0f, w = 0.0f;
        finish1<PAIR, kSlope, ACT>(g, u, o, v, w);
        store1(e.out, m * e.out_rs + n, v, e.out_f32, e.half);
        if (PAIR) store1(e.out2, m * e.out2_rs + n, w, e.out_f32, e.half);
    }
}

// Column sums in a fixed order: each of `parts` row ranges summed by one
// thread a column, then the ranges' sums by one thread a column.
__global__ void __launch_bounds__(256) column_part_kernel(const char* z, int64_t rs, int64_t cs, int f32, int half,
                                                          int64_t rows, int64_t cols, float* part)
{
    wait_previous();
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    const int64_t per = (rows + gridDim.y - 1) / gridDim.y;
    const int64_t m1 = min(rows, (blockIdx.y + 1) * per);
    float s = 0.0f;
    for (int64_t m = blockIdx.y * per; m < m1; m++) s += load1(z, m * rs + n * cs, f32, half);
    part[blockIdx.y * cols + n] = s;
}

__global__ void __launch_bounds__(256) column_join_kernel(const float* part, int parts, int64_t cols, char* out,
                                                          int out_f32, int half)
{
    wait_previous();
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    float s = 0.0f;
    for (int i = 0; i < parts; i++) s += part[i * cols + n];
    store1(out, n, s, out_f32, half);
}

__global__ void __launch_bounds__(256) pack_kernel(const char* src, int64_t rs, int64_t cs, int f32, int half,
                                                   int64_t rows, int64_t cols, char* dst, int64_t ld)
{
    wait_previous();
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y)
        store1(dst, m * ld + n, load1(src, m * rs + n * cs, f32, half), 0, half);
}

unsigned blocks_of(int64_t n) { return unsigned((n + 255) / 256); }
unsigned row_blocks(int64_t rows) { return unsigned(rows < 1024 ? rows : 1024); }

}  // namespace

int slope_launch(const Epilogue& e, bool pair, int64_t rows, int64_t cols, cudaStream_t s)
{
    if (rows == 0 || cols == 0) return DPDR_OK;
    const dim3 grid(blocks_of(cols), row_blocks(rows));
    void (*kernel)(Epilogue, int64_t, int64_t) = nullptr;
#define DPDR_CALL(A) kernel = pair ? slope_kernel<true, A> : slope_kernel<false, A>
    DPDR_FOR_ACT(e.act, DPDR_CALL)
#undef DPDR_CALL
    return launch(kernel, grid, 256, 0, 1, s, "projection gradient", e, rows, cols);
}

int column_sum_parts(int64_t rows) { return int(rows < 64 ? 1 : rows < 16384 ? rows / 64 : 256); }

int column_sums_launch(const char* z, int64_t rs, int64_t cs, int z_f32, int half, int64_t rows, int64_t cols,
                       void* out, int out_f32, float* scratch, cudaStream_t s)
{
    const int parts = column_sum_parts(rows);
    const int rc = launch(column_part_kernel, dim3(blocks_of(cols), parts), 256, 0, 1, s, "bias gradient", z, rs, cs,
                          z_f32, half, rows, cols, scratch);
    if (rc) return rc;
    return launch(column_join_kernel, dim3(blocks_of(cols)), 256, 0, 1, s, "bias gradient", scratch, parts, cols,
                  static_cast<char*>(out), out_f32, half);
}

int pack_launch(const char* src, int64_t rs, int64_t cs, int src_f32, int half, int64_t rows, int64_t cols,
                char* dst, int64_t ld, cudaStream_t s)
{
    if (rows == 0 || cols == 0) return DPDR_OK;
    return launch(pack_kernel, dim3(blocks_of(cols), row_blocks(rows)), 256, 0, 1, s, "operand copy", src, rs, cs,
                  src_f32, half, rows, cols, dst, ld);
}

}  // namespace proj
}  // namespace dpdr
