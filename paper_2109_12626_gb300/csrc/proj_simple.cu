// proj_simple.cu -- the projections' products, one output tile a CTA on the
// FP32 units: every kind, stride and size.  Also the element-wise and
// reducing kernels of their gradients.
#include "proj_common.cuh"

namespace dpdr {
namespace proj {

namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

// A CTA sums a 64 x 64 tile over k in steps of 16; a thread holds 4 x 4 of it.
// The tile's rows and columns are strided by 16 over the threads, so that
// neighbouring threads store neighbouring columns.
__global__ void __launch_bounds__(kThreads) product_kernel(const Product p)
{
    __shared__ float sa[kStep][kTile + 1], sb[2][kStep][kTile + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const bool pair = p.kind == kPair;
    const int twin = p.kind == kTwin ? int(blockIdx.z) : 0;
    const int64_t n0 = int64_t(blockIdx.x) * kTile, m0 = int64_t(blockIdx.y) * kTile;
    float acc[2][4][4] = {};
    for (int seg = 0; seg < (p.kind == kChain ? 2 : 1); seg++) {
        const Operand a = p.a[twin ? 1 : seg], b = p.b[seg], b2 = p.b[1];
        for (int64_t k0 = 0; k0 < p.K; k0 += kStep) {
            for (int i = threadIdx.x; i < kTile * kStep; i += kThreads) {
                const int r = i / kStep, c = i % kStep;
                const int64_t k = k0 + c;
                const bool in = k < p.K;
                sa[c][r] = in && m0 + r < p.M ? load1(a.p, (m0 + r) * a.is + k * a.ks, 0, p.e.half) : 0.0f;
                sb[0][c][r] = in && n0 + r < p.N ? load1(b.p, (n0 + r) * b.is + k * b.ks, 0, p.e.half) : 0.0f;
                if (pair)
                    sb[1][c][r] = in && n0 + r < p.N ? load1(b2.p, (n0 + r) * b2.is + k * b2.ks, 0, p.e.half)
                                                     : 0.0f;
            }
            __syncthreads();
            for (int c = 0; c < kStep; c++) {
                float x[4], y[4], z[4];
                for (int i = 0; i < 4; i++) {
                    x[i] = sa[c][ty + 16 * i];
                    y[i] = sb[0][c][tx + 16 * i];
                    z[i] = pair ? sb[1][c][tx + 16 * i] : 0.0f;
                }
                for (int i = 0; i < 4; i++)
                    for (int j = 0; j < 4; j++) {
                        acc[0][i][j] += x[i] * y[j];
                        acc[1][i][j] += x[i] * z[j];
                    }
            }
            __syncthreads();
        }
    }
    const Epilogue& e = p.e;
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= p.M || n >= p.N) continue;
            const float z = acc[0][i][j] + (e.bias ? load1(static_cast<const char*>(e.bias), n, 0, e.half) : 0.0f);
            const float u = acc[1][i][j];
            if (e.pre) {
                e.pre[m * e.pre_rs + n] = z;
                if (pair) e.pre[m * e.pre_rs + e.pre_up + n] = u;
            }
            const float o = e.other ? load1(e.other, m * e.other_rs + n * e.other_cs, e.other_f32, e.half) : 0.0f;
            float v = 0.0f, w = 0.0f;
            finish1(e, pair, z, u, o, v, w);
            store1(twin ? e.out2 : e.out, m * (twin ? e.out2_rs : e.out_rs) + n, v, e.out_f32, e.half);
            if (pair && e.finish == kSlope) store1(e.out2, m * e.out2_rs + n, w, e.out_f32, e.half);
        }
}

__global__ void __launch_bounds__(256) slope_kernel(const Epilogue e, int pair, int64_t rows, int64_t cols)
{
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y) {
        const float g = e.pre ? e.pre[m * e.pre_rs + n] : 0.0f;
        const float u = pair ? e.pre[m * e.pre_rs + e.pre_up + n] : 0.0f;
        const float o = load1(e.other, m * e.other_rs + n * e.other_cs, e.other_f32, e.half);
        float v = 0.0f, w = 0.0f;
        finish1(e, pair, g, u, o, v, w);
        store1(e.out, m * e.out_rs + n, v, e.out_f32, e.half);
        if (pair) store1(e.out2, m * e.out2_rs + n, w, e.out_f32, e.half);
    }
}

// Column sums in a fixed order: each of `parts` row ranges summed by one
// thread a column, then the ranges' sums by one thread a column.
__global__ void __launch_bounds__(256) column_part_kernel(const char* z, int64_t rs, int64_t cs, int f32, int half,
                                                          int64_t rows, int64_t cols, float* part)
{
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
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    float s = 0.0f;
    for (int i = 0; i < parts; i++) s += part[i * cols + n];
    store1(out, n, s, out_f32, half);
}

__global__ void __launch_bounds__(256) pack_kernel(const char* src, int64_t rs, int64_t cs, int f32, int half,
                                                   int64_t rows, int64_t cols, char* dst, int64_t ld)
{
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= cols) return;
    for (int64_t m = blockIdx.y; m < rows; m += gridDim.y)
        store1(dst, m * ld + n, load1(src, m * rs + n * cs, f32, half), 0, half);
}

int launched(const char* what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? DPDR_OK : cuda_fail_c(e, what);
}

unsigned blocks_of(int64_t n) { return unsigned((n + 255) / 256); }
unsigned row_blocks(int64_t rows) { return unsigned(rows < 1024 ? rows : 1024); }

}  // namespace

int product_launch(Proj*, const Product& p, cudaStream_t s)
{
    if (p.M == 0 || p.N == 0) return DPDR_OK;
    const int64_t my = (p.M + kTile - 1) / kTile;
    for (int64_t y0 = 0; y0 < my; y0 += 65535) {   // grid.y holds 16 bits
        Product q = p;
        const int64_t r0 = y0 * kTile;
        q.M = p.M - r0 < 65535 * int64_t(kTile) ? p.M - r0 : 65535 * int64_t(kTile);
        for (auto& a : q.a) a.p += 2 * r0 * a.is;
        q.e.out += r0 * q.e.out_rs * (q.e.out_f32 ? 4 : 2);
        if (q.e.out2) q.e.out2 += r0 * q.e.out2_rs * (q.e.out_f32 ? 4 : 2);
        if (q.e.other) q.e.other += r0 * q.e.other_rs * (q.e.other_f32 ? 4 : 2);
        if (q.e.pre) q.e.pre += r0 * q.e.pre_rs;
        product_kernel<<<dim3(unsigned((p.N + kTile - 1) / kTile), unsigned((q.M + kTile - 1) / kTile),
                              p.kind == kTwin ? 2 : 1), kThreads, 0, s>>>(q);
    }
    return launched("projection");
}

int slope_launch(const Epilogue& e, bool pair, int64_t rows, int64_t cols, cudaStream_t s)
{
    if (rows == 0 || cols == 0) return DPDR_OK;
    slope_kernel<<<dim3(blocks_of(cols), row_blocks(rows)), 256, 0, s>>>(e, pair, rows, cols);
    return launched("projection gradient");
}

int column_sum_parts(int64_t rows) { return int(rows < 64 ? 1 : rows < 16384 ? rows / 64 : 256); }

int column_sums_launch(const char* z, int64_t rs, int64_t cs, int z_f32, int half, int64_t rows, int64_t cols,
                       void* out, int out_f32, float* scratch, cudaStream_t s)
{
    const int parts = column_sum_parts(rows);
    column_part_kernel<<<dim3(blocks_of(cols), parts), 256, 0, s>>>(z, rs, cs, z_f32, half, rows, cols, scratch);
    column_join_kernel<<<blocks_of(cols), 256, 0, s>>>(scratch, parts, cols, static_cast<char*>(out), out_f32,
                                                       half);
    return launched("bias gradient");
}

int pack_launch(const char* src, int64_t rs, int64_t cs, int src_f32, int half, int64_t rows, int64_t cols,
                char* dst, int64_t ld, cudaStream_t s)
{
    if (rows == 0 || cols == 0) return DPDR_OK;
    pack_kernel<<<dim3(blocks_of(cols), row_blocks(rows)), 256, 0, s>>>(src, rs, cs, src_f32, half, rows, cols,
                                                                        dst, ld);
    return launched("operand copy");
}

}  // namespace proj
}  // namespace dpdr
