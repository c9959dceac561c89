// proj_elem.cu -- the projections' element-wise and reducing kernels: dz from
// kept projections, the bias gradient's column sums, copies of operands.  All
// are bound by the bytes they move.
#include <algorithm>

#include "proj_common.cuh"
#include "proj_launch.cuh"

namespace dpdr {
namespace proj {

namespace {

constexpr int kElemThreads = 256;

// dz (or dg and du) of a block's rows and columns from the kept projections,
// into e.out (and out2) if there is one; the column sums of dz over the block's
// rows into sums[blockIdx.y], from the values before they are rounded.  A
// thread takes four columns (one where VEC is not set) and every blockDim.y-th
// row, two rows asked for before the first is used (four spilled, or halved
// the threads).  4096 x 4096, gelu_tanh, with the sums of its columns: 134 MB
// in 29 us (4.6 TB/s).
template <bool PAIR, int ACT, bool VEC>
__global__ void __launch_bounds__(kElemThreads, 4) slope_kernel(const Epilogue e, int64_t rows, int64_t cols, int64_t per,
                                                             float* sums)
{
    constexpr int kW = VEC ? 4 : 1;
    constexpr int kAhead = 2;
    __shared__ float part[kElemThreads][kW];
    wait_previous();
    const int64_t n = (int64_t(blockIdx.x) * blockDim.x + threadIdx.x) * kW;
    const int64_t m1 = min(rows, (int64_t(blockIdx.y) + 1) * per);
    float sum[kW] = {};
    if (n < cols)
        for (int64_t m0 = int64_t(blockIdx.y) * per + threadIdx.y; m0 < m1; m0 += kAhead * blockDim.y) {
            float g[kAhead][kW], u[kAhead][kW], o[kAhead][kW];
#pragma unroll
            for (int r = 0; r < kAhead; r++) {
                const int64_t m = m0 + r * int64_t(blockDim.y);
#pragma unroll
                for (int i = 0; i < kW; i++) g[r][i] = u[r][i] = o[r][i] = 0.0f;
                if (m >= m1) continue;
                if (VEC) {
                    const char* pre = reinterpret_cast<const char*>(e.pre);
                    if (e.pre) load4(pre, m * e.pre_rs + n, 1, 0, reinterpret_cast<float(&)[4]>(g[r]));
                    if (PAIR) load4(pre, m * e.pre_rs + e.pre_up + n, 1, 0, reinterpret_cast<float(&)[4]>(u[r]));
                    load4(e.other, m * e.other_rs + n, e.other_f32, e.half, reinterpret_cast<float(&)[4]>(o[r]));
                } else {
                    if (e.pre) g[r][0] = e.pre[m * e.pre_rs + n];
                    if (PAIR) u[r][0] = e.pre[m * e.pre_rs + e.pre_up + n];
                    o[r][0] = load1(e.other, m * e.other_rs + n * e.other_cs, e.other_f32, e.half);
                }
            }
#pragma unroll
            for (int r = 0; r < kAhead; r++) {
                const int64_t m = m0 + r * int64_t(blockDim.y);
                if (m >= m1) continue;
                float v[kW], w[kW];
#pragma unroll
                for (int i = 0; i < kW; i++) {
                    w[i] = 0.0f;
                    finish1<PAIR, kSlope, ACT>(g[r][i], u[r][i], o[r][i], v[i], w[i]);
                    sum[i] += v[i];
                }
                if (!e.out) continue;
                if (VEC) {
                    store4(e.out, m * e.out_rs + n, 0, e.half, reinterpret_cast<float(&)[4]>(v));
                    if (PAIR) store4(e.out2, m * e.out2_rs + n, 0, e.half, reinterpret_cast<float(&)[4]>(w));
                } else {
                    store1(e.out, m * e.out_rs + n, v[0], 0, e.half);
                    if (PAIR) store1(e.out2, m * e.out2_rs + n, w[0], 0, e.half);
                }
            }
        }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < kW; i++) part[threadIdx.y * blockDim.x + threadIdx.x][i] = sum[i];
    __syncthreads();
    if (threadIdx.y != 0 || n >= cols) return;
#pragma unroll
    for (int i = 0; i < kW; i++) {
        float s = sum[i];
        for (int y = 1; y < int(blockDim.y); y++) s += part[y * blockDim.x + threadIdx.x][i];
        if (n + i < cols) sums[int64_t(blockIdx.y) * cols + n + i] = s;
    }
}

// The blocks' column sums added up in their order: eight runs of them by
// eight threads, then those.
__global__ void __launch_bounds__(256) join_kernel(const float* sums, int parts, int64_t cols, char* out, int out_f32,
                                                   int half)
{
    __shared__ float run[8][32];
    wait_previous();
    allow_next();
    const int64_t n = int64_t(blockIdx.x) * 32 + threadIdx.x;
    const int per = (parts + 7) / 8, p0 = threadIdx.y * per, p1 = min(parts, p0 + per);
    float s = 0.0f;
    if (n < cols) {
#pragma unroll 8
        for (int i = p0; i < p1; i++) s += sums[int64_t(i) * cols + n];
    }
    run[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y != 0 || n >= cols) return;
    for (int y = 1; y < 8; y++) s += run[y][threadIdx.x];
    store1(out, n, s, out_f32, half);
}

// Eight elements as they lie, loaded by as many bytes at a time as their place
// allows
__device__ __forceinline__ uint4 load8(const uint16_t* p)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    uint4 w;
    if (at % 16 == 0) {
        w = *reinterpret_cast<const uint4*>(p);
    } else if (at % 8 == 0) {
        const uint2 a = *reinterpret_cast<const uint2*>(p), b = *reinterpret_cast<const uint2*>(p + 4);
        w = make_uint4(a.x, a.y, b.x, b.y);
    } else if (at % 4 == 0) {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
        w = make_uint4(q[0], q[1], q[2], q[3]);
    } else {   // the seven halves between the words' ends, and the two at them
        const uint32_t* q = reinterpret_cast<const uint32_t*>(p + 1);
        const uint32_t a = p[0], b = q[0], c = q[1], d = q[2], e = p[7];
        w = make_uint4(a | b << 16, b >> 16 | c << 16, c >> 16 | d << 16, d >> 16 | e << 16);
    }
    return w;
}

// The copies of one call, one a blockIdx.y.  A thread copies eight elements of a
// row at a time, two such before it stores the first, by 16 bytes.  4096 x 4099
// (rows at every second byte): 67 MB moved in 15 us (4.4 TB/s).
__global__ void __launch_bounds__(256) copy_kernel(const Copies c)
{
    wait_previous();
    allow_next();
    const Copies::Job& j = c.job[blockIdx.y];
    const uint64_t units = uint64_t(j.cols + 7) / 8, all = units * uint64_t(j.rows), apart = uint64_t(gridDim.x) * 256;
    for (uint64_t i0 = uint64_t(blockIdx.x) * 256 + threadIdx.x; i0 < all; i0 += 2 * apart) {
        uint4 w[2];
        uint16_t* q[2] = {nullptr, nullptr};
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint64_t i = i0 + h * apart;
            if (i >= all) continue;
            const uint64_t m = all >> 32 ? i / units : uint32_t(i) / uint32_t(units);
            const int64_t n = int64_t(i - m * units) * 8;
            const uint16_t* p = reinterpret_cast<const uint16_t*>(j.src) + int64_t(m) * j.rs + n * j.cs;
            uint16_t* to = reinterpret_cast<uint16_t*>(j.dst) + int64_t(m) * j.ld + n;
            if (j.cs == 1 && n + 8 <= j.cols) {
                w[h] = load8(p);
                q[h] = to;
            } else {
                const int some = int(min(int64_t(8), j.cols - n));
                for (int k = 0; k < some; k++) to[k] = p[k * j.cs];
            }
        }
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (q[h]) *reinterpret_cast<uint4*>(q[h]) = w[h];
    }
}

// threads along `units` of a row, the rest along the rows
dim3 block_for(int64_t units)
{
    unsigned x = 32;
    while (x < unsigned(kElemThreads) && x < units) x *= 2;
    return dim3(x, unsigned(kElemThreads) / x);
}

}  // namespace

// Blocks down the rows: 16 rows each, but of few rows as many as keep the SMs
// at work
int column_sum_parts(int64_t rows)
{
    return int(std::min<int64_t>(std::max<int64_t>((rows + 15) / 16, std::min<int64_t>(rows, 64)), 512));
}

int slope_launch(const Epilogue& e, bool pair, int64_t rows, int64_t cols, float* sums, cudaStream_t s)
{
    // fours: as for an epilogue, and no ragged last group
    const bool vec = by_fours(e) && cols % 4 == 0;
    const int64_t units = vec ? cols / 4 : cols;
    const dim3 block = block_for(units);
    const int parts = column_sum_parts(rows);
    const int64_t per = (rows + parts - 1) / parts;
    const dim3 grid(unsigned((units + block.x - 1) / block.x), unsigned(parts));
    void (*kernel)(Epilogue, int64_t, int64_t, int64_t, float*) = nullptr;
#define DPDR_CALL(A)                                                                       \
    kernel = vec ? (pair ? slope_kernel<true, A, true> : slope_kernel<false, A, true>)     \
                 : (pair ? slope_kernel<true, A, false> : slope_kernel<false, A, false>)
    DPDR_FOR_ACT(e.act, DPDR_CALL)
#undef DPDR_CALL
    return launch(kernel, grid, block, 0, 1, s, "projection gradient", e, rows, cols, per, sums);
}

int join_launch(const float* sums, int parts, int64_t cols, void* out, int out_f32, int half, cudaStream_t s)
{
    return launch(join_kernel, dim3(unsigned((cols + 31) / 32)), dim3(32, 8), 0, 1, s, "bias gradient", sums, parts,
                  cols, static_cast<char*>(out), out_f32, half);
}

int copies_launch(Proj* P, const Copies& c, cudaStream_t s)
{
    int64_t most = 0;
    for (int i = 0; i < c.n; i++) most = std::max(most, c.job[i].rows * ((c.job[i].cols + 7) / 8));
    const unsigned blocks = unsigned(std::min<int64_t>((most + 511) / 512, int64_t(P->num_sms) * 16));
    return launch(copy_kernel, dim3(blocks, unsigned(c.n)), dim3(256), 0, 1, s, "operand copy", c);
}

}  // namespace proj
}  // namespace dpdr
