// experts_down.cu -- the down products of a layer of experts (experts.cu).
#include "experts.cuh"

namespace dpdr {
namespace experts {

using namespace stream;

namespace {

// Of up to 8 tokens: units of 32 features of the result, their sums over all
// entries one after another, a column a token.  One that did not choose an entry has
// zeros there, whose sums are left out: an infinity or NaN among the entry's weights or
// scales would make them NaN.  Of more: units of 32 features and an entry, their results to
// z by pairs.
template <int WT, int NT, int XT, bool WHOLE>
struct Down {
    const Layer& l;
    const Choice& c;
    float* tile;
    const int lane, blocks, parts, units;
    static constexpr bool kScales = WT == kI8;
    uint32_t* count;

    __device__ __forceinline__ Down(const Layer& layer, const Choice& choice, float* room, int ln)
        : l(layer),
          c(choice),
          tile(room),
          lane(ln),
          blocks((l.d + 31) / 32),
          parts(WHOLE ? c.entries : 1),
          units(WHOLE ? blocks : c.entries * blocks),
          count(l.down_count)
    {
    }
    __device__ __forceinline__ int entry(int p) const { return WHOLE ? p % parts : p / blocks; }
    __device__ __forceinline__ int block(int p) const { return WHOLE ? p / parts : p % blocks; }
    __device__ __forceinline__ Unit part(int p, int first, int last) const
    {
        const int row = block(p) * 32;
        const int64_t stride = l.w[2].row_stride * size_of(WT);
        Unit q;
        q.a[0] = static_cast<const char*>(l.w[2].data) +
                 (c.number(entry(p)) * l.w[2].stride + row * l.w[2].row_stride) * size_of(WT);
        q.a[1] = q.a[0] + 16 * stride;
        q.a_stride[0] = q.a_stride[1] = stride;
        q.rows_left[0] = min(16, l.d - row);
        q.rows_left[1] = max(0, min(16, l.d - row - 16));
        q.row_bytes = l.h * size_of(WT);
        q.first = first;
        q.last = last;
        if (WHOLE) q.counts = c.chose(entry(p));
        return q;
    }
    __device__ __forceinline__ auto columns(int p) const
    {
        const int i = entry(p), n = c.count(i), from = c.from(i);
        return [=](int col) -> const char* {
            int pair = c.order[from + min(col, n - 1)];
            if (WHOLE) {   // the token's, if it chose this entry
                pair = -1;
                for (int k = 0; k < n; k++) {
                    const int p = c.order[from + k];
                    if (p >= col * l.top && p < (col + 1) * l.top) pair = p;
                }
            }
            return pair < 0 ? nullptr : l.hidden + pair * l.h_pad * size_of(XT);
        };
    }
    __device__ __forceinline__ void scales(int p, float (&by)[4]) const
    {
        const int row = block(p) * 32 + lane / 4;
        const int64_t at = int64_t(c.number(entry(p))) * l.d;
#pragma unroll
        for (int k = 0; k < 4; k++) by[k] = l.scale[2][at + min(row + 8 * k, l.d - 1)];
    }
    __device__ __forceinline__ void finish(int u, const float (&sum)[2][NT][4]) const
    {
        const int feature = (WHOLE ? u : u % blocks) * 32 + lane, i = WHOLE ? 0 : u / blocks;
        const int n = WHOLE ? l.rows : c.count(i), from = c.from(i);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            put_tile(tile, sum[0][t], sum[1][t], lane);
            __syncwarp();
            if (feature < l.d)
#pragma unroll 1
                for (int col = 0; col < min(8, n - 8 * t); col++) {
                    const float v = tile[col * kJoinPitch + lane];
                    if (WHOLE) proj::store1(l.y, col * l.y_rs + feature, v, l.out_f32, l.half);
                    else l.z[int64_t(c.order[from + 8 * t + col]) * l.d + feature] = v;
                }
            __syncwarp();
        }
    }
};

template <int WT, int NT, bool SHIFT, int TERMS, bool WHOLE>
__device__ __forceinline__ void down_units(const Layer& l, const Choice& c, char* raw, int warp, int lane)
{
    // float16 weights take the float32 values, others their terms
    constexpr int kXT = TERMS == 1 ? kF32 : kBf16, kPiece = piece_of(WT, kXT, NT, SHIFT, TERMS);
    static_assert(kPad % (kPiece / size_of(WT)) == 0, "a piece stays in its row of hidden values");
    using S = Stream<WT, kXT, NT, SHIFT, TERMS, kPiece, 1, WHOLE>;
    S st(shared_at(raw), warp, lane, l.pairs * l.h_pad * size_of(kXT));
    const Down<WT, NT, kXT, WHOLE> job(l, c, reinterpret_cast<float*>(raw + kRings) + warp * kTile, lane);
    Run<S, NT, Down<WT, NT, kXT, WHOLE>> run{st, job, l, (l.h * size_of(WT) + kPiece - 1) / kPiece, lane, warp,
                                             reinterpret_cast<float*>(raw + warp * S::kWarpBytes)};
    run.template go<true>();
}

// The choice is there: up_kernel let this kernel start after it had waited for it.
template <int WT, bool SHIFT, int TERMS, bool FEW>
__global__ void __launch_bounds__(bound_of(FEW), 2) down_kernel(const __grid_constant__ Layer l)
{
    extern __shared__ __align__(128) char raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // eights of columns that the ring has room for
    constexpr int kMost = FEW ? 1 : (WT == kI8 ? 2 : 4) / (TERMS == 3 || SHIFT ? 2 : 1);
    Choice c(raw + kBefore, l.rows * l.top);
    allow_next();
    list_all(l, c, raw, 8 * kMost, warp, lane);
    if (c.entries == 0) {   // no token chose an expert that is here
        wait_previous();
        for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; FEW && i < int64_t(l.rows) * l.d;
             i += int64_t(gridDim.x) * kThreads)
            proj::store1(l.y, i / l.d * l.y_rs + i % l.d, 0.0f, l.out_f32, l.half);
        return;
    }
    if (FEW || c.columns <= 8) down_units<WT, 1, SHIFT, TERMS, FEW>(l, c, raw, warp, lane);
    else if (c.columns <= 16) down_units<WT, kMost < 2 ? 1 : 2, SHIFT, TERMS, FEW>(l, c, raw, warp, lane);
    else down_units<WT, kMost, SHIFT, TERMS, FEW>(l, c, raw, warp, lane);
}

template <bool SHIFT, bool FEW>
Kernel down_of(const Layer& l)
{
    if (l.w_int8) return down_kernel<kI8, SHIFT, 3, FEW>;
    return l.half ? down_kernel<kF16, SHIFT, 1, FEW> : down_kernel<kBf16, SHIFT, 3, FEW>;
}

}  // namespace

Kernel down_of(const Layer& l, bool shift, bool few)
{
    if (few) return shift ? down_of<true, true>(l) : down_of<false, true>(l);
    return shift ? down_of<true, false>(l) : down_of<false, false>(l);
}

}  // namespace experts
}  // namespace dpdr
