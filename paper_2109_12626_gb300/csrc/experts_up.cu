// experts_up.cu -- the gate and up products of a layer of experts (experts.cu).
#include "experts.cuh"

namespace dpdr {
namespace experts {

using namespace stream;

namespace {

__device__ __forceinline__ void put_hidden(const Layer& l, int pair, int feature, float h)
{
    if (l.terms == 1) {
        reinterpret_cast<float*>(l.hidden)[pair * l.h_pad + feature] = h;
        return;
    }
    uint16_t v[3];
    split_bf16(h, v);
    uint16_t* to = reinterpret_cast<uint16_t*>(l.hidden) + pair * l.h_pad + feature;
    const int64_t apart = l.pairs * l.h_pad;
    to[0] = v[0];
    to[apart] = v[1];
    to[2 * apart] = v[2];
}

// Units of 16 hidden features of an entry
template <int WT, int XT, int NT>
struct Up {
    const Layer& l;
    const Choice& c;
    float* tile;
    const int lane, blocks, units;
    static constexpr int parts = 1;
    static constexpr bool kScales = WT == kI8;
    uint32_t* count;

    __device__ __forceinline__ Up(const Layer& layer, const Choice& choice, float* room, int ln)
        : l(layer),
          c(choice),
          tile(room),
          lane(ln),
          blocks((l.h + 15) / 16),
          units(c.entries * blocks),
          count(l.up_count)
    {
    }
    __device__ __forceinline__ Unit part(int u, int first, int last) const
    {
        const int i = u / blocks, row = (u - i * blocks) * 16;
        Unit q;
        const int64_t e = c.number(i);
#pragma unroll
        for (int k = 0; k < 2; k++) {
            q.a[k] =
                static_cast<const char*>(l.w[k].data) + (e * l.w[k].stride + row * l.w[k].row_stride) * size_of(WT);
            q.a_stride[k] = l.w[k].row_stride * size_of(WT);
        }
        q.rows_left[0] = q.rows_left[1] = min(16, l.h - row);
        q.row_bytes = l.d * size_of(WT);
        q.first = first;
        q.last = last;
        return q;
    }
    __device__ __forceinline__ auto columns(int u) const
    {
        const int i = u / blocks, n = c.count(i), from = c.from(i);
        return [=](int col) {   // columns that there are not repeat the last, for nothing
            return l.x_copy + c.order[from + min(col, n - 1)] / l.top * l.d_pad * size_of(XT);
        };
    }
    // the factors of a lane's rows, 8 apart
    __device__ __forceinline__ void scales(int u, float (&by)[4]) const
    {
        const int i = u / blocks, row = (u - i * blocks) * 16 + lane / 4;
        const int64_t at = int64_t(c.number(i)) * l.h;
#pragma unroll
        for (int k = 0; k < 4; k++) by[k] = l.scale[k / 2][at + min(row + 8 * (k % 2), l.h - 1)];
    }
    // by way of the warp's tile: rows 0 to 15 of it are g, the others u
    __device__ __forceinline__ void finish(int u, const float (&sum)[2][NT][4]) const
    {
        const int i = u / blocks, feature = (u - i * blocks) * 16 + (lane & 15), n = c.count(i), from = c.from(i);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            put_tile(tile, sum[0][t], sum[1][t], lane);
            __syncwarp();
            if (feature < l.h)
#pragma unroll 1
                for (int col = lane >> 4; col < min(8, n - 8 * t); col += 2) {
                    const int pair = c.order[from + 8 * t + col];
                    const float* at = tile + col * kJoinPitch + (lane & 15);
                    put_hidden(l, pair, feature, act_of(l.act, at[0]) * at[16] * c.share[pair]);
                }
            __syncwarp();
        }
    }
};

template <int WT, int XT, int NT, bool SHIFT, bool FEW>
__device__ __forceinline__ void up_units(const Layer& l, const Choice& c, char* raw, int warp, int lane)
{
    constexpr int kPiece = piece_of(WT, XT, NT, SHIFT, 1);
    static_assert((WT == kI8 ? kPad8 : kPad) % (kPiece / size_of(WT)) == 0, "a piece stays in its row of x");
    using S = Stream<WT, XT, NT, SHIFT, 1, kPiece, 1>;
    S st(shared_at(raw), warp, lane);
    const Up<WT, XT, NT> job(l, c, reinterpret_cast<float*>(raw + kRings) + warp * kTile, lane);
    Run<S, NT, Up<WT, XT, NT>> run{st, job, l, (l.d * size_of(WT) + kPiece - 1) / kPiece, lane, warp,
                                   reinterpret_cast<float*>(raw + warp * S::kWarpBytes)};
    run.template go<false>();
}

template <int WT, int XT, bool SHIFT, bool FEW>
__global__ void __launch_bounds__(bound_of(FEW), 2) up_kernel(const __grid_constant__ Layer l)
{
    extern __shared__ __align__(128) char raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kMost = FEW ? 1 : WT == kI8 ? 2 : 4;
    Choice c(raw + kBefore, l.rows * l.top);
    wait_previous();
    allow_next();
    list_all(l, c, raw, 8 * kMost, warp, lane);
    if (FEW || c.columns <= 8) up_units<WT, XT, 1, SHIFT, FEW>(l, c, raw, warp, lane);
    else if (c.columns <= 16) up_units<WT, XT, FEW ? 1 : 2, SHIFT, FEW>(l, c, raw, warp, lane);
    else up_units<WT, XT, kMost, SHIFT, FEW>(l, c, raw, warp, lane);
}

template <bool SHIFT, bool FEW>
Kernel up_of(const Layer& l)
{
    if (l.w_int8) return l.half ? up_kernel<kI8, kF16, SHIFT, FEW> : up_kernel<kI8, kBf16, SHIFT, FEW>;
    return l.half ? up_kernel<kF16, kF16, SHIFT, FEW> : up_kernel<kBf16, kBf16, SHIFT, FEW>;
}

}  // namespace

Kernel up_of(const Layer& l, bool shift, bool few)
{
    if (few) return shift ? up_of<true, true>(l) : up_of<false, true>(l);
    return shift ? up_of<true, false>(l) : up_of<false, false>(l);
}

}  // namespace experts
}  // namespace dpdr
