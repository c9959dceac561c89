// experts.cu -- a layer of experts for a few tokens: which experts each token
// takes, their gated products and the weighted sum of these.
//
//   l = x r^T;  the `top` largest of a token's l, ties to the lowest number
//   share = exp(l - max) over the sum of these (of the chosen, or of all)
//   h_e = share_e act(x wg_e^T) (x wu_e^T);  y = sum_e h_e wd_e^T
//
// Three kernels, each set up while the one before drains: scores_kernel forms l
// and lays x out for the products; up_kernel's CTAs all choose the experts for
// themselves (a few hundred values from L2: less than one CTA doing so and the
// others waiting for it), then stream the chosen experts' gate and up weights
// past the tokens that chose them (stream.cuh), a unit being 16 hidden features
// of an expert; down_kernel does the same with the down weights, a unit being 32
// features of the result of one expert, and the last CTA of those 32 features
// adds up what each token's experts gave, in the order of their shares.  Where there are
// fewer units than CTAs a unit's sum is split along k, and the parts joined in
// order by the last CTA to come.  No CTA waits for another, no sum's order
// depends on timing.
//
// The hidden values are not rounded to 16 bits: they are kept as terms of bfloat16 that
// add up to them (two for a 16-bit result: 2^-16 of a value, far below what the
// result's rounding may be off by; three, which hold all of a float32 value, for a float32
// result), and for float16 weights as float32.
#include <algorithm>
#include <mutex>

#include "experts.h"
#include "stream.cuh"

namespace dpdr {
namespace experts {

using namespace stream;

namespace {

constexpr int kScoreWarps = 4;

// ------------------------------------------------------------------ scores

// A CTA forms the scores of TOK tokens with one expert, and all CTAs lay out x's
// rows.  The products of 16-bit values are exact in float32; a thread sums every
// 128th group of 8 and the threads' sums are added pairwise, so that few
// roundings lie on top of each other: which experts are chosen hangs on these.
// Bound by a trip to memory: each thread asks for all that it needs at once.
template <int TOK, bool VEC>
__global__ void __launch_bounds__(32 * kScoreWarps) scores_kernel(const __grid_constant__ Layer l)
{
    __shared__ float part[kScoreWarps][TOK];
    constexpr int kThreads = 32 * kScoreWarps;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int e = blockIdx.x % l.total, t0 = blockIdx.x / l.total * TOK;
    const uint16_t* x = reinterpret_cast<const uint16_t*>(l.x);
    const uint16_t* r = reinterpret_cast<const uint16_t*>(l.router) + e * l.router_rs;
    if (VEC)   // while the kernel before drains
        for (int k = 64 * int(threadIdx.x); k < l.d; k += 64 * kThreads) asm volatile("prefetch.global.L2 [%0];" ::"l"(r + k));
    wait_previous();
    allow_next();
    float acc[TOK] = {};
    int done = 0;
    if (VEC) {
        const int units = l.d / 8;
        done = units * 8;
#pragma unroll(TOK == 8 ? 1 : 2)
        for (int u = threadIdx.x; u < units; u += kThreads) {
            const uint4 a = *reinterpret_cast<const uint4*>(r + 8 * u);
            uint4 b[TOK];
#pragma unroll
            for (int i = 0; i < TOK; i++)
                b[i] = *reinterpret_cast<const uint4*>(x + min(t0 + i, l.rows - 1) * l.x_rs + 8 * u);
            float f[2][4];
            proj::widen4(make_uint4(a.x, a.y, 0, 0), 0, l.half, f[0]);
            proj::widen4(make_uint4(a.z, a.w, 0, 0), 0, l.half, f[1]);
#pragma unroll
            for (int i = 0; i < TOK; i++) {
                float v[2][4];
                proj::widen4(make_uint4(b[i].x, b[i].y, 0, 0), 0, l.half, v[0]);
                proj::widen4(make_uint4(b[i].z, b[i].w, 0, 0), 0, l.half, v[1]);
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    acc[i] = fmaf(f[0][k], v[0][k], acc[i]);
                    acc[i] = fmaf(f[1][k], v[1][k], acc[i]);
                }
            }
        }
    }
#pragma unroll(VEC || TOK == 8 ? 1 : 4)
    for (int k = done + int(threadIdx.x); k < l.d; k += kThreads) {
        const float f = proj::widen(r[k * l.router_cs], l.half);
#pragma unroll
        for (int i = 0; i < TOK; i++)
            acc[i] = fmaf(f, proj::widen(x[min(t0 + i, l.rows - 1) * l.x_rs + k * l.x_cs], l.half), acc[i]);
    }
#pragma unroll
    for (int i = 0; i < TOK; i++) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], o);
        if (lane == 0) part[warp][i] = acc[i];
    }
    __syncthreads();
    if (threadIdx.x < TOK && t0 + int(threadIdx.x) < l.rows) {
        const int i = threadIdx.x;
        l.logits[int64_t(t0 + i) * l.total + e] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
    }
    // x by rows of d_pad
    const int64_t units = l.rows * (l.d_pad / 8), apart = int64_t(gridDim.x) * blockDim.x;
    for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < units; i += apart) {
        const int64_t t = i / (l.d_pad / 8);
        const int k = int(i - t * (l.d_pad / 8)) * 8;
        uint16_t* to = reinterpret_cast<uint16_t*>(l.x_copy) + t * l.d_pad + k;
        if (VEC && k + 8 <= l.d) {
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(x + t * l.x_rs + k);
        } else {
            uint16_t v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = k + j < l.d ? x[t * l.x_rs + (k + j) * l.x_cs] : uint16_t(0);
            *reinterpret_cast<uint4*>(to) = make_uint4(v[0] | uint32_t(v[1]) << 16, v[2] | uint32_t(v[3]) << 16,
                                                       v[4] | uint32_t(v[5]) << 16, v[6] | uint32_t(v[7]) << 16);
        }
    }
}

// ------------------------------------------------------------------ choice

// What a CTA knows of the choice, in shared memory.  A pair is a token's number
// times `top` plus the place of one of its experts.
struct Choice {
    float* share;         // of a pair
    uint32_t* entry;      // an expert with up to `most` of its pairs: number among
                          // the local ones, how many pairs, the first of them in `order`
    int16_t* expert;      // of a pair
    int16_t* order;       // pairs, those of an expert together, by token
    int entries, columns; // the most pairs of an entry

    __device__ __forceinline__ Choice(char* at, int pairs)
        : share(reinterpret_cast<float*>(at)),
          entry(reinterpret_cast<uint32_t*>(share + pairs)),
          expert(reinterpret_cast<int16_t*>(entry + pairs)),
          order(expert + pairs)
    {
    }
    static __device__ __forceinline__ uint32_t packed(int e, int n, int from)
    {
        return uint32_t(e) | uint32_t(n) << 10 | uint32_t(from) << 17;
    }
    __device__ __forceinline__ int number(int i) const { return entry[i] & 1023u; }
    __device__ __forceinline__ int count(int i) const { return entry[i] >> 10 & 127u; }
    __device__ __forceinline__ int from(int i) const { return entry[i] >> 17; }
};

// Order of scores as whole numbers above 0: NaN highest, -0 as 0
__device__ __forceinline__ uint32_t rank_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The experts of every eighth token, by this warp: lane j the j-th chosen
template <int EACH>
__device__ __forceinline__ void choose(const Layer& l, const Choice& c, int warp, int lane)
{
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    for (int t = warp; t < l.rows; t += kWarps) {
        float v[EACH];
        uint32_t rank[EACH];
#pragma unroll
        for (int j = 0; j < EACH; j++) {
            const int e = lane + 32 * j;
            v[j] = e < l.total ? __ldcg(l.logits + int64_t(t) * l.total + e) : 0.0f;
            rank[j] = e < l.total ? rank_of(v[j]) : 0u;
        }
        int mine = 0;
        float score = 0.0f;
        for (int i = 0; i < l.top; i++) {
            uint32_t best = 0;
            int at = 1 << 30;
            float value = 0.0f;
#pragma unroll
            for (int j = 0; j < EACH; j++)
                if (rank[j] > best) best = rank[j], at = lane + 32 * j, value = v[j];
            const uint32_t most = __reduce_max_sync(kAll, best);
            const int who = int(__reduce_min_sync(kAll, uint32_t(best == most ? at : 1 << 30)));
            value = __shfl_sync(kAll, value, who & 31);
            if (lane == i) mine = who, score = value;
#pragma unroll
            for (int j = 0; j < EACH; j++)
                if (who == lane + 32 * j) rank[j] = 0u;
        }
        const float high = __shfl_sync(kAll, score, 0);
        const float weight = lane < l.top ? expf(score - high) : 0.0f;
        float sum = weight;
        if (!l.normalise) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < EACH; j++)
                if (lane + 32 * j < l.total) sum += expf(v[j] - high);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
        if (lane < l.top) {
            c.share[t * l.top + lane] = weight / sum;
            c.expert[t * l.top + lane] = int16_t(mine);
        }
    }
}

// All of it, in every CTA alike.  `room`: shared memory that is free so far, 10
// bytes for each local expert.  `most`: pairs of an entry.
__device__ void choose_all(const Layer& l, Choice& c, char* room, int most, int warp, int lane)
{
    __shared__ int entries, columns;
    uint64_t* mask = reinterpret_cast<uint64_t*>(room);   // an expert's tokens
    int16_t* from = reinterpret_cast<int16_t*>(mask + l.local);
    const int pairs = l.rows * l.top;
    for (int e = threadIdx.x; e < l.local; e += kThreads) mask[e] = 0;
    if (l.total <= 32) choose<1>(l, c, warp, lane);
    else if (l.total <= 64) choose<2>(l, c, warp, lane);
    else if (l.total <= 128) choose<4>(l, c, warp, lane);
    else choose<16>(l, c, warp, lane);
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += kThreads) {
        const int e = c.expert[p] - l.first;
        if (e >= 0 && e < l.local)
            atomicOr(reinterpret_cast<unsigned long long*>(mask + e), 1ull << (p / l.top));
    }
    __syncthreads();
    if (warp == 0) {
        int pairs_before = 0, entries_before = 0, high = 0;
        for (int e0 = 0; e0 < l.local; e0 += 32) {
            const int e = e0 + lane, n = e < l.local ? __popcll(mask[e]) : 0, k = (n + most - 1) / most;
            int n_to = n, k_to = k;   // up to and with this lane
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int a = __shfl_up_sync(0xFFFFFFFFu, n_to, o), b = __shfl_up_sync(0xFFFFFFFFu, k_to, o);
                if (lane >= o) n_to += a, k_to += b;
            }
            const int p0 = pairs_before + n_to - n, i0 = entries_before + k_to - k;
            if (e < l.local) from[e] = int16_t(p0);
            for (int i = 0; i < k; i++) c.entry[i0 + i] = Choice::packed(e, min(most, n - i * most), p0 + i * most);
            high = max(high, min(n, most));
            pairs_before += __shfl_sync(0xFFFFFFFFu, n_to, 31);
            entries_before += __shfl_sync(0xFFFFFFFFu, k_to, 31);
        }
        high = __reduce_max_sync(0xFFFFFFFFu, high);
        if (lane == 0) entries = entries_before, columns = high;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < l.local; e += kThreads) {
        int at = from[e];
        for (uint64_t m = mask[e]; m; m &= m - 1) {
            const int t = __ffsll(m) - 1;
            int p = t * l.top;
            while (c.expert[p] != e + l.first) p++;
            c.order[at++] = int16_t(p);
        }
    }
    c.entries = entries;
    c.columns = columns;
    __syncthreads();   // `room` is free again
}

// ---------------------------------------------------------------- products

// How many parts a unit's sum is cut into: as many CTAs as there are, while a
// warp keeps two pieces
__device__ __forceinline__ int parts_of(int units, int ctas, int pieces)
{
    if (units == 0) return 1;
    return max(1, min(ctas / units, pieces / (2 * kWarps)));
}

__device__ __forceinline__ float act_of(int act, float z)
{
    float v = z;
#define DPDR_CALL(A) v = proj::act_value<A>(z)
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return v;
}

template <int WT, int XT, int NT, bool SHIFT>
__device__ __forceinline__ void up_units(const Layer& l, const Choice& c, uint32_t ring, float* room, int warp, int lane)
{
    using S = Stream<WT, XT, NT, SHIFT>;
    S st(ring, warp, lane);
    const int blocks = (l.h + 15) / 16, units = c.entries * blocks;
    const int pieces = (l.d * size_of(WT) + kPiece - 1) / kPiece;
    const int parts = parts_of(units, gridDim.x, pieces), all = units * parts;
    auto unit = [&](int u, int& i, int& row) {
        const int part = u % parts, b = u / parts;
        i = b / blocks;
        row = (b - i * blocks) * 16;
        Unit q;
        const int64_t e = c.number(i);
        for (int k = 0; k < 2; k++)
            q.a[k] = static_cast<const char*>(l.w[k].data) + (e * l.w[k].stride + row * l.w[k].row_stride) * size_of(WT);
        q.a_stride[0] = l.w[0].row_stride * size_of(WT);
        q.a_stride[1] = l.w[1].row_stride * size_of(WT);
        q.rows_left[0] = q.rows_left[1] = min(16, l.h - row);
        q.row_bytes = l.d * size_of(WT);
        q.first = int(int64_t(pieces) * part / parts);
        q.last = int(int64_t(pieces) * (part + 1) / parts);
        return q;
    };
    int loading = int(blockIdx.x) - int(gridDim.x);
    auto next = [&]() {
        while (!st.more() && loading + int(gridDim.x) < all) {
            loading += gridDim.x;
            int i, row;
            const Unit q = unit(loading, i, row);
            const int n = c.count(i), from = c.from(i);
            st.load_from(q, [&](int col) {   // columns that there are not repeat the last, for nothing
                return l.x_copy + c.order[from + min(col, n - 1)] / l.top * l.d_pad * size_of(XT);
            });
        }
    };
    st.begin(next);
    for (int u = blockIdx.x; u < all; u += gridDim.x) {
        int i, row;
        const Unit q = unit(u, i, row);
        float sum[2][NT][4], v[NT];
        st.sums(q, sum, next);
#pragma unroll
        for (int n = 0; n < NT; n++) v[n] = join_columns<false>(room, sum[0][n], sum[1][n], warp, lane);
        if (parts > 1) {
            float* mine = l.parts + (int64_t(u) * NT) * kThreads + threadIdx.x;
#pragma unroll
            for (int n = 0; n < NT; n++) mine[n * kThreads] = v[n];
            if (!last_to_come(l.up_count + u / parts, parts)) continue;
            const float* from = l.parts + (int64_t(u / parts) * parts * NT) * kThreads + threadIdx.x;
#pragma unroll
            for (int n = 0; n < NT; n++) v[n] = __ldcg(from + n * kThreads);
            for (int p = 1; p < parts; p++)
#pragma unroll
                for (int n = 0; n < NT; n++) v[n] += __ldcg(from + (p * NT + n) * kThreads);
        }
        // lanes 0 to 15 have g, the others u of the same features
        const int feature = row + (lane & 15), e = c.number(i);
#pragma unroll
        for (int n = 0; n < NT; n++) {
            const int col = n * 8 + warp;
            if (l.scale[0] && feature < l.h) v[n] *= (lane < 16 ? l.scale[0] : l.scale[1])[int64_t(e) * l.h + feature];
            const float up = __shfl_down_sync(0xFFFFFFFFu, v[n], 16);
            if (lane < 16 && feature < l.h && col < c.count(i)) {
                const int pair = c.order[c.from(i) + col];
                const float h = act_of(l.act, v[n]) * up * c.share[pair];
                if (l.terms == 1) {
                    reinterpret_cast<float*>(l.hidden)[pair * l.h_pad + feature] = h;
                } else {
                    uint16_t t[3];
                    split_bf16(h, l.terms, t);
                    for (int k = 0; k < l.terms; k++)
                        reinterpret_cast<uint16_t*>(l.hidden)[(k * int64_t(l.pairs) + pair) * l.h_pad + feature] = t[k];
                }
            }
        }
    }
}

template <int WT, int NT, bool SHIFT, int TERMS>
__device__ __forceinline__ void down_units(const Layer& l, const Choice& c, uint32_t ring, float* room, int warp, int lane)
{
    // float16 weights take the float32 values, others their terms
    constexpr int kXT = TERMS == 1 ? kF32 : kBf16;
    using S = Stream<WT, kXT, NT, SHIFT, TERMS>;
    S st(ring, warp, lane, l.pairs * l.h_pad * size_of(kXT));
    const int blocks = (l.d + 31) / 32, units = c.entries * blocks;
    const int pieces = (l.h * size_of(WT) + kPiece - 1) / kPiece;
    const int parts = parts_of(units, gridDim.x, pieces), all = units * parts, pairs = l.rows * l.top;
    const int64_t stride = l.w[2].row_stride * size_of(WT);
    auto unit = [&](int u, int& i, int& row, int& part) {
        part = u % parts;
        const int b = u / parts;
        i = b / blocks;
        row = (b - i * blocks) * 32;
        Unit q;
        q.a[0] = static_cast<const char*>(l.w[2].data) + (c.number(i) * l.w[2].stride + row * l.w[2].row_stride) * size_of(WT);
        q.a[1] = q.a[0] + 16 * stride;
        q.a_stride[0] = q.a_stride[1] = stride;
        q.rows_left[0] = min(16, l.d - row);
        q.rows_left[1] = max(0, min(16, l.d - row - 16));
        q.row_bytes = l.h * size_of(WT);
        q.first = int(int64_t(pieces) * part / parts);
        q.last = int(int64_t(pieces) * (part + 1) / parts);
        return q;
    };
    // the first unit's weights are asked into L2 while up_kernel drains
    if (int(blockIdx.x) < all) {
        int i, row, part;
        const Unit q = unit(blockIdx.x, i, row, part);
        const int r = threadIdx.x / 8;
        if (r % 16 < q.rows_left[r / 16]) {
            const char* p = q.a[r / 16] + (r % 16) * stride;
            const int to = min(q.last * kPiece, q.row_bytes), from = q.first * kPiece;
            for (int k = from + 128 * int(threadIdx.x % 8); k < min(to, from + 4096); k += 1024)
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p + k));
        }
    }
    wait_previous();
    int loading = int(blockIdx.x) - int(gridDim.x);
    auto next = [&]() {
        while (!st.more() && loading + int(gridDim.x) < all) {
            loading += gridDim.x;
            int i, row, part;
            const Unit q = unit(loading, i, row, part);
            const int n = c.count(i), from = c.from(i);
            st.load_from(q, [&](int col) {
                return l.hidden + c.order[from + min(col, n - 1)] * l.h_pad * size_of(kXT);
            });
        }
    };
    st.begin(next);
    for (int u = blockIdx.x; u < all; u += gridDim.x) {
        int i, row, part;
        const Unit q = unit(u, i, row, part);
        float sum[2][NT][4];
        st.sums(q, sum, next);
        const int feature = row + lane;
#pragma unroll
        for (int n = 0; n < NT; n++) {
            float v = join_columns<false>(room, sum[0][n], sum[1][n], warp, lane);
            const int col = n * 8 + warp;
            if (feature < l.d && col < c.count(i)) {
                if (l.scale[2]) v *= l.scale[2][int64_t(c.number(i)) * l.d + feature];
                l.z[(int64_t(part) * pairs + c.order[c.from(i) + col]) * l.d + feature] = v;
            }
        }
        if (!last_to_come(l.down_count + row / 32, uint32_t(c.entries) * parts)) continue;
        for (int t = warp; t < l.rows; t += kWarps) {
            if (feature >= l.d) continue;
            float y = 0.0f;
            for (int k = 0; k < l.top; k++) {
                const int pair = t * l.top + k, e = c.expert[pair] - l.first;
                if (e < 0 || e >= l.local) continue;
                for (int p = 0; p < parts; p++) y += __ldcg(l.z + (int64_t(p) * pairs + pair) * l.d + feature);
            }
            proj::store1(l.y, t * l.y_rs + feature, y, l.out_f32, l.half);
        }
    }
}

// Bytes of shared memory in front of the choice
constexpr int before_choice(bool shift) { return kWarps * ring_bytes(shift) + kJoin * 4; }

template <int WT, int XT, bool SHIFT>
__global__ void __launch_bounds__(kThreads, 2) up_kernel(const __grid_constant__ Layer l)
{
    extern __shared__ __align__(128) char raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kMost = WT == kI8 ? 2 : 4;
    Choice c(raw + before_choice(SHIFT), l.rows * l.top);
    wait_previous();
    allow_next();
    choose_all(l, c, raw, 8 * kMost, warp, lane);
    if (blockIdx.x == 0)
        for (int p = threadIdx.x; p < l.rows * l.top; p += kThreads) {
            if (l.chosen) l.chosen[p] = c.expert[p];
            if (l.share) l.share[p] = c.share[p];
        }
    float* room = reinterpret_cast<float*>(raw + kWarps * ring_bytes(SHIFT));
    if (c.columns <= 8) up_units<WT, XT, 1, SHIFT>(l, c, shared_at(raw), room, warp, lane);
    else if (c.columns <= 16) up_units<WT, XT, 2, SHIFT>(l, c, shared_at(raw), room, warp, lane);
    else up_units<WT, XT, kMost, SHIFT>(l, c, shared_at(raw), room, warp, lane);
}

// The choice is made again from the scores, which are there: up_kernel let this
// kernel start after it had waited for them.
template <int WT, bool SHIFT, int TERMS>
__global__ void __launch_bounds__(kThreads, 2) down_kernel(const __grid_constant__ Layer l)
{
    extern __shared__ __align__(128) char raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kMost = (WT == kI8 ? 2 : 4) / (TERMS == 3 ? 2 : 1);   // eights of columns that the ring has room for
    Choice c(raw + before_choice(SHIFT), l.rows * l.top);
    choose_all(l, c, raw, 8 * kMost, warp, lane);
    if (c.entries == 0) {   // no token chose an expert that is here
        wait_previous();
        for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < int64_t(l.rows) * l.d;
             i += int64_t(gridDim.x) * kThreads)
            proj::store1(l.y, i / l.d * l.y_rs + i % l.d, 0.0f, l.out_f32, l.half);
        return;
    }
    float* room = reinterpret_cast<float*>(raw + kWarps * ring_bytes(SHIFT));
    if (c.columns <= 8) down_units<WT, 1, SHIFT, TERMS>(l, c, shared_at(raw), room, warp, lane);
    else if (c.columns <= 16) down_units<WT, kMost < 2 ? 1 : 2, SHIFT, TERMS>(l, c, shared_at(raw), room, warp, lane);
    else down_units<WT, kMost, SHIFT, TERMS>(l, c, shared_at(raw), room, warp, lane);
}

using Kernel = void (*)(Layer);

// Whether every row of a stack of matrices starts at a multiple of 16 bytes
bool aligned(const dpdr_matrices& m, int local, int64_t rows, int esize)
{
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows == 1 || m.row_stride * esize % 16 == 0) &&
           (local == 1 || m.stride * esize % 16 == 0);
}

bool up_shifted(const Layer& l)
{
    const int es = l.w_int8 ? 1 : 2;
    return !aligned(l.w[0], l.local, l.h, es) || !aligned(l.w[1], l.local, l.h, es);
}
bool down_shifted(const Layer& l) { return !aligned(l.w[2], l.local, l.d, l.w_int8 ? 1 : 2); }

Kernel up_of(const Layer& l, bool shift)
{
    if (l.w_int8) {
        if (l.half) return shift ? up_kernel<kI8, kF16, true> : up_kernel<kI8, kF16, false>;
        return shift ? up_kernel<kI8, kBf16, true> : up_kernel<kI8, kBf16, false>;
    }
    if (l.half) return shift ? up_kernel<kF16, kF16, true> : up_kernel<kF16, kF16, false>;
    return shift ? up_kernel<kBf16, kBf16, true> : up_kernel<kBf16, kBf16, false>;
}

template <bool SHIFT>
Kernel down_of(const Layer& l)
{
    if (l.w_int8) return l.terms == 2 ? down_kernel<kI8, SHIFT, 2> : down_kernel<kI8, SHIFT, 3>;
    if (l.half) return down_kernel<kF16, SHIFT, 1>;
    return l.terms == 2 ? down_kernel<kBf16, SHIFT, 2> : down_kernel<kBf16, SHIFT, 3>;
}
Kernel down_of(const Layer& l, bool shift) { return shift ? down_of<true>(l) : down_of<false>(l); }

size_t product_smem(const Layer& l, bool shift) { return size_t(before_choice(shift)) + size_t(l.rows) * l.top * 12; }

// The CTAs of a kernel that fit the device at a time, after it may use the shared
// memory that it takes.  That is only raised: another plan may need more.
int resident(Kernel k, size_t bytes, int num_sms, int* ctas)
{
    const void* f = reinterpret_cast<const void*>(k);
    static std::mutex hold;
    std::lock_guard<std::mutex> one(hold);
    cudaFuncAttributes at;
    cudaError_t e = cudaFuncGetAttributes(&at, f);
    if (e == cudaSuccess && size_t(at.maxDynamicSharedSizeBytes) < bytes)
        e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
    int each = 0;
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, f, kThreads, bytes);
    if (e != cudaSuccess) return cuda_fail_c(e, "experts kernel");
    if (each < 1) return fail_c(DPDR_ERR_CUDA, "experts: a kernel does not fit the device");
    *ctas = each * num_sms;
    return DPDR_OK;
}

}  // namespace

int product_ctas(Layer& l, int num_sms)
{
    for (int shift = 0; shift < 2; shift++) {
        const size_t bytes = product_smem(l, shift);
        int rc = resident(up_of(l, shift), bytes, num_sms, &l.up_ctas[shift]);
        if (!rc) rc = resident(down_of(l, shift), bytes, num_sms, &l.down_ctas[shift]);
        if (rc) return rc;
    }
    return DPDR_OK;
}

int launch(const Layer& l, int num_sms, cudaStream_t s)
{
    const bool vec = l.x_cs == 1 && l.router_cs == 1 && reinterpret_cast<uintptr_t>(l.x) % 16 == 0 &&
                     reinterpret_cast<uintptr_t>(l.router) % 16 == 0 && (l.rows == 1 || l.x_rs % 8 == 0) &&
                     (l.total == 1 || l.router_rs % 8 == 0);
    Kernel scores = nullptr;
    int tok = 8;
    if (l.rows == 1) tok = 1, scores = vec ? scores_kernel<1, true> : scores_kernel<1, false>;
    else if (l.rows <= 16) tok = 4, scores = vec ? scores_kernel<4, true> : scores_kernel<4, false>;
    else scores = vec ? scores_kernel<8, true> : scores_kernel<8, false>;
    const int grid = (l.rows + tok - 1) / tok * l.total;
    int rc = proj::launch(scores, dim3(unsigned(grid)), dim3(32 * kScoreWarps), 0, 1, s, "experts' scores", l);
    const bool up = up_shifted(l), down = down_shifted(l);
    if (!rc)
        rc = proj::launch(up_of(l, up), dim3(unsigned(l.up_ctas[up])), dim3(kThreads), product_smem(l, up), 1, s,
                          "experts' up products", l);
    if (!rc)
        rc = proj::launch(down_of(l, down), dim3(unsigned(l.down_ctas[down])), dim3(kThreads), product_smem(l, down), 1, s,
                          "experts' down products", l);
    return rc;
}

}  // namespace experts
}  // namespace dpdr
