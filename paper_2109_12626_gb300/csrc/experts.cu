// experts.cu -- a layer of experts for a few tokens: which experts each token
// takes, their gated products and the weighted sum of these.
//
//   l = x r^T;  the `top` largest of a token's l, ties to the lowest number
//   share = exp(l - max) over the sum of these (of the chosen, or of all)
//   h_e = share_e act(x wg_e^T) (x wu_e^T);  y = sum_e h_e wd_e^T
//
// Three kernels, each set up while the one before drains: scores_kernel forms l,
// chooses, and lays x out for the products; up_kernel streams the chosen experts'
// gate and up weights past the tokens that chose them (stream.cuh), a unit being 16 hidden features
// of an expert; down_kernel does the same with the down weights, a unit being 32
// features of the result.  Up to 8 tokens have a column each there, and the sum runs
// through all experts; more have their results by expert, which combine_kernel
// adds up in the order of the shares.
//
// All pieces of all units are dealt out to the warps in equal contiguous shares, or
// where units are few each to a team of warps.  A unit that lies in several shares, or
// a team in several CTAs, is finished by the last of its warps (CTAs) to come, which adds
// up their sums in order: none waits for another, no sum's order depends on timing.  (A CTA a unit, its sum over
// eight warps, with two barriers and a fence each: 8 rows of 64 experts of 2048 x
// 1024 125 us.)
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

// warps of a CTA that forms scores: room beside the product kernels of few tokens,
// and one for each token whose experts it chooses
constexpr int score_warps(int tok) { return tok == 8 ? 8 : 4; }

// ------------------------------------------------------------------ scores

// Order of scores as whole numbers above 0: NaN highest, -0 as 0
__device__ __forceinline__ uint32_t rank_of(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The experts of token t, by a warp: lane j the j-th chosen
template <int EACH>
__device__ __forceinline__ void choose(const Layer& l, int t, int lane)
{
    constexpr uint32_t kAll = 0xFFFFFFFFu;
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
        const int pair = t * l.top + lane;
        l.expert[pair] = mine;
        l.shares[pair] = weight / sum;
        if (l.chosen) l.chosen[pair] = mine;
        if (l.share) l.share[pair] = weight / sum;
    }
}

// A CTA forms the scores of TOK tokens with one expert, and all CTAs lay out x's
// rows.  The products of 16-bit values are exact in float32; a thread sums every
// 128th or 256th group of 8 and the threads' sums are added pairwise, so that few
// roundings lie on top of each other: which experts are chosen hangs on these.  The
// last CTA of the tokens' to come chooses for them: once for all, since a choice in
// every CTA of the product kernels took those 20 us each with 64 tokens of 128.
// Bound by a trip to memory: each thread asks for all that it needs at once.
template <int TOK, bool VEC>
__global__ void __launch_bounds__(32 * score_warps(TOK), TOK == 8 ? 3 : 8) scores_kernel(const __grid_constant__ Layer l)
{
    constexpr int kScoreWarps = score_warps(TOK);
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
        float sum[kScoreWarps];
#pragma unroll
        for (int w = 0; w < kScoreWarps; w++) sum[w] = part[w][i];
#pragma unroll
        for (int o = kScoreWarps / 2; o > 0; o /= 2)
#pragma unroll
            for (int w = 0; w < o; w++) sum[w] += sum[w + o];
        l.logits[int64_t(t0 + i) * l.total + e] = sum[0];
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
    if (last_to_come(l.score_count + blockIdx.x / l.total, uint32_t(l.total)))
        for (int t = t0 + warp; t < min(t0 + TOK, l.rows); t += kScoreWarps) {
            if (l.total <= 32) choose<1>(l, t, lane);
            else if (l.total <= 64) choose<2>(l, t, lane);
            else if (l.total <= 128) choose<4>(l, t, lane);
            else choose<16>(l, t, lane);
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

// The lists of it, in every CTA alike.  `room`: shared memory that is free so far, 10
// bytes for each local expert.  `most`: pairs of an entry.
__device__ void list_all(const Layer& l, Choice& c, char* room, int most, int warp, int lane)
{
    __shared__ int entries, before[kWarps], high[kWarps];
    const int pairs = l.rows * l.top;
    if (l.rows == 1) {   // a pair an entry
        if (warp == 0) {
            const int e = lane < pairs ? __ldcg(l.expert + lane) - l.first : -1;
            const float share = lane < pairs ? __ldcg(l.shares + lane) : 0.0f;
            const bool here = e >= 0 && e < l.local;
            const uint32_t all = __ballot_sync(0xFFFFFFFFu, here);
            const int at = __popc(all & ((1u << lane) - 1));
            if (here) c.entry[at] = Choice::packed(e, 1, at), c.order[at] = int16_t(lane);
            if (lane < pairs) c.share[lane] = share;
            if (lane == 0) entries = __popc(all);
        }
        __syncthreads();
        c.entries = entries;
        c.columns = 1;
        return;
    }
    uint64_t* mask = reinterpret_cast<uint64_t*>(room);   // an expert's tokens
    int16_t* from = reinterpret_cast<int16_t*>(mask + l.local);
    for (int e = threadIdx.x; e < l.local; e += kThreads) mask[e] = 0;
    for (int p = threadIdx.x; p < pairs; p += kThreads) {
        c.expert[p] = int16_t(__ldcg(l.expert + p));
        c.share[p] = __ldcg(l.shares + p);
    }
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += kThreads) {   // its own
        const int e = c.expert[p] - l.first, t = p / l.top;
        if (e >= 0 && e < l.local) atomicOr(reinterpret_cast<uint32_t*>(mask + e) + t / 32, 1u << t % 32);
    }
    __syncthreads();
    // a thread one or two experts next to each other: their pairs, and their entries above
    // those, added up over the threads before
    static_assert(kMostExperts <= 2 * kThreads, "two experts a thread");
    const int each = l.local > kThreads ? 2 : 1, e0 = each * threadIdx.x;
    int n[2] = {0, 0}, sum = 0;
    for (int i = 0; i < each && e0 + i < l.local; i++) {
        n[i] = __popcll(mask[e0 + i]);
        sum += n[i] | (n[i] + most - 1) / most << 16;
    }
    int to = sum;   // up to and with this thread
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, to, o);
        if (lane >= o) to += v;
    }
    const int top = __reduce_max_sync(0xFFFFFFFFu, max(n[0], n[1]));
    if (lane == 31) before[warp] = to, high[warp] = top;
    __syncthreads();
    int all = 0;
    c.columns = 0;
#pragma unroll
    for (int w = 0; w < kWarps; w++) {
        if (w < warp) to += before[w];
        all += before[w];
        c.columns = max(c.columns, min(most, high[w]));
    }
    c.entries = all >> 16;
    int p0 = (to - sum) & 0xFFFF, i0 = (to - sum) >> 16;
    for (int i = 0; i < each && e0 + i < l.local; i++) {
        from[e0 + i] = int16_t(p0);
        for (int k = 0; k < n[i]; k += most) c.entry[i0++] = Choice::packed(e0 + i, min(most, n[i] - k), p0 + k);
        p0 += n[i];
    }
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += kThreads) {
        const int e = c.expert[p] - l.first, t = p / l.top;
        if (e >= 0 && e < l.local) c.order[from[e] + __popcll(mask[e] & ((1ull << t) - 1))] = int16_t(p);
    }
    __syncthreads();   // `room` is free again
}

// Whether every row of a stack of matrices starts at a multiple of 16 bytes
__host__ __device__ bool aligned(const dpdr_matrices& m, int local, int64_t rows, int esize)
{
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (rows == 1 || m.row_stride * esize % 16 == 0) &&
           (local == 1 || m.stride * esize % 16 == 0);
}

__host__ __device__ bool up_shifted(const Layer& l)
{
    const int es = l.w_int8 ? 1 : 2;
    return !aligned(l.w[0], l.local, l.h, es) || !aligned(l.w[1], l.local, l.h, es);
}
__host__ __device__ bool down_shifted(const Layer& l) { return !aligned(l.w[2], l.local, l.d, l.w_int8 ? 1 : 2); }

// ---------------------------------------------------------------- products

__device__ __forceinline__ float act_of(int act, float z)
{
    float v = z;
#define DPDR_CALL(A) v = proj::act_value<A>(z)
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return v;
}

constexpr int kAsked = 8192;   // bytes that a warp asks into L2 ahead

// What a warp does with its pieces: job.part(i) is the i-th run of `each` pieces along
// k, job.parts of them a unit; job.columns(i) where its columns lie; job.finish(u,
// sums).
template <typename S, int NT, typename Job>
struct Run {
    S& st;
    const Job& job;
    const Layer& l;
    const int each, lane, warp;
    float* const room;   // of this warp, NT tiles, once its loads are done

    // Asks the first of pieces [at, end) into L2
    __device__ __forceinline__ void ask(int at, int end) const
    {
        end = min(end, at + kAsked / (kRows * S::kPiece));
        while (at < end) {
            const int i = at / each, there = min(end, (i + 1) * each);
            const Unit q = job.part(i, at - i * each, there - i * each);
            const char* p = q.row(lane);
            const int to = min(q.last * S::kPiece, q.row_bytes);
            for (int k = q.first * S::kPiece; k < to; k += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + k));
            at = there;
        }
    }

    // Pieces [at, to) of one unit added to `sum`
    template <typename Next>
    __device__ __forceinline__ void sums(int at, int to, float (&sum)[2][NT][4], Next next)
    {
        S::clear(sum);
        while (at < to) {
            const int i = at / each, there = min(to, (i + 1) * each);
            const Unit q = job.part(i, at - i * each, there - i * each);
            if constexpr (Job::kScales) {   // of this part's rows
                float part[2][NT][4], by[4];
                S::clear(part);
                st.sums(q, part, next);
                job.scales(i, by);
#pragma unroll
                for (int k = 0; k < 2; k++)
#pragma unroll
                    for (int n = 0; n < NT; n++)
#pragma unroll
                        for (int j = 0; j < 4; j++) sum[k][n][j] += part[k][n][j] * by[2 * k + j / 2];
            } else {
                st.sums(q, sum, next);
            }
            at = there;
        }
    }

    __device__ __forceinline__ auto loads(int& loading, int end)
    {
        return [this, &loading, end]() {
            if (loading >= end) return;
            const int i = loading / each, to = min(end, (i + 1) * each);
            st.load_from(job.part(i, loading - i * each, to - i * each), job.columns(i));
            loading = to;
        };
    }

    // Many units: contiguous shares; one that a unit begins or ends in leaves its part.
    // Warps next to each other are of different CTAs.
    template <bool ASK>
    __device__ __forceinline__ void shares()
    {
        const int id = warp * gridDim.x + blockIdx.x, per = job.parts * each, total = job.units * per;
        const Shares s(total, max(1, min(int(gridDim.x) * kWarps, total / kLeast)), per);
        int at = s.start(min(id, s.of)), loading = at;
        const int end = s.start(min(id + 1, s.of));
        if (ASK) {
            ask(at, end);
            wait_previous();
        }
        auto next = loads(loading, end);
        st.begin(next);
        while (at < end) {
            const int u = at / per, to = min(end, (u + 1) * per);
            float sum[2][NT][4];
            sums(at, to, sum, next);
            const bool some = to - at < per;
            at = to;
            if (some) {
                const int from = u * per, first = s.owner(from), last = s.owner(from + per - 1);
                auto place = [&](int w) { return l.parts + (int64_t(w) * 2 + (s.start(w) < from)) * (NT * 256); };
                if (!join_parts<NT>(sum, id, first, last, place, job.count + first, lane)) continue;
            }
            job.finish(u, sum);
        }
    }

    // Few: teams of warps that follow each other; those of one CTA join their sums in
    // its shared memory.
    template <bool ASK>
    __device__ __forceinline__ void teams()
    {
        const int per = job.parts * each;
        const Teams t{job.units, int(gridDim.x) * kWarps, per};
        const int base = int(blockIdx.x) * kWarps, id = base + warp;
        const int u = t.unit(id), begins = t.start(u), size = t.size(u), place_of = id - begins;
        const bool in = place_of < size;
        const int from = u * per, at = in ? from + int(int64_t(per) * place_of / size) : 0,
                  end = in ? from + int(int64_t(per) * (place_of + 1) / size) : 0;
        if (ASK) {
            ask(at, end);
            wait_previous();
        }
        int loading = at;
        auto next = loads(loading, end);
        st.begin(next);
        float sum[2][NT][4];
        sums(at, end, sum, next);
        // of the team, the warps of this CTA
        const int low = max(0, begins - base), high = min(kWarps, begins + size - base);
        if (size > 1) {
            copies_wait<0>();
            if (in && warp > low)
#pragma unroll
                for (int n = 0; n < NT; n++) put_tile(room + n * kTile, sum[0][n], sum[1][n], lane);
            __syncwarp();
        }
        __syncthreads();
        if (!in || warp > low) return;
        for (int w = low + 1; w < high; w++) {
            const float* other = room + (w - warp) * (S::kWarpBytes / 4);
#pragma unroll
            for (int n = 0; n < NT; n++) add_tile(other + n * kTile, sum[0][n], sum[1][n], lane);
        }
        if (high - low < size) {   // at most two of a CTA's units reach into others
            const int first = begins / kWarps, last = (begins + size - 1) / kWarps;
            auto place = [&](int c) { return l.parts + (int64_t(c) * 2 + (c == first)) * (NT * 256); };
            if (!join_parts<NT>(sum, int(blockIdx.x), first, last, place, job.count + first, lane)) return;
        }
        job.finish(u, sum);
    }

    // ASK: the first weights are asked into L2 while the kernel before drains, which is
    // then waited for
    template <bool ASK>
    __device__ __forceinline__ void go()
    {
        if (job.units <= 0) return;
        if (2 * job.units <= int(gridDim.x) * kWarps) teams<ASK>();
        else shares<ASK>();
    }
};

__device__ __forceinline__ void put_hidden(const Layer& l, int pair, int feature, float h)
{
    if (l.terms == 1) {
        reinterpret_cast<float*>(l.hidden)[pair * l.h_pad + feature] = h;
        return;
    }
    uint16_t v[3];
    split_bf16(h, l.terms, v);
    uint16_t* to = reinterpret_cast<uint16_t*>(l.hidden) + pair * l.h_pad + feature;
    const int64_t apart = l.pairs * l.h_pad;
    to[0] = v[0];
    to[apart] = v[1];
    if (l.terms == 3) to[2 * apart] = v[2];
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
        : l(layer), c(choice), tile(room), lane(ln), blocks((l.h + 15) / 16), units(c.entries * blocks), count(l.up_count)
    {
    }
    __device__ __forceinline__ Unit part(int u, int first, int last) const
    {
        const int i = u / blocks, row = (u - i * blocks) * 16;
        Unit q;
        const int64_t e = c.number(i);
#pragma unroll
        for (int k = 0; k < 2; k++) {
            q.a[k] = static_cast<const char*>(l.w[k].data) + (e * l.w[k].stride + row * l.w[k].row_stride) * size_of(WT);
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

// Of up to 8 tokens: units of 32 features of the result, their sums over all
// entries one after another, a column a token; one that did not choose an entry has
// zeros there.  Of more: units of 32 features and an entry, their results to
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

// bytes of shared memory in front of the choice: rings, then tiles
constexpr int kRings = kWarps * kRing, kBefore = kRings + kJoin * 4;

// Bytes of a row of weights that a stage holds: as many as let the ring hold two
constexpr int piece_of(int wt, int xt, int nt, bool shift, int terms)
{
    const int stage = kRows * (128 + 16 * shift) + terms * nt * 8 * (128 / size_of(wt)) * size_of(xt);
    return 5 * stage <= kRing ? 128 : 64;
}

template <int WT, int XT, int NT, bool SHIFT, bool FEW>
__device__ __forceinline__ void up_units(const Layer& l, const Choice& c, char* raw, int warp, int lane)
{
    constexpr int kPiece = piece_of(WT, XT, NT, SHIFT, 1);
    using S = Stream<WT, XT, NT, SHIFT, 1, kPiece, 1>;
    S st(shared_at(raw), warp, lane);
    const Up<WT, XT, NT> job(l, c, reinterpret_cast<float*>(raw + kRings) + warp * kTile, lane);
    Run<S, NT, Up<WT, XT, NT>> run{st, job, l, (l.d * size_of(WT) + kPiece - 1) / kPiece, lane, warp,
                                   reinterpret_cast<float*>(raw + warp * S::kWarpBytes)};
    run.template go<false>();
}

template <int WT, int NT, bool SHIFT, int TERMS, bool WHOLE>
__device__ __forceinline__ void down_units(const Layer& l, const Choice& c, char* raw, int warp, int lane)
{
    // float16 weights take the float32 values, others their terms
    constexpr int kXT = TERMS == 1 ? kF32 : kBf16, kPiece = piece_of(WT, kXT, NT, SHIFT, TERMS);
    using S = Stream<WT, kXT, NT, SHIFT, TERMS, kPiece, 1, WHOLE>;
    S st(shared_at(raw), warp, lane, l.pairs * l.h_pad * size_of(kXT));
    const Down<WT, NT, kXT, WHOLE> job(l, c, reinterpret_cast<float*>(raw + kRings) + warp * kTile, lane);
    Run<S, NT, Down<WT, NT, kXT, WHOLE>> run{st, job, l, (l.h * size_of(WT) + kPiece - 1) / kPiece, lane, warp,
                                             reinterpret_cast<float*>(raw + warp * S::kWarpBytes)};
    run.template go<true>();
}

// FEW: up to 8 tokens.  These kernels hold the code for one eight of columns alone,
// and leave registers (of 288 threads, in the bounds) for the next call's
// scores_kernel to be set up beside them.
constexpr int bound_of(bool few) { return few ? kThreads + 32 : kThreads; }

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

// What each token's experts gave, added up in the order of their shares
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ Layer l)
{
    wait_previous();
    allow_next();
    const int t = blockIdx.y;
    const int feature = blockIdx.x * 256 + threadIdx.x;
    if (feature >= l.d) return;
    float v[kMostTop];
#pragma unroll
    for (int k = 0; k < kMostTop; k++) {
        v[k] = 0.0f;
        if (k >= l.top) continue;
        const int pair = t * l.top + k, e = l.expert[pair] - l.first;
        if (e >= 0 && e < l.local) v[k] = l.z[int64_t(pair) * l.d + feature];
    }
    float y = v[0];
#pragma unroll
    for (int k = 1; k < kMostTop; k++) y += v[k];
    proj::store1(l.y, t * l.y_rs + feature, y, l.out_f32, l.half);
}

using Kernel = void (*)(Layer);

template <bool SHIFT, bool FEW>
Kernel up_of(const Layer& l)
{
    if (l.w_int8) return l.half ? up_kernel<kI8, kF16, SHIFT, FEW> : up_kernel<kI8, kBf16, SHIFT, FEW>;
    return l.half ? up_kernel<kF16, kF16, SHIFT, FEW> : up_kernel<kBf16, kBf16, SHIFT, FEW>;
}
Kernel up_of(const Layer& l, bool shift, bool few)
{
    if (few) return shift ? up_of<true, true>(l) : up_of<false, true>(l);
    return shift ? up_of<true, false>(l) : up_of<false, false>(l);
}

template <bool SHIFT, bool FEW>
Kernel down_of(const Layer& l)
{
    if (l.w_int8) return l.terms == 2 ? down_kernel<kI8, SHIFT, 2, FEW> : down_kernel<kI8, SHIFT, 3, FEW>;
    if (l.half) return down_kernel<kF16, SHIFT, 1, FEW>;
    return l.terms == 2 ? down_kernel<kBf16, SHIFT, 2, FEW> : down_kernel<kBf16, SHIFT, 3, FEW>;
}
Kernel down_of(const Layer& l, bool shift, bool few)
{
    if (few) return shift ? down_of<true, true>(l) : down_of<false, true>(l);
    return shift ? down_of<true, false>(l) : down_of<false, false>(l);
}

size_t product_smem(const Layer& l) { return size_t(kBefore) + size_t(l.rows) * l.top * 12; }

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
    const size_t bytes = product_smem(l);
    for (int shift = 0; shift < 2; shift++) {
        l.up_ctas[shift] = l.down_ctas[shift] = 1 << 30;
        for (int few = 0; few < 2; few++) {
            int up = 0, down = 0;
            int rc = resident(up_of(l, shift, few), bytes, num_sms, &up);
            if (!rc) rc = resident(down_of(l, shift, few), bytes, num_sms, &down);
            if (rc) return rc;
            l.up_ctas[shift] = std::min(l.up_ctas[shift], up);
            l.down_ctas[shift] = std::min(l.down_ctas[shift], down);
        }
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
    int rc = proj::launch(scores, dim3(unsigned(grid)), dim3(32 * score_warps(tok)), 0, 1, s, "experts' scores", l);
    const bool up = up_shifted(l), down = down_shifted(l), few = l.rows <= kWholeRows;
    if (!rc)
        rc = proj::launch(up_of(l, up, few), dim3(unsigned(l.up_ctas[up])), dim3(kThreads), product_smem(l), 1, s,
                          "experts' up products", l);
    if (!rc)
        rc = proj::launch(down_of(l, down, few), dim3(unsigned(l.down_ctas[down])), dim3(kThreads), product_smem(l), 1, s,
                          "experts' down products", l);
    if (!rc && !few)
        rc = proj::launch(combine_kernel, dim3(unsigned((l.d + 255) / 256), unsigned(l.rows)), dim3(256), 0, 1, s,
                          "experts' sum", l);
    return rc;
}

}  // namespace experts
}  // namespace dpdr
