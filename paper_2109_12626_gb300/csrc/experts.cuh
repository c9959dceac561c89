// experts.cuh -- what the two product kernels of a layer of experts share: the lists of
// which tokens chose which experts, and how a warp goes through its pieces of weights.
#pragma once

#include "experts.h"
#include "stream.cuh"

namespace dpdr {
namespace experts {

using namespace stream;

namespace {

// ------------------------------------------------------------------ choice

// What a CTA knows of the choice, in shared memory.  A pair is a token's number
// times `top` plus the place of one of its experts.
struct Choice {
    float* share;         // of a pair
    uint32_t* entry;      // an expert with up to `most` of its pairs: number among
                          // the local ones, how many pairs, the first of them in `order`,
                          // which of the first 8 tokens chose it
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
    static __device__ __forceinline__ uint32_t packed(int e, int n, int from, uint32_t tokens)
    {
        static_assert(kMostExperts <= 1 << 9 && kMostRows * kMostTop <= 1 << 10 && kWholeRows <= 8, "9, 5, 10 and 8 bits");
        return uint32_t(e) | uint32_t(n - 1) << 9 | uint32_t(from) << 14 | tokens << 24;
    }
    __device__ __forceinline__ int number(int i) const { return entry[i] & 511u; }
    __device__ __forceinline__ int count(int i) const { return (entry[i] >> 9 & 31u) + 1; }
    __device__ __forceinline__ int from(int i) const { return entry[i] >> 14 & 1023u; }
    __device__ __forceinline__ uint32_t chose(int i) const { return entry[i] >> 24; }
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
            if (here) c.entry[at] = Choice::packed(e, 1, at, 1u), c.order[at] = int16_t(lane);
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
        for (int k = 0; k < n[i]; k += most) c.entry[i0++] = Choice::packed(e0 + i, min(most, n[i] - k), p0 + k, uint32_t(mask[e0 + i]));
        p0 += n[i];
    }
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += kThreads) {
        const int e = c.expert[p] - l.first, t = p / l.top;
        if (e >= 0 && e < l.local) c.order[from[e] + __popcll(mask[e] & ((1ull << t) - 1))] = int16_t(p);
    }
    __syncthreads();   // `room` is free again
}

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
                        for (int j = 0; j < 4; j++)
                            if (!S::kZeros || st.counts[j & 1]) sum[k][n][j] += part[k][n][j] * by[2 * k + j / 2];
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
        // Teams of two and three warps are 3 to 2, which is less than joining shares costs
        // while a piece's columns are few: 16 rows of 8 experts of 4096 x 1792 with teams
        // of two or more, and of four or more, 81.0 and 83.6 us, 64 rows 128.9 and 118.7.
        if ((NT > 2 ? 4 : 2) * job.units <= int(gridDim.x) * kWarps) teams<ASK>();
        else shares<ASK>();
    }
};

// bytes of shared memory in front of the choice: rings, then tiles
constexpr int kRings = kWarps * kRing, kBefore = kRings + kJoin * 4;

// Bytes of a row of weights that a stage holds.  Where widening binds (8-bit weights,
// tf32) 128 bytes save turns of the loop, if the ring holds two such stages; else more
// and smaller ones keep more under way.  With 64 and 128, on one GPU: 16 rows of 64
// experts in 8 bits 91 and 89 us, 8 rows in 16 bits 100.7 and 102.3.
constexpr int piece_of(int wt, int xt, int nt, bool shift, int terms)
{
    const int stage = kRows * (128 + 16 * shift) + terms * nt * 8 * (128 / size_of(wt)) * size_of(xt);
    return (wt == kI8 || xt == kF32) && 2 * stage <= kRing ? 128 : 64;
}

// FEW: up to 8 tokens.  These kernels hold the code for one eight of columns alone,
// and leave registers (of 288 threads, in the bounds) for the next call's
// scores_kernel to be set up beside them.
constexpr int bound_of(bool few) { return few ? kThreads + 32 : kThreads; }

}  // namespace

using Kernel = void (*)(Layer);
Kernel up_of(const Layer& l, bool shift, bool few);     // experts_up.cu
Kernel down_of(const Layer& l, bool shift, bool few);   // experts_down.cu

}  // namespace experts
}  // namespace dpdr
