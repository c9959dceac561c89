// experts.cu -- a layer of experts for a few tokens: which experts each token
// takes, their gated products and the weighted sum of these.
//
//   l = x r^T;  the `top` largest of a token's l, ties to the lowest number
//   share = exp(l - max) over the sum of these (of the chosen, or of all)
//   h_e = share_e act(x wg_e^T) (x wu_e^T);  y = sum_e h_e wd_e^T
//
// Three kernels, each set up while the one before drains: scores_kernel forms l,
// chooses, and lays x out for the products; up_kernel streams the chosen experts' gate
// and up weights past the tokens that chose them (stream.cuh), a unit being 16 hidden
// features of an expert; down_kernel does the same with the down weights, a unit being
// 32 features of the result.  Up to 8 tokens have a column each there, and the sum runs
// through all experts; more have their results by expert, which combine_kernel adds up
// in the order of the shares.
//
// All pieces of all units are dealt out to the warps in equal contiguous shares, or
// where units are few each to a team of warps.  A unit that lies in several shares, or a
// team in several CTAs, is finished by the last of its warps (CTAs) to come, which adds
// up their sums in order: none waits for another, and no sum's order depends on timing,
// though where sums are cut depends on what all tokens chose.  (A CTA a unit, its sum
// over eight warps, with two barriers and a fence each: 8 rows of 64 experts of 2048 x
// 1024 125 us instead of 106.)
//
// Bound by the weights' bytes from some 50 MB of chosen experts on: 64 rows of 128
// experts of 2048 x 1024, 8 a token, 1.6 GB in 282 to 298 us (5.4 TB/s), 8 rows of 64
// such experts 0.5 GB in 100 to 106 (5.1).  One token of 8 experts of 4096 x 1792, 2 a
// token, 88 MB in 30 us, is a chain: scores and choice 4 us, lists 1, the up weights 11,
// joining a unit's parts 3, the down weights 5, joining those 3, the rest the ends and
// beginnings of kernels.  8-bit weights are
// widened in registers, which takes the issue slots to their limit: 16 rows of 64 such
// experts 0.36 GB in 90 us.
//
// The hidden values are not rounded to 16 bits: they are kept as three terms of bfloat16,
// which hold all of a float32 value, and for float16 weights as float32, of which the
// product takes 21 bits.  (With two terms, 16 bits, 64 rows of 128 experts take 276
// instead of 282 us, 16 rows of 64 in 8 bits 88.8 instead of 89.5, one token 30.4 and
// 30.4; what they lose shows where large products cancel.)
#include <algorithm>
#include <mutex>

#include "experts.cuh"

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
__global__ void __launch_bounds__(32 * score_warps(TOK), TOK == 8 ? 3 : 8)
    scores_kernel(const __grid_constant__ Layer l)
{
    constexpr int kScoreWarps = score_warps(TOK);
    __shared__ float part[kScoreWarps][TOK];
    constexpr int kThreads = 32 * kScoreWarps;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int e = blockIdx.x % l.total, t0 = blockIdx.x / l.total * TOK;
    const uint16_t* x = reinterpret_cast<const uint16_t*>(l.x);
    const uint16_t* r = reinterpret_cast<const uint16_t*>(l.router) + e * l.router_rs;
    if (VEC)   // while the kernel before drains
        for (int k = 64 * int(threadIdx.x); k < l.d; k += 64 * kThreads)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(r + k));
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

size_t product_smem(const Layer& l) { return size_t(kBefore) + size_t(l.rows) * l.top * 12; }

}  // namespace

// Every plan's calls may use as much shared memory as the largest plan's, so that it is
// set once a device.
int product_ctas(Layer& l, int num_sms)
{
    static std::mutex hold;
    static uint64_t set = 0;   // devices, of the first 64
    int device = 0, an_sm = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&an_sm, cudaDevAttrMaxSharedMemoryPerMultiprocessor, device);
    if (e == cudaSuccess) {
        std::lock_guard<std::mutex> one(hold);
        const uint64_t bit = device < 64 ? 1ull << device : 0;
        if (!(set & bit)) {
            Layer q = l;
            for (int w_int8 = 0; w_int8 < 2; w_int8++)
                for (int half = 0; half < 2; half++)
                    for (int shift = 0; shift < 2; shift++)
                        for (int few = 0; few < 2 && e == cudaSuccess; few++) {
                            q.w_int8 = w_int8, q.half = half;
                            for (Kernel k : {up_of(q, shift, few), down_of(q, shift, few)})
                                if (e == cudaSuccess)
                                    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(k),
                                                             cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                             kBefore + kMostRows * kMostTop * 12);
                        }
            if (e == cudaSuccess) set |= bit;
        }
    }
    if (e != cudaSuccess) return cuda_fail_c(e, "experts kernels");
    // Two CTAs an SM, as their registers allow, where it has shared memory for them: with
    // what the system takes of each and what the kernels hold besides.  That is up to 640
    // pairs of the plan's largest call; plans for more run every call on one an SM.
    const size_t each = product_smem(l) + 1024 + 512;
    l.ctas = (2 * each <= size_t(an_sm) ? 2 : 1) * num_sms;
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
        rc = proj::launch(up_of(l, up, few), dim3(unsigned(l.ctas)), dim3(kThreads), product_smem(l), 1, s,
                          "experts' up products", l);
    if (!rc)
        rc = proj::launch(down_of(l, down, few), dim3(unsigned(l.ctas)), dim3(kThreads), product_smem(l), 1, s,
                          "experts' down products", l);
    if (!rc && !few)
        rc = proj::launch(combine_kernel, dim3(unsigned((l.d + 255) / 256), unsigned(l.rows)), dim3(256), 0, 1, s,
                          "experts' sum", l);
    return rc;
}

}  // namespace experts
}  // namespace dpdr
