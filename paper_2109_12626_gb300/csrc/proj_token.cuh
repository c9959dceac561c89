// proj_token.cuh -- the projections' forward products for one row: the
// weights stream past once, each row of them to one warp or a few.
//
// One row's product is a sum of K per feature on the FP32 units, bound by the
// weights' bytes.  A group of `share` warps takes two features (of a pair one,
// and its two weights): each lane loads 16 bytes of both rows four times over
// before it uses the first, so that some 100 KB an SM are under way; x comes
// from L1.  Nothing is set up or joined between CTAs, which is what
// row_kernel's tensor memory, barriers and clusters cost: 1024 x 1024 weights
// in 1.9 against 3.7 us, 512 x 8192 in 3.2 against 8.3, 4096 x 4096 in 6.8
// against 8.8 (5.0 TB/s), 8192 x 8192 in 22.9 against 24.4 (5.9 TB/s); back to
// back, weights not in L2.  From two rows on the additions and the reads of x
// take longer than row_kernel's set-up (four rows, 4096 x 4096: 15.5 against
// 9.5).  Rows that are not 16-byte aligned are read element by element (4096 x
// 4099 in 18.5 us), still less than a copy of them first.
#pragma once

#include "proj_common.cuh"
#include "proj_launch.cuh"

namespace dpdr {
namespace proj {

constexpr int kTokenWarps = 8;

struct TokenArgs {
    Operand x, w[2];               // summed index contiguous
    int64_t K, N;
    int share;                     // warps of a group: 1, 2, 4 or 8
    int aligned;                   // 16-byte loads
    Epilogue e;
};

namespace {

constexpr int kTokenDeep = 4;      // 16-byte loads of a row before the first is used

__device__ __forceinline__ void widen8(const uint4& v, int half, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (half) {
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = p.x, f[2 * i + 1] = p.y;
        } else {   // a bfloat16 is the upper half of a float
            f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

// eight products of either weight row with x
__device__ __forceinline__ void sum8(const uint4& a, const uint4& b, const uint4& x, int half, float (&acc)[2])
{
    float f[8], g[8], v[8];
    widen8(a, half, f);
    widen8(b, half, g);
    widen8(x, half, v);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        acc[0] += f[i] * v[i];
        acc[1] += g[i] * v[i];
    }
}

template <bool PAIR, int ACT>
__global__ void __launch_bounds__(32 * kTokenWarps) token_kernel(const TokenArgs t)
{
    __shared__ float parts[kTokenWarps][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = warp / t.share, mine = warp % t.share;
    const int64_t first = (int64_t(blockIdx.x) * (kTokenWarps / t.share) + group) * (PAIR ? 1 : 2);
    // the two weight rows; a last odd feature is taken twice
    const int64_t second = PAIR || first + 1 >= t.N ? first : first + 1;
    const Operand o1 = t.w[PAIR ? 1 : 0];
    const uint16_t* w0 = reinterpret_cast<const uint16_t*>(t.w[0].p) + first * t.w[0].is;
    const uint16_t* w1 = reinterpret_cast<const uint16_t*>(o1.p) + second * o1.is;
    // The first loads' lines are asked into L2 while the kernel before drains
    // (4096 x 4096 in 8.1 us without); whatever it still writes there is seen,
    // since L2 is where all SMs meet.
    if (t.aligned && first < t.N)
        for (int64_t at = 64 * (mine * 32 + lane); at < t.K && at < 64 * 32 * t.share; at += 64 * 32 * t.share) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + at));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(w1 + at));
        }
    wait_previous();
    allow_next();
    float acc[2] = {0.0f, 0.0f};
    if (first < t.N) {
        const uint16_t* x = reinterpret_cast<const uint16_t*>(t.x.p);
        const int half = t.e.half;
        const int64_t step = 32 * t.share;
        int64_t done = 0;   // elements summed by the aligned loops
        if (t.aligned) {
            const int64_t units = t.K / 8;
            done = units * 8;
            const uint4 *p0 = reinterpret_cast<const uint4*>(w0), *p1 = reinterpret_cast<const uint4*>(w1),
                        *px = reinterpret_cast<const uint4*>(x);
            uint4 a[kTokenDeep], b[kTokenDeep], v[kTokenDeep];
            int64_t u = mine * 32 + lane;
            for (; u + (kTokenDeep - 1) * step < units; u += kTokenDeep * step) {
#pragma unroll
                for (int d = 0; d < kTokenDeep; d++) a[d] = __ldcs(p0 + u + d * step), b[d] = __ldcs(p1 + u + d * step);
#pragma unroll
                for (int d = 0; d < kTokenDeep; d++) v[d] = px[u + d * step];
#pragma unroll
                for (int d = 0; d < kTokenDeep; d++) sum8(a[d], b[d], v[d], half, acc);
            }
#pragma unroll
            for (int d = 0; d < kTokenDeep - 1; d++)
                if (u + d * step < units) {
                    a[d] = __ldcs(p0 + u + d * step);
                    b[d] = __ldcs(p1 + u + d * step);
                    v[d] = px[u + d * step];
                }
#pragma unroll
            for (int d = 0; d < kTokenDeep - 1; d++)
                if (u + d * step < units) sum8(a[d], b[d], v[d], half, acc);
        }
        constexpr int kDeep = 16;
        for (int64_t k0 = done + mine * 32 + lane; k0 < t.K; k0 += kDeep * step) {
            uint16_t a[kDeep], b[kDeep], v[kDeep];
#pragma unroll
            for (int d = 0; d < kDeep; d++) {
                const int64_t k = k0 + d * step;
                a[d] = b[d] = v[d] = 0;
                if (k < t.K) a[d] = w0[k], b[d] = w1[k], v[d] = x[k];
            }
#pragma unroll
            for (int d = 0; d < kDeep; d++) {
                if (k0 + d * step >= t.K) break;
                acc[0] += widen(a[d], half) * widen(v[d], half);
                acc[1] += widen(b[d], half) * widen(v[d], half);
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        acc[0] += __shfl_xor_sync(0xFFFFFFFFu, acc[0], o);
        acc[1] += __shfl_xor_sync(0xFFFFFFFFu, acc[1], o);
    }
    if (t.share > 1) {   // the group's warps in their order
        if (lane == 0) parts[warp][0] = acc[0], parts[warp][1] = acc[1];
        __syncthreads();
        for (int s = 1; s < t.share && mine == 0; s++) {
            acc[0] += parts[warp + s][0];
            acc[1] += parts[warp + s][1];
        }
    }
    if (mine != 0) return;
    const int64_t n = first + lane;   // lane i finishes feature i of the group
    if (lane >= (PAIR ? 1 : 2) || n >= t.N) return;
    const Epilogue& e = t.e;
    const float bias = e.bias ? load1(static_cast<const char*>(e.bias), n, 0, e.half) : 0.0f;
    put1<PAIR, kValue, ACT>(e, e.out, e.out_rs, 0, n, PAIR || lane == 0 ? acc[0] : acc[1], acc[1], bias, other1(e, 0, n));
}

}  // namespace

using TokenKernel = void (*)(TokenArgs);

template <bool PAIR>
TokenKernel token_kernel_of(int act)
{
    TokenKernel k = nullptr;
#define DPDR_CALL(A) k = token_kernel<PAIR, A>
    DPDR_FOR_ACT(act, DPDR_CALL)
#undef DPDR_CALL
    return k;
}

}  // namespace proj
}  // namespace dpdr
