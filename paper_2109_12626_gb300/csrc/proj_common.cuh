// proj_common.cuh -- the projections' arithmetic: 16-bit operands widened and
// rounded, activations with their slopes, and what becomes of a finished sum.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "proj.h"

namespace dpdr {
namespace proj {

__device__ __forceinline__ float widen(uint16_t v, int half)
{
    return half ? __half2float(__ushort_as_half(v)) : __bfloat162float(__ushort_as_bfloat16(v));
}

__device__ __forceinline__ uint16_t narrow(float v, int half)
{
    return half ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v));
}

// two values rounded, the first in the lower half
__device__ __forceinline__ uint32_t narrow2(float a, float b, int half)
{
    if (half) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ float load1(const char* p, int64_t i, int f32, int half)
{
    return f32 ? reinterpret_cast<const float*>(p)[i] : widen(reinterpret_cast<const uint16_t*>(p)[i], half);
}

__device__ __forceinline__ void store1(char* p, int64_t i, float v, int f32, int half)
{
    if (f32) reinterpret_cast<float*>(p)[i] = v;
    else reinterpret_cast<uint16_t*>(p)[i] = narrow(v, half);
}

// The logistic function, by CUDA's fast exponential and division, whose errors
// (a few units of 2^-23, and 2^-24 of the exponent's size) are far below a
// 16-bit result's rounding and of the order of a float32 sum's; the exact ones
// made the element-wise kernels wait for arithmetic.  The divisor is at least
// 1; where exp(-z) overflows (z below -88) the quotient is 0.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

constexpr float kRootHalf = 0.70710678118654752f;   // sqrt(1/2)
constexpr float kRoot8Pi = 1.59576912160573072f;    // 2 sqrt(2/pi)
constexpr float kRoot2PiInv = 0.39894228040143268f; // 1/sqrt(2 pi)
constexpr float kCubic = 0.044715f;

// (1 + tanh(a)) / 2 is the logistic function of 2 a, so the tanh form of gelu
// is z logistic(2 sqrt(2/pi) (z + 0.044715 z^3)).
template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    switch (ACT) {
    case DPDR_ACT_RELU: return z < 0.0f ? 0.0f : z;   // NaN stays NaN
    case DPDR_ACT_GELU: return 0.5f * z * erfcf(-z * kRootHalf);
    case DPDR_ACT_GELU_TANH: return z * logistic(kRoot8Pi * (z + kCubic * z * z * z));
    case DPDR_ACT_SILU: return z * logistic(z);
    case DPDR_ACT_SIGMOID: return logistic(z);
    default: return z;
    }
}

// act(z) and act'(z)
template <int ACT>
__device__ __forceinline__ void act_both(float z, float& v, float& d)
{
    switch (ACT) {
    case DPDR_ACT_RELU:
        v = z < 0.0f ? 0.0f : z;
        d = z > 0.0f ? 1.0f : 0.0f;
        return;
    case DPDR_ACT_GELU: {
        const float phi = 0.5f * erfcf(-z * kRootHalf);
        v = z * phi;
        d = phi + z * kRoot2PiInv * __expf(-0.5f * z * z);
        return;
    }
    case DPDR_ACT_GELU_TANH: {
        const float s = logistic(kRoot8Pi * (z + kCubic * z * z * z));
        v = z * s;
        // s is 0 or 1 long before z z is infinite, which would make 0 times it NaN
        const float a = fminf(fabsf(z), 1e9f);
        d = s + v * (1.0f - s) * kRoot8Pi * (1.0f + 3.0f * kCubic * a * a);
        return;
    }
    case DPDR_ACT_SILU: {
        const float s = logistic(z);
        v = z * s;
        d = s + v * (1.0f - s);
        return;
    }
    case DPDR_ACT_SIGMOID:
        v = logistic(z);
        d = v * (1.0f - v);
        return;
    default:
        v = z;
        d = 1.0f;
    }
}

// One output: z (the bias in it), or the pair g, u -> what Finish says.
template <bool PAIR, int FINISH, int ACT>
__device__ __forceinline__ void finish1(float g, float u, float other, float& out, float& out2)
{
    if (FINISH == kValue) {
        const float v = act_value<ACT>(g);
        out = PAIR ? v * u : v + other;
    } else {
        float v, d;
        act_both<ACT>(g, v, d);
        out = PAIR ? other * u * d : other * d;
        out2 = other * v;
    }
}

// ------------------------------------------------ results by fours

__device__ __forceinline__ void widen4(const uint4& x, int f32, int half, float (&v)[4])
{
    if (f32) {
        v[0] = __uint_as_float(x.x), v[1] = __uint_as_float(x.y);
        v[2] = __uint_as_float(x.z), v[3] = __uint_as_float(x.w);
    } else if (half) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&x.x)),
                     b = __half22float2(*reinterpret_cast<const __half2*>(&x.y));
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    } else {   // a bfloat16 is the upper half of a float
        v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
        v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
    }
}

__device__ __forceinline__ void load4(const char* p, int64_t i, int f32, int half, float (&v)[4])
{
    uint4 x = make_uint4(0, 0, 0, 0);
    if (f32) {
        x = *reinterpret_cast<const uint4*>(p + 4 * i);
    } else {
        const uint2 y = *reinterpret_cast<const uint2*>(p + 2 * i);
        x.x = y.x, x.y = y.y;
    }
    widen4(x, f32, half, v);
}

__device__ __forceinline__ void store4(char* p, int64_t i, int f32, int half, const float (&v)[4])
{
    if (f32)
        *reinterpret_cast<float4*>(p + 4 * i) = make_float4(v[0], v[1], v[2], v[3]);
    else
        *reinterpret_cast<uint2*>(p + 2 * i) = make_uint2(narrow2(v[0], v[1], half), narrow2(v[2], v[3], half));
}

// what else a result element needs
__device__ __forceinline__ float other1(const Epilogue& e, int64_t m, int64_t n)
{
    return e.other ? load1(e.other, m * e.other_rs + n * e.other_cs, e.other_f32, e.half) : 0.0f;
}

// One result element from its sum (or pair of sums); its value before rounding
template <bool PAIR, int FINISH, int ACT>
__device__ __forceinline__ float put1(const Epilogue& e, char* out, int64_t out_rs, int64_t m, int64_t n, float z,
                                     float u, float bias, float o)
{
    z += bias;
    if (e.pre) {
        e.pre[m * e.pre_rs + n] = z;
        if (PAIR) e.pre[m * e.pre_rs + e.pre_up + n] = u;
    }
    float v = 0.0f, w = 0.0f;
    finish1<PAIR, FINISH, ACT>(z, u, o, v, w);
    store1(out, m * out_rs + n, v, e.out_f32, e.half);
    if (PAIR && FINISH == kSlope) store1(e.out2, m * e.out2_rs + n, w, e.out_f32, e.half);
    return v;
}

// Four of them side by side, their values in v
template <bool PAIR, int FINISH, int ACT>
__device__ __forceinline__ void put4(const Epilogue& e, char* out, int64_t out_rs, int64_t m, int64_t n, float (&z)[4],
                                     const float (&u)[4], const float (&bias)[4], const float (&o)[4], float (&v)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i++) z[i] += bias[i];
    if (e.pre) {
        *reinterpret_cast<float4*>(e.pre + m * e.pre_rs + n) = make_float4(z[0], z[1], z[2], z[3]);
        if (PAIR)
            *reinterpret_cast<float4*>(e.pre + m * e.pre_rs + e.pre_up + n) = make_float4(u[0], u[1], u[2], u[3]);
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        w[i] = 0.0f;
        finish1<PAIR, FINISH, ACT>(z[i], u[i], o[i], v[i], w[i]);
    }
    store4(out, m * out_rs + n, e.out_f32, e.half, v);
    if (PAIR && FINISH == kSlope) store4(e.out2, m * e.out2_rs + n, e.out_f32, e.half, w);
}

// f<ACT>() for the activation that a call names.  Each is a kernel of its
// own: with the choice made per element, one kernel's row loop held the code
// of all of them, and fetching it took 38 us a 256 x 256 tile.
#define DPDR_FOR_ACT(act, CALL)                              \
    switch (act) {                                           \
    case DPDR_ACT_RELU: CALL(DPDR_ACT_RELU); break;          \
    case DPDR_ACT_GELU: CALL(DPDR_ACT_GELU); break;          \
    case DPDR_ACT_GELU_TANH: CALL(DPDR_ACT_GELU_TANH); break;\
    case DPDR_ACT_SILU: CALL(DPDR_ACT_SILU); break;          \
    case DPDR_ACT_SIGMOID: CALL(DPDR_ACT_SIGMOID); break;    \
    default: CALL(DPDR_ACT_NONE);                            \
    }

}  // namespace proj
}  // namespace dpdr
