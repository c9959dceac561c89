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

__device__ __forceinline__ float load1(const char* p, int64_t i, int f32, int half)
{
    return f32 ? reinterpret_cast<const float*>(p)[i] : widen(reinterpret_cast<const uint16_t*>(p)[i], half);
}

__device__ __forceinline__ void store1(char* p, int64_t i, float v, int f32, int half)
{
    if (f32) reinterpret_cast<float*>(p)[i] = v;
    else reinterpret_cast<uint16_t*>(p)[i] = narrow(v, half);
}

// The logistic function.  Both divisions are by at least 1, so exp(-z) may
// overflow to infinity (z below -88) and the quotient is then 0.
__device__ __forceinline__ float logistic(float z) { return 1.0f / (1.0f + expf(-z)); }

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
        d = phi + z * kRoot2PiInv * expf(-0.5f * z * z);
        return;
    }
    case DPDR_ACT_GELU_TANH: {
        const float s = logistic(kRoot8Pi * (z + kCubic * z * z * z));
        v = z * s;
        d = s + v * (1.0f - s) * kRoot8Pi * (1.0f + 3.0f * kCubic * z * z);
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
