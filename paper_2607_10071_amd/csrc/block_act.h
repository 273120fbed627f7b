// The activations of the encoder block's operators and their slopes.
#pragma once

#include "block/flashblock.h"
#include "hip_common.h"

namespace {

// On the hardware's exp2 and reciprocal (one unit in the last place each): an
// output of 40000 x 1024 gelus is 41 M of them, and with the library's erff, expf and
// IEEE division its product took 109 us where it takes 75 with these.
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSqrt2OverPi = 0.79788456080286536f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

__device__ __forceinline__ float sigmoid(float v)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// v, or the nearest of -m and m: factors of terms that are 0 there, so that an
// infinite v does not make them NaN
__device__ __forceinline__ float within(float v, float m)
{
    return __builtin_fminf(__builtin_fmaxf(v, -m), m);
}

// erfc(|v| / sqrt 2) = t P(t) exp(-v^2 / 2) with t = 1 / (1 + 0.43 |v| / sqrt 2): P is
// the polynomial of degree 7 with the least relative error over |v| <= 17
// (1.8e-7), found by weighted least squares in float64.  `e` gets the exponential.
// From erfc of |v| neither tail of gelu cancels.
__device__ __forceinline__ float erfc_half(float v, float &e)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(v), 0.30405591591021541f, 1.0f));
    e = __builtin_amdgcn_exp2f(v * v * (-0.5f * kLog2e));
    float q = 0.070911642f;
    q = __builtin_fmaf(q, t, -0.299038637f);
    q = __builtin_fmaf(q, t, 0.364747453f);
    q = __builtin_fmaf(q, t, -0.068830498f);
    q = __builtin_fmaf(q, t, 0.238214638f);
    q = __builtin_fmaf(q, t, 0.207467761f);
    q = __builtin_fmaf(q, t, 0.243988763f);
    q = __builtin_fmaf(q, t, 0.242538700f);
    return q * t * e;
}

__device__ __forceinline__ float act_value(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? v : (v == v ? 0.0f : v);
    case FLASHBLOCK_ACT_GELU: {
        float e;
        const float h = 0.5f * __builtin_fminf(__builtin_fabsf(v), 20.0f) * erfc_half(v, e);
        return v > 0.0f ? v - h : -h;   // (erfc is 0 at 20 already)
    }
    case FLASHBLOCK_ACT_GELU_TANH:   // (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        return v * sigmoid(2.0f * kSqrt2OverPi * v * __builtin_fmaf(0.044715f, v * v, 1.0f));
    case FLASHBLOCK_ACT_SILU: return v * sigmoid(v);
    default: return v;
    }
}

__device__ __forceinline__ float act_slope(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? 1.0f : 0.0f;
    case FLASHBLOCK_ACT_GELU: {
        float e;
        const float h = 0.5f * erfc_half(v, e);
        return __builtin_fmaf(within(v, 20.0f) * kInvSqrt2Pi, e, v > 0.0f ? 1.0f - h : h);
    }
    case FLASHBLOCK_ACT_GELU_TANH: {
        const float p = sigmoid(2.0f * kSqrt2OverPi * v * __builtin_fmaf(0.044715f, v * v, 1.0f));
        const float w = within(v, 20.0f);
        const float dz = 2.0f * kSqrt2OverPi * __builtin_fmaf(0.134145f, w * w, 1.0f);
        return __builtin_fmaf(w * p * (1.0f - p), dz, p);
    }
    case FLASHBLOCK_ACT_SILU: {
        const float p = sigmoid(v);
        return p * __builtin_fmaf(within(v, 100.0f), 1.0f - p, 1.0f);
    }
    default: return 1.0f;
    }
}

}  // namespace
