// Activations of the gated block and their derivatives, in fp32.
#pragma once
#include "gvq_internal.h"

namespace gvq {

// e^x and 1 / x by the hardware's units (two units of the last place each), subnormal results 0: without that, e^x takes three
// more instructions, and instructions are what bounds the epilogue of a short contraction.  The argument's rounding moves e^x by
// 2^-23 |x| of itself.
__device__ __forceinline__ float exp_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
    return r;
}
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + e^-x): 0 where e^-x overflows, off by at most a quarter of what e^-x is of itself.
__device__ __forceinline__ float logistic(float x) { return reciprocal(1.0f + exp_approx(-x)); }
constexpr float kTanhScale = 1.5957691216057308f, kTanhCubic = 0.044715f;      // 2 sqrt(2 / pi)

template <int ACT>
__device__ __forceinline__ float activation_of(float x)
{
    if (ACT == GVQ_SILU) return x * logistic(x);
    if (ACT == GVQ_GELU) return 0.5f * x * erfcf(-0.70710678118654752f * x);      // (erfc keeps the small values of negative x)
    // 0.5 (1 + tanh z) is the logistic function of 2 z
    if (ACT == GVQ_GELU_TANH) return x * logistic(kTanhScale * (x + kTanhCubic * x * x * x));
    if (ACT == GVQ_RELU) return x <= 0.0f ? 0.0f : x;      // (a NaN stays one)
    return logistic(x);
}
__device__ __forceinline__ float activation(int act, float x)
{
    switch (act) {
    case GVQ_SILU: return activation_of<GVQ_SILU>(x);
    case GVQ_GELU: return activation_of<GVQ_GELU>(x);
    case GVQ_GELU_TANH: return activation_of<GVQ_GELU_TANH>(x);
    case GVQ_RELU: return activation_of<GVQ_RELU>(x);
    default: return activation_of<GVQ_SIGMOID>(x);
    }
}
// v = act(v) * u
template <int ACT, int N>
__device__ __forceinline__ void activate_as(float (&v)[N], const float (&u)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activation_of<ACT>(v[i]) * u[i];
}
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N], const float (&u)[N])
{
    switch (act) {
    case GVQ_SILU: activate_as<GVQ_SILU>(v, u); break;
    case GVQ_GELU: activate_as<GVQ_GELU>(v, u); break;
    case GVQ_GELU_TANH: activate_as<GVQ_GELU_TANH>(v, u); break;
    case GVQ_RELU: activate_as<GVQ_RELU>(v, u); break;
    default: activate_as<GVQ_SIGMOID>(v, u);
    }
}
// The activation and its derivative.
template <int ACT>
__device__ __forceinline__ float2 activation_and_slope(float x)
{
    if (ACT == GVQ_GELU) {
        const float cdf = 0.5f * erfcf(-0.70710678118654752f * x);
        return make_float2(x * cdf, cdf + x * 0.3989422804014327f * expf(-0.5f * x * x));
    }
    if (ACT == GVQ_RELU) return make_float2(x <= 0.0f ? 0.0f : x, x > 0.0f ? 1.0f : 0.0f);
    if (ACT == GVQ_GELU_TANH) {
        const float s = logistic(kTanhScale * (x + kTanhCubic * x * x * x));
        const float t = s * (1.0f - s);      // (0 where the square below may overflow)
        return make_float2(x * s, s + (t > 0.0f ? x * t * kTanhScale * (1.0f + 3.0f * kTanhCubic * x * x) : t));
    }
    const float s = logistic(x);
    if (ACT == GVQ_SIGMOID) return make_float2(s, s * (1.0f - s));
    return make_float2(x * s, s + x * s * (1.0f - s));
}

}  // namespace gvq
