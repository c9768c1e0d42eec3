// Activations of the gated block and their derivatives, in fp32.
#pragma once
#include "gvq_internal.h"

namespace gvq {

// e^x and 1 / x by the hardware's units (two units of the last place each), subnormal results 0: without that, e^x takes three
// more instructions, and instructions are what bounds the epilogue of a short contraction.  The argument's rounding moves e^x by
// 2^-23 |x| of itself.
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float exp_approx(float x) { return exp2_approx(x * kLog2e); }
__device__ __forceinline__ float reciprocal(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + e^-x): 0 where e^-x overflows, off by at most a quarter of what e^-x is of itself.
__device__ __forceinline__ float logistic(float x) { return reciprocal(1.0f + exp_approx(-x)); }
constexpr float kTanhScale = 1.5957691216057308f, kTanhCubic = 0.044715f;      // 2 sqrt(2 / pi)
// The normal distribution's cdf is erfc(-x / sqrt 2) / 2, and its density has the exponential that erfc has as a factor: with
// z = |x| / sqrt 2 and t = 1 / (1 + z / 2), erfc z = t e^(p(t) - z^2) by the rational fit of Press, Flannery, Teukolsky and Vetterling's
// "Numerical Recipes" (off by 1.2e-7 of itself at most; with fp32's exponents, whose roundings grow with z^2, 7 * 10^-7 down to x = -3 and
// 10^-5 down to -12.9, where a 16-bit result's half step is 5 * 10^-4 at least; below that the cdf is subnormal in fp32, and 0 here).
// A third of the instructions of erfcf and expf: slopes of 8192 x 8192 in 112 us, not 176.
struct Normal { float p, z2; };      // exponents of 2: of t e^p, and of the density
__device__ __forceinline__ float normal_terms(float x, Normal &n)
{
    const float t = reciprocal(fmaf(0.35355339059327376f, fabsf(x), 1.0f));
    constexpr float c[10] = {-1.26551223f * kLog2e, 1.00002368f * kLog2e,  0.37409196f * kLog2e, 0.09678418f * kLog2e,  -0.18628806f * kLog2e,
                             0.27886807f * kLog2e,  -1.13520398f * kLog2e, 1.48851587f * kLog2e, -0.82215223f * kLog2e, 0.17087277f * kLog2e};
    float p = c[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = fmaf(p, t, c[i]);
    n.p = p;
    n.z2 = x * x * (-0.5f * kLog2e);
    return t;
}
// From e^(p - z^2) t / 2, which keeps the small values of negative x.
__device__ __forceinline__ float normal_cdf(float x, float half_erfc) { return x < 0.0f ? half_erfc : 1.0f - half_erfc; }

template <int ACT>
__device__ __forceinline__ float activation_of(float x)
{
    if (ACT == GVQ_SILU) return x * logistic(x);
    if (ACT == GVQ_GELU) {
        Normal n;
        const float t = normal_terms(x, n);
        return x * normal_cdf(x, 0.5f * t * exp2_approx(n.p + n.z2));
    }
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
        Normal n;
        const float t = normal_terms(x, n), e = exp2_approx(n.z2), cdf = normal_cdf(x, 0.5f * t * exp2_approx(n.p) * e);
        return make_float2(x * cdf, cdf + x * 0.3989422804014327f * e);
    }
    if (ACT == GVQ_RELU) return make_float2(x <= 0.0f ? 0.0f : x, x > 0.0f ? 1.0f : 0.0f);
    if (ACT == GVQ_GELU_TANH) {
        const float s = logistic(kTanhScale * (x + kTanhCubic * x * x * x));
        const float t = s * (1.0f - s);      // (0 where the square below may overflow)
        return make_float2(x * s, s + (t > 0.0f ? x * t * kTanhScale * (1.0f + 3.0f * kTanhCubic * x * x) : t));
    }
    if (ACT == GVQ_SIGMOID) {      // with t = e^-|x|, t / (1 + t)^2: s (1 - s) has no digit left at 16
        const float t = exp_approx(-fabsf(x)), s = reciprocal(1.0f + t);
        return make_float2(x < 0.0f ? t * s : s, t * s * s);
    }
    const float s = logistic(x);
    return make_float2(x * s, s + x * s * (1.0f - s));
}

}  // namespace gvq
