// Activations and their slopes in fp32, two values at a time (packed.cu, packed_linear.cu).
//
//   gelu(a) = a s, s = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (a + 0.044715 a^3)   (the tanh form: 2s = 1 + tanh u)
//   silu(a) = a s, s = 1 / (1 + exp(-a));   relu(a) = max(a, 0)
#pragma once

#include "inner_common.cuh"

namespace dipaco {

// The approximations are good to two units in the last place.
__device__ __forceinline__ float exp2_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float reciprocal_of(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// d = exp(-2u) and s = 1 / (1 + d) of two values; -2u log2(e) = a (c1 + c3 a^2).
__device__ __forceinline__ void gelu_share(f32x2 a, f32x2 square, f32x2 &d, f32x2 &s)
{
    constexpr float c1 = -2.0f * 0.7978845608028654f * 1.4426950408889634f, c3 = c1 * 0.044715f;
    const float2 e = values_of(mul2(a, fma2(square, pair_of(c3), pair_of(c1))));
    d = pair_of(exp2_of(e.x), exp2_of(e.y));
    const float2 t = values_of(add2(d, pair_of(1.0f)));
    s = pair_of(reciprocal_of(t.x), reciprocal_of(t.y));
}
__device__ __forceinline__ f32x2 gelu(f32x2 a)
{
    f32x2 d, s;
    gelu_share(a, mul2(a, a), d, s);
    return mul2(a, s);
}

// s + a s (1 - s) 2u' = s (1 + a d s 2u') with d = exp(-2u): no cancellation where s is near 1.  a is held
// within +-10.03, NaN kept: there the slope is 1, or 0 (d is still finite and s flushed to zero).
__device__ __forceinline__ float held(float a)
{
    asm("min.NaN.f32 %0, %0, 0f41208000;\n\tmax.NaN.f32 %0, %0, 0fC1208000;" : "+f"(a));
    return a;
}
__device__ __forceinline__ f32x2 gelu_slope(f32x2 value)
{
    constexpr float k1 = 2.0f * 0.7978845608028654f, k3 = 3.0f * 0.044715f * k1;
    const float2 v = values_of(value);
    const f32x2 a = pair_of(held(v.x), held(v.y)), square = mul2(a, a);
    f32x2 d, s;
    gelu_share(a, square, d, s);
    return mul2(s, fma2(mul2(d, s), mul2(a, fma2(square, pair_of(k3), pair_of(k1))), pair_of(1.0f)));
}

// s of silu, and d = exp(-a).
__device__ __forceinline__ void silu_share(f32x2 a, f32x2 &d, f32x2 &s)
{
    const float2 e = values_of(mul2(a, pair_of(-1.4426950408889634f)));
    d = pair_of(exp2_of(e.x), exp2_of(e.y));
    const float2 t = values_of(add2(d, pair_of(1.0f)));
    s = pair_of(reciprocal_of(t.x), reciprocal_of(t.y));
}
__device__ __forceinline__ f32x2 silu(f32x2 a)
{
    f32x2 d, s;
    silu_share(a, d, s);
    return mul2(a, s);
}
// s + a s (1 - s) = s (1 + a d s).  a is held within +-80, NaN kept: there the slope is 1, or 0 within 1e-32.
__device__ __forceinline__ f32x2 silu_slope(f32x2 value)
{
    float2 v = values_of(value);
    asm("min.NaN.f32 %0, %0, 0f42A00000;\n\tmax.NaN.f32 %0, %0, 0fC2A00000;" : "+f"(v.x));
    asm("min.NaN.f32 %0, %0, 0f42A00000;\n\tmax.NaN.f32 %0, %0, 0fC2A00000;" : "+f"(v.y));
    const f32x2 a = pair_of(v.x, v.y);
    f32x2 d, s;
    silu_share(a, d, s);
    return mul2(s, fma2(mul2(d, s), a, pair_of(1.0f)));
}

__device__ __forceinline__ float relu1(float a)  // NaN stays
{
    asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(a));
    return a;
}
__device__ __forceinline__ float relu_slope1(float a) { return a > 0.0f ? 1.0f : a <= 0.0f ? 0.0f : a; }

template <int ACTIVATION> __device__ __forceinline__ f32x2 activate(f32x2 a)
{
    if constexpr (ACTIVATION == DIPACO_ACTIVATION_GELU) {
        return gelu(a);
    } else if constexpr (ACTIVATION == DIPACO_ACTIVATION_SILU) {
        return silu(a);
    } else if constexpr (ACTIVATION == DIPACO_ACTIVATION_RELU) {
        const float2 v = values_of(a);
        return pair_of(relu1(v.x), relu1(v.y));
    } else {
        return a;
    }
}
template <int ACTIVATION> __device__ __forceinline__ f32x2 slope(f32x2 a)
{
    if constexpr (ACTIVATION == DIPACO_ACTIVATION_GELU) {
        return gelu_slope(a);
    } else if constexpr (ACTIVATION == DIPACO_ACTIVATION_SILU) {
        return silu_slope(a);
    } else if constexpr (ACTIVATION == DIPACO_ACTIVATION_RELU) {
        const float2 v = values_of(a);
        return pair_of(relu_slope1(v.x), relu_slope1(v.y));
    } else {
        return pair_of(1.0f);
    }
}

// The same with one reciprocal for two values, 1/x = y / (x y): where powers stay under 2^63, and no value is NaN.
template <int ACTIVATION> __device__ __forceinline__ f32x2 activate_in_pairs(f32x2 a)
{
    if constexpr (ACTIVATION == DIPACO_ACTIVATION_GELU || ACTIVATION == DIPACO_ACTIVATION_SILU) {
        constexpr float c1 = -2.0f * 0.7978845608028654f * 1.4426950408889634f, c3 = c1 * 0.044715f;
        const float2 e = values_of(ACTIVATION == DIPACO_ACTIVATION_GELU ? mul2(a, fma2(mul2(a, a), pair_of(c3), pair_of(c1)))
                                                                        : mul2(a, pair_of(-1.4426950408889634f)));
        const float2 t = values_of(add2(pair_of(exp2_of(e.x), exp2_of(e.y)), pair_of(1.0f)));
        return mul2(a, mul2(pair_of(t.y, t.x), pair_of(reciprocal_of(t.x * t.y))));
    } else {
        return activate<ACTIVATION>(a);
    }
}
// Up to which magnitude: -2u log2(e) is 54 at -7.2, -a log2(e) 58 at -40.
template <int ACTIVATION> __device__ __forceinline__ constexpr float pairs_up_to()
{
    return ACTIVATION == DIPACO_ACTIVATION_GELU ? 7.2f : ACTIVATION == DIPACO_ACTIVATION_SILU ? 40.0f : 1e38f;
}

// Where the largest value of a set is at least this, its activation is the largest magnitude among the set's
// activations: they grow there, and below zero none is larger than the activation of this value (0.170 against 0.185,
// 0.279 against 0.387).
template <int ACTIVATION> __device__ __forceinline__ constexpr float grows_from()
{
    return ACTIVATION == DIPACO_ACTIVATION_GELU ? 0.3f : ACTIVATION == DIPACO_ACTIVATION_SILU ? 0.6f : 0.0f;
}

} // namespace dipaco
