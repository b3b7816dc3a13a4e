// Activations of the gated feed-forward block and the linear layer and their slopes, in registers.
#pragma once
#include <cuda_runtime.h>

#include <type_traits>

#include "atb.h"
#include "f32x2.cuh"

namespace glu {

// 2^x; results below the normal range become 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// act(g) and act'(g) of two values.  The kernels that call this are short of issue slots where K is shallow, hence the two-wide
// arithmetic and the fast instructions for exp and 1 / x: 1 to 2 ulp, and the rounding of the exponent's argument, whose size times
// 2^-24 the result is off by.  Far below bf16's rounding, to which most results go; where the linear layer's are FP32, act(z) is off by at
// most this much of itself, as measured (silu, gelu, tanh-gelu): 3e-7, 6e-7, 3e-7 from z = -1 on, 4e-7, 1.5e-6, 2.3e-6 from -5,
// 6e-7, 5e-6, 1.3e-5 from -10, and act'(z) by 1e-6, 3e-7, 2e-6 of 1.  Phi(-x) = exp(-x^2 / 2) times a polynomial of degree 8 in
// t = 1 / (1 + 0.3 x) without a constant term, x >= 0, and
// Phi(x) = 1 - Phi(-x): the exponential is the one that the slope needs.  The form is that of Abramowitz and Stegun 7.1.26, whose
// five terms are off by 1.5e-7 of 1, and so by more than bf16's half unit of g Phi(g) below g = -4.4; these eight coefficients
// are a least-squares fit, reweighted to even out the relative error on 0 <= x <= 14, which is 1.5e-7 of Phi(-x) (4.4e-7 in FP32).
template <int ACT>
__device__ __forceinline__ void act_value_slope(float2 g, float2& a, float2& slope) {
    using namespace f32x2;
    const float2 one = both(1.f);
    if constexpr (ACT == ATB_ACT_SILU) {
        const float2 x = mul2(g, both(-kLog2e));
        const float2 d = add2(make_float2(exp2_fast(x.x), exp2_fast(x.y)), one);
        const float2 s = make_float2(rcp_fast(d.x), rcp_fast(d.y));
        a = mul2(g, s);
        slope = fma2(a, fma2(s, both(-1.f), one), s);
    } else if constexpr (ACT == ATB_ACT_GELU) {
        const float2 d = fma2(make_float2(fabsf(g.x), fabsf(g.y)), both(0.3f), one);
        const float2 t = make_float2(rcp_fast(d.x), rcp_fast(d.y));
        const float2 x = mul2(mul2(g, both(-0.5f * kLog2e)), g);
        const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
        constexpr float c[] = {0.206353191f, -0.0536833441f, 0.128561463f, 0.0999135428f, 0.120753948f, 0.119629299f};
        float2 poly = fma2(t, both(0.0356747341f), both(-0.157202907f));
#pragma unroll
        for (const float k : c) poly = fma2(t, poly, both(k));
        const float2 tail = mul2(mul2(t, poly), e), rest = fma2(tail, both(-1.f), one);
        const float2 phi = make_float2(g.x < 0.f ? tail.x : rest.x, g.y < 0.f ? tail.y : rest.y);
        a = mul2(g, phi);
        slope = fma2(mul2(g, both(0.39894228040143268f)), e, phi);
    } else {
        // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z)), z = c g (1 + 0.044715 g^2): 0 or 1 long before g^2 = 1e9
        constexpr float c = 0.79788456080286536f;
        const float2 sq = mul2(g, g), q = make_float2(fminf(sq.x, 1e9f), fminf(sq.y, 1e9f));
        const float2 x = mul2(fma2(q, both(-2.f * kLog2e * c * 0.044715f), both(-2.f * kLog2e * c)), g);
        const float2 d = add2(make_float2(exp2_fast(x.x), exp2_fast(x.y)), one);
        const float2 s = make_float2(rcp_fast(d.x), rcp_fast(d.y));
        a = mul2(g, s);
        slope = fma2(mul2(a, fma2(q, both(2.f * c * 0.134145f), both(2.f * c))), fma2(s, both(-1.f), one), s);
    }
}
// The same with relu and none at all, which only the linear layer takes.
template <int ACT>
__device__ __forceinline__ void linear_act(float2 z, float2& a, float2& slope) {
    if constexpr (ACT == ATB_ACT_NONE) {
        a = z;
        slope = f32x2::both(1.f);
    } else if constexpr (ACT == ATB_ACT_RELU) {
        // NaN stays NaN
        a = make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);
        slope = make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
    } else {
        // slopes are 0 or 1 long before 1e9, and no product of larger z and 0 is in them; NaN stays NaN.  A caller takes a or the slope.
        const auto near = [](float v) { return v > 1e9f ? 1e9f : v < -1e9f ? -1e9f : v; };
        float2 unused;
        act_value_slope<ACT>(z, a, unused);
        act_value_slope<ACT>(make_float2(near(z.x), near(z.y)), unused, slope);
    }
}
template <int ACT>
__device__ __forceinline__ float2 act_value(float2 z) {
    float2 a, slope;
    linear_act<ACT>(z, a, slope);
    return a;
}
template <class F>
__device__ __forceinline__ void with_linear_act(int act, F&& f) {
    if (act == ATB_ACT_NONE) f(std::integral_constant<int, ATB_ACT_NONE>());
    else if (act == ATB_ACT_RELU) f(std::integral_constant<int, ATB_ACT_RELU>());
    else if (act == ATB_ACT_SILU) f(std::integral_constant<int, ATB_ACT_SILU>());
    else if (act == ATB_ACT_GELU) f(std::integral_constant<int, ATB_ACT_GELU>());
    else f(std::integral_constant<int, ATB_ACT_GELU_TANH>());
}
// f<ACT>() for the runtime value, one branch for a whole tile.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == ATB_ACT_SILU) f(std::integral_constant<int, ATB_ACT_SILU>());
    else if (act == ATB_ACT_GELU) f(std::integral_constant<int, ATB_ACT_GELU>());
    else f(std::integral_constant<int, ATB_ACT_GELU_TANH>());
}

}  // namespace glu
