// Activations of the gated feed-forward block and their slopes, in registers.
#pragma once
#include <cuda_runtime.h>

#include <type_traits>

#include "atb.h"

namespace glu {

// 2^x; results below the normal range become 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// act(g) and act'(g).  exp by the fast instruction (2 ulp and the argument's rounding): the results are rounded to
// bf16, 2^-9.  Phi by formula 7.1.26 of Abramowitz and Stegun (erfc(x) = exp(-x^2) times a polynomial of degree 5 in
// 1 / (1 + p x), error below 1.5e-7 for x >= 0; Phi(-g) = 1 - Phi(g)): its exponential is the one that the slope needs.
template <int ACT>
__device__ __forceinline__ void act_value_slope(float g, float& a, float& slope) {
    if constexpr (ACT == ATB_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + exp2_fast(-g * kLog2e));
        a = g * s;
        slope = s + a * (1.f - s);
    } else if constexpr (ACT == ATB_ACT_GELU) {
        const float x = fabsf(g) * 0.70710678118654752f;
        const float t = __fdividef(1.f, 1.f + 0.3275911f * x), e = exp2_fast(-0.5f * kLog2e * g * g);
        const float poly = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
        const float tail = 0.5f * poly * e, phi = g < 0.f ? tail : 1.f - tail;
        a = g * phi;
        slope = phi + g * e * 0.39894228040143268f;
    } else {
        // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
        const float c = 0.79788456080286536f, q = fminf(g * g, 1e9f);     // s is 0 or 1 long before that
        const float s = __fdividef(1.f, 1.f + exp2_fast(-2.f * kLog2e * c * g * (1.f + 0.044715f * q)));
        a = g * s;
        slope = s + 2.f * a * (1.f - s) * c * (1.f + 0.134145f * q);
    }
}
// f<ACT>() for the runtime value, one branch for a whole tile.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == ATB_ACT_SILU) f(std::integral_constant<int, ATB_ACT_SILU>());
    else if (act == ATB_ACT_GELU) f(std::integral_constant<int, ATB_ACT_GELU>());
    else f(std::integral_constant<int, ATB_ACT_GELU_TANH>());
}

}  // namespace glu
