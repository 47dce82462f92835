// The activations of modse_linear and their slopes, shared by the epilogues and the gradient's elementwise pass.
#pragma once

#include "f32x2.h"
#include "modse_internal.h"

namespace modse {

__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Phi(z) - 1/2 of two numbers, Phi the normal distribution function, and e = exp(-z^2 / 2): the rational approximation
// 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions (erfc(x) = (a1 t + .. + a5 t^5) exp(-x^2),
// t = 1 / (1 + p x), error of erf at most 1.5e-7) at x = |z| / sqrt 2, the 1/2 of Phi folded into the coefficients.
// In the epilogue the activation runs beside the tensor cores with two warps a scheduler, so what counts is the length of
// its instruction chain: erff (both of its branches run in every warp) took about 35 instructions an element and the
// product of 8192 x 2048 -> 5632 from 146 to 196 us; this takes 8, and the product from 136 to 145.  Its error is far below the bf16
// rounding of anything computed from it.
__device__ __forceinline__ f32x2 normal_cdf2(f32x2 z, f32x2 &e)
{
    float z0, z1, q0, q1, d0, d1;
    unpack2(z, z0, z1);
    unpack2(fma2(both(0.23164188f), pack2(fabsf(z0), fabsf(z1)), both(1.f)), d0, d1);      // 0.3275911 / sqrt 2
    const f32x2 t = pack2(rcp_approx(d0), rcp_approx(d1));
    unpack2(mul2(mul2(z, z), both(-0.72134752f)), q0, q1);                                  // log2(e) / 2
    e = pack2(ex2_approx(q0), ex2_approx(q1));
    f32x2 p = fma2(t, both(0.5307027145f), both(-0.7265760135f));
    p = fma2(t, p, both(0.7107068705f));
    p = fma2(t, p, both(-0.142248368f));
    p = fma2(t, p, both(0.127414796f));
    float h0, h1;                                                                           // 1/2 - tail, tail = p t e
    unpack2(fma2(mul2(p, t), mul2(e, both(-1.f)), both(0.5f)), h0, h1);
    return pack2(copysignf(h0, z0), copysignf(h1, z1));
}

// Activations of two numbers in place.  A NaN stays; infinities go where the limits are.
template <int ACT>
__device__ __forceinline__ void activate2(float &a, float &b)
{
    if constexpr (ACT == MODSE_ACT_RELU) {
        a = a < 0.f ? 0.f : a;
        b = b < 0.f ? 0.f : b;
    } else if constexpr (ACT == MODSE_ACT_GELU) {
        f32x2 e;
        const f32x2 z = pack2(a, b);
        unpack2(fma2(z, normal_cdf2(z, e), mul2(z, both(0.5f))), a, b);
    } else if constexpr (ACT == MODSE_ACT_SILU) {
        float q0, q1;
        unpack2(mul2(pack2(a, b), both(-1.4426950409f)), q0, q1);
        a *= rcp_approx(1.f + ex2_approx(q0));
        b *= rcp_approx(1.f + ex2_approx(q1));
    }
}

// Slopes of two numbers.
template <int ACT>
__device__ __forceinline__ void act_slope2(float &a, float &b)
{
    if constexpr (ACT == MODSE_ACT_RELU) {
        a = a > 0.f ? 1.f : 0.f;
        b = b > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == MODSE_ACT_GELU) {
        f32x2 e;
        const f32x2 z = pack2(a, b), h = normal_cdf2(z, e);
        float h0, h1;
        unpack2(h, h0, h1);
        unpack2(fma2(mul2(z, e), both(0.39894228040143268f), pack2(h0 + 0.5f, h1 + 0.5f)), a, b);     // 1 / sqrt(2 pi)
    } else if constexpr (ACT == MODSE_ACT_SILU) {
        float q0, q1;
        unpack2(mul2(pack2(a, b), both(-1.4426950409f)), q0, q1);
        const float s0 = rcp_approx(1.f + ex2_approx(q0)), s1 = rcp_approx(1.f + ex2_approx(q1));
        a = s0 * fmaf(a, 1.f - s0, 1.f);
        b = s1 * fmaf(b, 1.f - s1, 1.f);
    } else {
        a = b = 1.f;
    }
}

}  // namespace modse
