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

// min and max that hand a NaN on
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The upper tail Q(a) = 1 - Phi(a) of two numbers a in [0, 16], Phi the normal distribution function, and e =
// exp(-a^2 / 2): Q(a) = e (c1 t + .. + c6 t^6), t = 1 / (1 + p a), the form of approximation 7.1.26 of Abramowitz and Stegun,
// Handbook of Mathematical Functions, with coefficients of its own.  Theirs bound the absolute error alone (gelu(-5) came
// out 4 % off, gelu(-6) as 0); these are the minimax fit over [0, 14.2] of the error relative to min(1e-4 Q, 1e-7): at most
// 6.1e-8, and 6.1e-5 of Q.  Beyond 13.2 e and with it Q is below the normal range of fp32 and becomes 0.
// In the epilogue the activation runs beside the tensor cores with two warps a scheduler, so what counts is the length of
// its instruction chain: erff (both of its branches run in every warp) took about 35 instructions an element and the
// product of 8192 x 2048 -> 5632 from 146 to 196 us; this takes about 10 (16384 x 2048 -> 5632 with bias and z: 346 us, as
// with the coefficients of 7.1.26).
__device__ __forceinline__ f32x2 normal_tail2(f32x2 a, f32x2 &e)
{
    float q0, q1, d0, d1;
    unpack2(fma2(both(0.292f), a, both(1.f)), d0, d1);
    const f32x2 t = pack2(rcp_approx(d0), rcp_approx(d1));
    unpack2(mul2(mul2(a, a), both(-0.72134752f)), q0, q1);                                  // log2(e) / 2
    e = pack2(ex2_approx(q0), ex2_approx(q1));
    f32x2 p = fma2(t, both(-0.08676107973f), both(0.2707946002f));
    p = fma2(t, p, both(-0.07628842443f));
    p = fma2(t, p, both(0.1709074378f));
    p = fma2(t, p, both(0.1039059311f));
    p = fma2(t, p, both(0.1174414828f));
    return mul2(mul2(p, t), e);
}

// Activations of two numbers in place.  A NaN stays; infinities go where the limits are: |z| is held to a number past
// which the function is 0 or z in fp32.
template <int ACT>
__device__ __forceinline__ void activate2(float &a, float &b)
{
    if constexpr (ACT == MODSE_ACT_RELU) {
        a = a < 0.f ? 0.f : a;
        b = b < 0.f ? 0.f : b;
    } else if constexpr (ACT == MODSE_ACT_GELU) {
        // z Phi(z) = max(z, 0) - |z| Q(|z|): nothing cancels where z is negative
        f32x2 e;
        const f32x2 m = pack2(min_nan(fabsf(a), 16.f), min_nan(fabsf(b), 16.f)), tail = normal_tail2(m, e);
        unpack2(fma2(mul2(m, both(-1.f)), tail, pack2(fmaxf(a, 0.f), fmaxf(b, 0.f))), a, b);
    } else if constexpr (ACT == MODSE_ACT_SILU) {
        a = max_nan(a, -100.f);
        b = max_nan(b, -100.f);
        float q0, q1;
        unpack2(mul2(pack2(a, b), both(-1.4426950409f)), q0, q1);
        a *= rcp_approx(1.f + ex2_approx(q0));
        b *= rcp_approx(1.f + ex2_approx(q1));
    }
}

// Slopes of two numbers; NaN and infinities as above.  relu's is in times_slope2.
template <int ACT>
__device__ __forceinline__ void act_slope2(float &a, float &b)
{
    if constexpr (ACT == MODSE_ACT_GELU) {
        // Phi(z) + z phi(z), Phi from the tail on its own side
        f32x2 e;
        const float m0 = min_nan(fabsf(a), 16.f), m1 = min_nan(fabsf(b), 16.f);
        float t0, t1;
        unpack2(normal_tail2(pack2(m0, m1), e), t0, t1);
        const f32x2 z = pack2(copysignf(m0, a), copysignf(m1, b));
        unpack2(fma2(mul2(z, e), both(0.39894228040143268f), pack2(a < 0.f ? t0 : 1.f - t0, b < 0.f ? t1 : 1.f - t1)), a, b);     // 1 / sqrt(2 pi)
    } else if constexpr (ACT == MODSE_ACT_SILU) {
        a = min_nan(max_nan(a, -100.f), 100.f);
        b = min_nan(max_nan(b, -100.f), 100.f);
        float q0, q1;
        unpack2(mul2(pack2(a, b), both(-1.4426950409f)), q0, q1);
        const float s0 = rcp_approx(1.f + ex2_approx(q0)), s1 = rcp_approx(1.f + ex2_approx(q1));
        a = s0 * fmaf(a, 1.f - s0, 1.f);
        b = s1 * fmaf(b, 1.f - s1, 1.f);
    }
}

// g times the slope at z, for two numbers.  relu selects: what it masks is 0 even where g is infinite or NaN.
template <int ACT>
__device__ __forceinline__ void times_slope2(float &g0, float &g1, float z0, float z1)
{
    if constexpr (ACT == MODSE_ACT_RELU) {
        g0 = z0 > 0.f ? g0 : 0.f;
        g1 = z1 > 0.f ? g1 : 0.f;
    } else {
        act_slope2<ACT>(z0, z1);
        g0 *= z0;
        g1 *= z1;
    }
}

}  // namespace modse
