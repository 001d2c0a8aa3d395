// Activations and their derivatives (CDL_ACT_*), and the 8-bit checkpoint of what they are taken of: e4m3 codes with one binary32
// scale per 128 consecutive entries of a row, the numbers of cdl_fp8_quantize.
//
//   relu       max(z, 0)
//   gelu       z F(z), F the normal distribution function;                     derivative F + z F'
//   gelu_tanh  z s, s = sigmoid(2 c (z + 0.044715 z^3)), c = sqrt(2 / pi)      (1 + tanh u = 2 sigmoid 2u: no cancellation)
//   silu       z s, s = sigmoid(z);                                            derivative of z s(u(z)): s + z s (1 - s) u'
// NaN gives NaN; at -infinity the values are their limit 0.
//
// F(z) for z < 0 is exp(-z^2 / 2) t P(t), t = 1 / (1 + 0.35 |z|), P a polynomial of degree 8 fitted here to 0.5 erfcx(|z| / sqrt 2) / t for
// the least relative error over 0 <= |z| <= 14.5 (3.2e-8).  There is no cancellation in the tail, where 0.5 (1 + erf) would have it; what the tail
// loses is the exponential's argument, which is rounded to binary32 twice, some z^2 2^-24 of the value.  Largest relative errors of the values in
// binary32, two million numbers a range: gelu 4.3e-7 for |z| up to 1, at z down to -2 5.0e-7, -4 8.6e-7, -6 2.0e-6, -8 3.1e-6, -12 7.6e-6, below 1e-7
// from 1 on; gelu_tanh 2.8e-7, 4.7e-7, 1.1e-6, 3.9e-6, 8.2e-6, and 1.2e-5 at -10; silu 2.2e-7 up to 1, 3.4e-7 at -4, 9.3e-7 at -12, 3.8e-6 at -80.
// Two special-function operations per entry in every activation.
#pragma once
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include "cdl_internal.h"
#include "cdl_softmax.cuh"

namespace cdl {

inline bool valid_act(int act) { return act >= CDL_ACT_NONE && act <= CDL_ACT_SILU; }

constexpr float kFp8InvMax = 1.0f / 448.0f;
constexpr float kFp8Tiny = 1.17549435e-38f;      // 2^-126, the smallest scale

__device__ __forceinline__ void fp8_scale_of(float amax, float &s, float &r)
{
    s = fmaxf(__fmul_rn(amax, kFp8InvMax), kFp8Tiny);
    r = __frcp_rn(s);
}
// codes of two values, the first in the low byte (saturating; NaN becomes the NaN code)
__device__ __forceinline__ uint32_t fp8_code2(float a, float b)
{
    uint16_t w;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(w) : "f"(b), "f"(a));
    return w;
}
// the values of two codes, the first in the low byte (exact: every e4m3 value is a binary16 number)
__device__ __forceinline__ float2 fp8_value2(uint32_t w)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)w));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float min_nan(float a, float b)
{
    float m;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ float rcp_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma_2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul_2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add_2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 exp2_2(float2 x) { return make_float2(exp2_fast(x.x), exp2_fast(x.y)); }
__device__ __forceinline__ float2 rcp_2(float2 x) { return make_float2(rcp_fast(x.x), rcp_fast(x.y)); }
// 1 / (1 + 2^x): 0 and 1 at the infinities
__device__ __forceinline__ float2 logistic_2(float2 x) { return rcp_2(add_2(exp2_2(x), both(1.0f))); }

struct ActPair {
    float2 value, slope;
};

// Two entries at a time, in packed arithmetic where there is one (GELU 12 instructions an entry, 22 without).  What is not asked for is
// not computed.  Arguments are clamped where the result no longer changes, so that no infinity meets a zero.
template <int ACT, bool VALUE, bool SLOPE>
__device__ __forceinline__ ActPair act_pair(float2 z)
{
    ActPair p{z, both(1.0f)};
    if (ACT == CDL_ACT_RELU) {
        p.value = make_float2(max_nan(z.x, 0.0f), max_nan(z.y, 0.0f));
        p.slope = make_float2(z.x <= 0.0f ? 0.0f : (z.x != z.x ? z.x : 1.0f), z.y <= 0.0f ? 0.0f : (z.y != z.y ? z.y : 1.0f));
    } else if (ACT == CDL_ACT_GELU) {
        // q = F(-|z|); the value is max(z, 0) - |z| q on either side
        const float2 a = make_float2(min_nan(fabsf(z.x), 14.5f), min_nan(fabsf(z.y), 14.5f));
        const float2 t = rcp_2(fma_2(both(0.35f), a, both(1.0f))), e = exp2_2(mul_2(mul_2(a, both(-0.5f * kLog2e)), a));
        float2 q = both(-0.029157737269997597f);
        q = fma_2(q, t, both(0.14403025805950165f));
        q = fma_2(q, t, both(-0.25583773851394653f));
        q = fma_2(q, t, both(0.15931838750839233f));
        q = fma_2(q, t, both(-0.023211535066366196f));
        q = fma_2(q, t, both(0.10555218905210495f));
        q = fma_2(q, t, both(0.11982136219739914f));
        q = fma_2(q, t, both(0.1398635059595108f));
        q = fma_2(q, t, both(0.139621302485466f));
        q = mul_2(q, mul_2(t, e));
        const float2 minus = mul_2(a, both(-1.0f));
        if (VALUE) p.value = fma_2(minus, q, make_float2(max_nan(z.x, 0.0f), max_nan(z.y, 0.0f)));
        if (SLOPE) {
            const float2 h = fma_2(mul_2(minus, both(0.39894228040143267794f)), e, q), g = fma_2(h, both(-1.0f), both(1.0f));
            p.slope = make_float2(z.x < 0.0f ? h.x : g.x, z.y < 0.0f ? h.y : g.y);
        }
    } else if (ACT == CDL_ACT_GELU_TANH) {
        constexpr float k2c = 1.59576912160573071176f;      // 2 sqrt(2 / pi)
        const float2 c = SLOPE ? make_float2(min_nan(max_nan(z.x, -30.0f), 30.0f), min_nan(max_nan(z.y, -30.0f), 30.0f)) : z;
        const float2 c2 = mul_2(c, c);
        const float2 s = logistic_2(mul_2(c, fma_2(c2, both(-kLog2e * k2c * 0.044715f), both(-kLog2e * k2c))));
        if (VALUE) p.value = mul_2(make_float2(max_nan(z.x, -FLT_MAX), max_nan(z.y, -FLT_MAX)), s);
        if (SLOPE) p.slope = fma_2(mul_2(mul_2(c, s), fma_2(s, both(-1.0f), both(1.0f))), fma_2(c2, both(k2c * 0.134145f), both(k2c)), s);
    } else if (ACT == CDL_ACT_SILU) {
        const float2 c = SLOPE ? make_float2(min_nan(max_nan(z.x, -100.0f), 100.0f), min_nan(max_nan(z.y, -100.0f), 100.0f)) : z;
        const float2 s = logistic_2(mul_2(c, both(-kLog2e)));
        if (VALUE) p.value = mul_2(make_float2(max_nan(z.x, -FLT_MAX), max_nan(z.y, -FLT_MAX)), s);
        if (SLOPE) p.slope = fma_2(mul_2(c, s), fma_2(s, both(-1.0f), both(1.0f)), s);
    }
    return p;
}
template <int ACT, int N>
__device__ __forceinline__ void act_each(float (&z)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 v = act_pair<ACT, true, false>(make_float2(z[i], N > 1 ? z[(i + 1) % N] : 0.0f)).value;
        z[i] = v.x;
        if (N > 1) z[(i + 1) % N] = v.y;
    }
}
template <int ACT, int N>
__device__ __forceinline__ void slope_each(float (&z)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float2 v = act_pair<ACT, false, true>(make_float2(z[i], N > 1 ? z[(i + 1) % N] : 0.0f)).slope;
        z[i] = v.x;
        if (N > 1) z[(i + 1) % N] = v.y;
    }
}
template <int ACT, int N>
__device__ __forceinline__ void both_each(float (&z)[N], float (&slope)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const ActPair p = act_pair<ACT, true, true>(make_float2(z[i], z[i + 1]));
        z[i] = p.value.x;
        z[i + 1] = p.value.y;
        slope[i] = p.slope.x;
        slope[i + 1] = p.slope.y;
    }
}

// N entries at a time; the activation is the same for a whole launch.
template <int N>
__device__ __forceinline__ void act_values(int act, float (&z)[N])
{
    switch (act) {
    case CDL_ACT_RELU: act_each<CDL_ACT_RELU>(z); break;
    case CDL_ACT_GELU: act_each<CDL_ACT_GELU>(z); break;
    case CDL_ACT_GELU_TANH: act_each<CDL_ACT_GELU_TANH>(z); break;
    case CDL_ACT_SILU: act_each<CDL_ACT_SILU>(z); break;
    default: break;
    }
}
template <int N>
__device__ __forceinline__ void act_slopes(int act, float (&z)[N])      // z -> the derivative there
{
    switch (act) {
    case CDL_ACT_RELU: slope_each<CDL_ACT_RELU>(z); break;
    case CDL_ACT_GELU: slope_each<CDL_ACT_GELU>(z); break;
    case CDL_ACT_GELU_TANH: slope_each<CDL_ACT_GELU_TANH>(z); break;
    case CDL_ACT_SILU: slope_each<CDL_ACT_SILU>(z); break;
    default: slope_each<CDL_ACT_NONE>(z); break;
    }
}
template <int N>
__device__ __forceinline__ void act_both(int act, float (&z)[N], float (&slope)[N])      // z -> the activation, and the derivative
{
    switch (act) {
    case CDL_ACT_RELU: both_each<CDL_ACT_RELU>(z, slope); break;
    case CDL_ACT_GELU: both_each<CDL_ACT_GELU>(z, slope); break;
    case CDL_ACT_GELU_TANH: both_each<CDL_ACT_GELU_TANH>(z, slope); break;
    case CDL_ACT_SILU: both_each<CDL_ACT_SILU>(z, slope); break;
    default: both_each<CDL_ACT_NONE>(z, slope); break;
    }
}

}  // namespace cdl
