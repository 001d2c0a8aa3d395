// Statistics of a softmax: a running maximum, in units of log 2, and the sum of exponentials relative to it.
#pragma once
#include <math.h>

namespace cdl {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void join_stats(float &m, float &s, float m2, float s2)
{
    const float mn = fmaxf(m, m2);
    if (mn != -INFINITY) s = s * exp2_fast(m - mn) + s2 * exp2_fast(m2 - mn);
    else s += s2;                                // (no maximum: 0, or NaN where a logit is NaN)
    m = mn;
}

}  // namespace cdl
