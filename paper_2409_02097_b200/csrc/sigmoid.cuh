// The logistic function from the special function unit: an exponential and a reciprocal a value.
#pragma once

#include "common.cuh"
#include "packed_math.cuh"

namespace lf {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / x of two values.
__device__ __forceinline__ f32x2 rcp2(f32x2 x)
{
    const float2 d = unpack2(x);
    return pack2(rcp_approx(d.x), rcp_approx(d.y));
}
// exp(-x) of two values.
__device__ __forceinline__ f32x2 exp_minus2(f32x2 x)
{
    const float2 t = unpack2(mul2(x, both(-kLog2e)));
    return pack2(ex2_approx(t.x), ex2_approx(t.y));
}
// 1 / (1 + exp(-x)), and of two values.
__device__ __forceinline__ float sigmoid1(float x) { return rcp_approx(1.0f + ex2_approx(-kLog2e * x)); }
__device__ __forceinline__ f32x2 sigmoid2(f32x2 x) { return rcp2(add2(exp_minus2(x), both(1.0f))); }

}  // namespace lf
