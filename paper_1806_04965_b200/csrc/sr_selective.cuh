// What the selective head's kernels compute with.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "sr_pair.cuh"

namespace srx {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^x for two values, to the last bit but one, and without a bias: what a state is multiplied with over thousands of frames may not drift (ex2 is low by 2e-8 in the mean, which
// a state that loses a thousandth of itself per frame makes 2e-5 of).  x = n + f, |f| <= 1/2, by adding 1.5 * 2^23; 2^f = 1 + f q(f) with q of degree 4 for the smallest
// largest error of f q(f) (9e-8 f, by Remez' exchange); n goes into the exponent.  Below -126: 2^-126; from 128 on: 2^128 but a little.  A NaN stays one: its bits and the exponent's could
// add up to any number, so it is chosen at the end.
__device__ __forceinline__ Pair exp2_exact(Pair x)
{
    const float2 v = split(x);
    float lo, hi;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(lo) : "f"(v.x), "f"(-126.0f));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(hi) : "f"(v.y), "f"(-126.0f));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(lo) : "f"(lo), "f"(127.99999f));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(hi) : "f"(hi), "f"(127.99999f));
    const Pair y = pair(lo, hi), magic = pair(12582912.0f, 12582912.0f), t = add2(y, magic);
    const Pair f = fma2(add2(t, pair(-12582912.0f, -12582912.0f)), pair(-1.0f, -1.0f), y);
    Pair q = pair(0.0013407238f, 0.0013407238f);
    q = fma2(q, f, pair(0.0096718613f, 0.0096718613f));
    q = fma2(q, f, pair(0.055503085f, 0.055503085f));
    q = fma2(q, f, pair(0.24022235f, 0.24022235f));
    q = fma2(q, f, pair(0.69314724f, 0.69314724f));
    const float2 m = split(fma2(q, f, pair(1.0f, 1.0f))), n = split(t);
    const float a = __uint_as_float(__float_as_uint(m.x) + (__float_as_uint(n.x) << 23)), b = __uint_as_float(__float_as_uint(m.y) + (__float_as_uint(n.y) << 23));
    return pair(v.x != v.x ? v.x : a, v.y != v.y ? v.y : b);
}
__device__ __forceinline__ float exp2_exact(float x) { return split(exp2_exact(pair(x, x))).x; }

// A state's decay per step, in base 2; finite, so that a step of nothing leaves the state as it is.
__device__ __forceinline__ float decay_base2(float a) { return a != a ? a : fminf(fmaxf(kLog2e * a, -3.0e38f), 3.0e38f); }

// log(1 + exp(x)) = max(x, 0) + log1p(e), e = exp(-|x|), and log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3: an odd series in s, here as s times the polynomial of degree 4 in
// s^2 whose largest relative error on [0, 1/9] is smallest (4e-9, by Remez' exchange).  Small steps keep all their digits, as they would not through log(1 + e).
// EXACT: e to its last bits, else to |x| 2^-24.
template <bool EXACT>
__device__ __forceinline__ float softplus(float x)
{
    const float e = EXACT ? expf(-fabsf(x)) : ex2(-kLog2e * fabsf(x)), s = e * reciprocal(2.0f + e), w = s * s;
    float p = 0.28191549f;
    p = fmaf(p, w, 0.27957666f);
    p = fmaf(p, w, 0.40025115f);
    p = fmaf(p, w, 0.66666311f);
    p = fmaf(p, w, 2.0f);
    return fmaf(s, p, fmaxf(x, 0.0f));
}

// 1 / (1 + exp(-x)), zero where that is below 2^-126; EXACT: to the last two bits of 32 (the approximate reciprocal is off by one), else to more than those of bf16
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float x)
{
    return reciprocal(1.0f + (EXACT ? expf(-x) : ex2(-kLog2e * x)));
}
template <bool EXACT>
__device__ __forceinline__ float silu(float x)
{
    return x * sigmoid<EXACT>(x);
}
template <bool EXACT>
__device__ __forceinline__ Pair sigmoid(Pair x)
{
    if constexpr (EXACT) {
        const float2 v = split(x);
        return pair(sigmoid<true>(v.x), sigmoid<true>(v.y));
    }
    const float2 e = split(mul2(x, pair(-kLog2e, -kLog2e))), n = split(add2(pair(ex2(e.x), ex2(e.y)), pair(1.0f, 1.0f)));
    return pair(reciprocal(n.x), reciprocal(n.y));
}
template <bool EXACT>
__device__ __forceinline__ Pair silu(Pair x)
{
    return mul2(x, sigmoid<EXACT>(x));
}

}  // namespace srx
