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

// log(1 + exp(x)) = max(x, 0) + log1p(e), e = exp(-|x|), and log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3: an odd series in s, here as s times the polynomial of degree 4 in
// s^2 whose largest relative error on [0, 1/9] is smallest (4e-9, by Remez' exchange).  Small steps keep all their digits, as they would not through log(1 + e).
__device__ __forceinline__ float softplus(float x)
{
    const float e = expf(-fabsf(x)), s = __fdividef(e, 2.0f + e), w = s * s;
    float p = 0.28191549f;
    p = fmaf(p, w, 0.27957666f);
    p = fmaf(p, w, 0.40025115f);
    p = fmaf(p, w, 0.66666311f);
    p = fmaf(p, w, 2.0f);
    return fmaf(s, p, fmaxf(x, 0.0f));
}

// 1 / (1 + exp(-x)); EXACT: to the last bits of 32, else to more than those of bf16
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float x)
{
    if constexpr (EXACT) return 1.0f / (1.0f + expf(-x));
    return __fdividef(1.0f, 1.0f + ex2(-kLog2e * x));
}
template <bool EXACT>
__device__ __forceinline__ float silu(float x)
{
    return x * sigmoid<EXACT>(x);
}

}  // namespace srx
