// Microscaled formats (see sr_rollout.h): rounding of a group of 32 values, and the values that codes stand for.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/sr_rollout.h"

// Scale byte of a group from the bits of its largest magnitude: with amax = 1.m * 2^e the smallest k with amax <= M * 2^k is e - 2 (M = 6 = 1.5 * 2^2)
// or e - 8 (M = 448 = 1.75 * 2^8), one more where m is beyond M's.  Infinities and NaNs have the largest exponent field.  The exponent field of
// a subnormal (0) is one less than its exponent, which the lower limit hides.
template <int FMT>
__device__ __forceinline__ uint32_t sr_scale_byte(uint32_t amax_bits)
{
    const int e = (int)(amax_bits >> 23);                             // exponent + 127
    if (e == 255) return 255u;
    const int k = FMT == SR_FORMAT_MX4 ? e - 2 + ((amax_bits & 0x7FFFFFu) > 0x400000u) : e - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u);
    return (uint32_t)(k > 0 ? k : 0);
}
// 2^-(byte - 127), exact for every byte up to 253 (254 does not occur: amax < 2^128); 0 for 255, so that zeros that pad a group which is not finite stay zeros
__device__ __forceinline__ float sr_inverse_scale(uint32_t byte) { return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23); }
// 2^(byte - 127); 2^-127 is subnormal
__device__ __forceinline__ float sr_scale(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FC00000u) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x400000u);
}

__device__ __forceinline__ uint32_t sr_round_e2m1x2(float lo, float hi) { return __nv_cvt_float2_to_fp4x2(make_float2(lo, hi), __NV_E2M1, cudaRoundNearest); }
__device__ __forceinline__ uint32_t sr_round_e4m3x2(float lo, float hi) { return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3); }

// e2m1: sign, two bits of exponent (bias 1), one bit behind the point
__device__ __forceinline__ float sr_e2m1_value(uint32_t code)
{
    const uint32_t e = (code >> 1) & 3u, m = code & 1u;
    const float a = e ? __uint_as_float(((e + 126u) << 23) | (m << 22)) : 0.5f * (float)m;
    return code & 8u ? -a : a;
}
// e4m3: sign, four bits of exponent (bias 7), three bits behind the point
__device__ __forceinline__ float sr_e4m3_value(uint32_t code)
{
    const uint32_t e = (code >> 3) & 15u, m = code & 7u;
    const float a = e ? __uint_as_float(((e + 120u) << 23) | (m << 20)) : (float)m * 0.001953125f;
    return code & 128u ? -a : a;
}

// Sizes of a matrix in a microscaled format.
struct SrScaled {
    int64_t groups, row_bytes, tiles_r, tiles_g;
};
inline SrScaled sr_scaled(int64_t rows, int64_t cols, int format)
{
    SrScaled s;
    s.groups = (cols + 31) / 32;
    s.row_bytes = s.groups * (format == SR_FORMAT_MX4 ? 16 : 32);
    s.tiles_r = (rows + 127) / 128;
    s.tiles_g = (s.groups + 3) / 4;
    return s;
}
__host__ __device__ inline int64_t sr_scale_place(int64_t row, int64_t group, int64_t tiles_g)
{
    return ((row >> 7) * tiles_g + (group >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (group & 3);
}
