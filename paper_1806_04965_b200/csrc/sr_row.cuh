// Rows of matrices in units of VEC elements: what the kernels that go over rows share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "sr_microscale.cuh"
#include "sr_pair.cuh"

namespace srx {

template <typename T, int VEC>
__device__ __forceinline__ void load_unit(const T* p, float (&f)[VEC])
{
    if constexpr (VEC == 1) {
        f[0] = (float)p[0];
    } else if constexpr (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_unit(T* p, const float (&f)[VEC])
{
    if constexpr (VEC == 1) {
        p[0] = (T)f[0];
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// The unit of VEC columns from c on (A: out, scales, groups, tiles_g), one of the lanes of its group of 32; all lanes of the warp take part.  most: bits of its largest magnitude (a NaN's
// are larger than all).
template <int VEC>
__device__ __forceinline__ uint32_t largest(const float (&y)[VEC])
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) most = max(most, __float_as_uint(y[i]) & 0x7FFFFFFFu);
    return most;
}
template <int VEC, int FMT, typename Args>
__device__ __forceinline__ void store_scaled(const Args& A, int64_t row, int64_t c, const float (&y)[VEC], uint32_t most, bool row_there)
{
#pragma unroll
    for (int d = 1; d < 32 / VEC; d *= 2) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    const uint32_t byte = sr_scale_byte<FMT>(most);
    const float inv = sr_inverse_scale(byte);
    const int64_t g = c >> 5;
    float z[VEC];
    if constexpr (VEC == 1) {
        z[0] = y[0] * inv;
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const float2 p = srx::split(srx::mul2(srx::pair(y[i], y[i + 1]), srx::pair(inv, inv)));
            z[i] = p.x;
            z[i + 1] = p.y;
        }
    }
    if constexpr (VEC == 1) {
        if (row_there && (c & 31) == 0 && g < A.tiles_g * 4) A.scales[sr_scale_place(row, g, A.tiles_g)] = (uint8_t)byte;
    } else {
        // the four bytes of a row in a scale tile in one store (two shuffles instead of three stores: as fast, a quarter of the scales' transactions)
        uint32_t word = byte << (8 * (g & 3));
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 32 / VEC);
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 64 / VEC);
        if (row_there && (c & 127) == 0 && g < A.tiles_g * 4) *reinterpret_cast<uint32_t*>(A.scales + sr_scale_place(row, g, A.tiles_g)) = word;
    }
    const bool there = row_there && g < A.groups;
    if constexpr (FMT == SR_FORMAT_MX4) {
        uint8_t* p = static_cast<uint8_t*>(A.out) + row * A.groups * 16 + c / 2;
        if constexpr (VEC == 1) {
            const float up = __shfl_down_sync(0xFFFFFFFFu, z[0], 1);
            if (there && !(c & 1)) *p = (uint8_t)sr_round_e2m1x2(z[0], up);
        } else if constexpr (VEC == 4) {
            if (there) *reinterpret_cast<uint16_t*>(p) = (uint16_t)(sr_round_e2m1x2(z[0], z[1]) | (sr_round_e2m1x2(z[2], z[3]) << 8));
        } else {
            if (there)
                *reinterpret_cast<uint32_t*>(p) = sr_round_e2m1x2(z[0], z[1]) | (sr_round_e2m1x2(z[2], z[3]) << 8) |
                                                  (sr_round_e2m1x2(z[4], z[5]) << 16) | (sr_round_e2m1x2(z[6], z[7]) << 24);
        }
    } else {
        uint8_t* p = static_cast<uint8_t*>(A.out) + row * A.groups * 32 + c;
        if constexpr (VEC == 1) {
            if (there) *p = (uint8_t)sr_round_e4m3x2(z[0], 0.0f);
        } else {
            uint32_t w[VEC / 4];
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) w[i] = sr_round_e4m3x2(z[4 * i], z[4 * i + 1]) | (sr_round_e4m3x2(z[4 * i + 2], z[4 * i + 3]) << 16);
            if (there) {
                if constexpr (VEC == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
                else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
            }
        }
    }
}

// N elements, side by side, at once.
template <typename T, int N>
struct Few {
    static constexpr int BYTES = N * (int)sizeof(T), WORDS = BYTES < 4 ? 1 : BYTES / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void get(const T* p)
    {
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (BYTES == 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[0] = v.x; w[1] = v.y;
        } else if constexpr (BYTES == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void put(T* p) const
    {
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else if constexpr (BYTES == 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (BYTES == 4) {
            *reinterpret_cast<uint32_t*>(p) = w[0];
        } else {
            *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
        }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&f)[N])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
        } else if constexpr (N == 1) {
            w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) w[i / 2] = round_bf16(pair(f[i], f[i + 1]));
        }
    }
};

}  // namespace srx
