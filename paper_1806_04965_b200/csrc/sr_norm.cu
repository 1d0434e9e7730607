// Root-mean-square norm with the residual's addition, and quantisation to the microscaled formats: both are one pass over
// rows, bound by memory: bytes of x, the residual, the sum and the output, each once.
//
//     s = x + residual,   out = s / sqrt(mean(s^2) + eps) * weight,   out rounded to its type, or to groups of 32 with a scale.
//
// A row lies in the registers of the threads that share it (32 to 1024 of them, a few units of VEC elements each) between the
// sum of squares and the output, so that nothing is read twice; longer rows are read again (they come out of L2).  The
// lanes of a group of 32 columns find its largest magnitude with shuffles.  16384 x 1024 fp32 with residual and sum 41.2 us (6.5 TB/s), bf16 22.7 (5.9);
// rows of 1003, which no 16-byte access fits by itself, 53.2.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "sr_microscale.cuh"
#include "sr_pair.cuh"
#include "sr_ptx.cuh"

namespace {

struct RowArgs {
    const void* x;
    const void* residual;
    const float* weight;
    void* sum;
    void* out;
    uint8_t* scales;
    int64_t rows, cols, x_stride, r_stride;
    int64_t tiles_g, groups;
    float eps;
};

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

// The unit of VEC columns from c on, one of the lanes of its group of 32; all lanes of the warp take part.  most: bits of its largest magnitude (a NaN's
// are larger than all).
template <int VEC>
__device__ __forceinline__ uint32_t largest(const float (&y)[VEC])
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) most = max(most, __float_as_uint(y[i]) & 0x7FFFFFFFu);
    return most;
}
template <int VEC, int FMT>
__device__ __forceinline__ void store_scaled(const RowArgs& A, int64_t row, int64_t c, const float (&y)[VEC], uint32_t most, bool row_there)
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

// HOLD: units of a thread that stay in registers; 0: rows of any length, read twice.  FMT F32: the type of x.
// Two blocks to an SM (32 registers) where single values are held or rows are read again: the code for rare rows would take 46 (16384 x 1003 fp32 to 8 bits 88 us and 104).
// SHIFT: rows that do not start on 16 bytes, but alike in all buffers: a thread's units do, the first of a row may begin ahead of it.
template <typename T, int VEC, int HOLD, bool NORM, int FMT, bool SHIFT>
__global__ void __launch_bounds__(1024, NORM && (HOLD == 0 || (VEC == 1 && HOLD == 8)) ? 2 : 0) sr_row_kernel(const __grid_constant__ RowArgs A)
{
    __shared__ float part[32];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool row_there = row < A.rows;
    const int64_t r0 = row_there ? row : 0;
    const T* x = static_cast<const T*>(A.x) + r0 * A.x_stride;
    const T* res = NORM && A.residual ? static_cast<const T*>(A.residual) + r0 * A.r_stride : nullptr;
    const int tpr = blockDim.x, tid = threadIdx.x;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols + (SHIFT ? VEC : 0);          // (units may begin a part of one ahead of the row)
    const int n_it = HOLD ? HOLD : (int)((end + (int64_t)tpr * VEC - 1) / ((int64_t)tpr * VEC));
    const int64_t shift = SHIFT ? (int64_t)(((uintptr_t)x & 15) / sizeof(T)) : 0;
    auto column = [&](int it) { return ((int64_t)it * tpr + tid) * VEC - shift; };
    // the whole unit, or its columns that there are
    auto whole = [&](int64_t c) { return !SHIFT || (c >= 0 && c + VEC <= A.cols); };

    auto load = [&](int it, float (&f)[VEC]) {
        const int64_t c = column(it);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = 0.0f;
        if (row_there && c < A.cols && !whole(c)) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i >= 0 && c + i < A.cols) f[i] = (float)x[c + i] + (res ? (float)res[c + i] : 0.0f);
        } else if (row_there && c < A.cols) {
            load_unit<T, VEC>(x + c, f);
            if (NORM && res) {
                float g[VEC];
                load_unit<T, VEC>(res + c, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[i] += g[i];
            }
        }
    };
    // a unit, or its columns that there are
    auto put = [&](T* to, int64_t c, const float (&s)[VEC]) {
        const bool there = row_there && c < A.cols;
        if (there && whole(c)) {
            store_unit<T, VEC>(to + row * A.cols + c, s);
        } else if (SHIFT && there) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (c + i >= 0 && c + i < A.cols) to[row * A.cols + c + i] = (T)s[i];
        }
    };
    float f[HOLD ? HOLD : 1][VEC];
    float inv = 1.0f, by = 1.0f;                       // what a row is multiplied with; ahead of that (rows that are read again)
    if (HOLD) {
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : 1); ++it) load(it, f[it]);
    }
    if (NORM) {
        float ss = 0.0f;
        if (HOLD) {
#pragma unroll
            for (int it = 0; it < (HOLD ? HOLD : 1); ++it)
#pragma unroll
                for (int i = 0; i < VEC; ++i) ss = fmaf(f[it][i], f[it][i], ss);
        } else {
            for (int it = 0; it < n_it; ++it) {
                load(it, f[0]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) ss = fmaf(f[0][i], f[0][i], ss);
            }
        }
        auto over_row = [&](float mine, auto join) {   // over the row's threads; 0 joins nothing
#pragma unroll
            for (int d = 16; d; d /= 2) mine = join(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, d));
            if (tpr > 32) {                            // (one row per block)
                if (!(tid & 31)) part[tid >> 5] = mine;
                __syncthreads();
                mine = (tid & 31) < (tpr >> 5) ? part[tid & 31] : 0.0f;
#pragma unroll
                for (int d = 16; d; d /= 2) mine = join(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, d));
            }
            return mine;
        };
        auto add = [](float a, float b) { return a + b; };
        ss = over_row(ss, add);
        const float mean = ss / (float)A.cols + A.eps;
        inv = 1.0f / sqrtf(mean);
        if (HOLD && A.sum)                             // (ahead of what a rare row does to its values)
#pragma unroll
            for (int it = 0; it < (HOLD ? HOLD : 1); ++it) put(static_cast<T*>(A.sum), column(it), f[it]);
        if (!(mean >= 0x1p-100f && ss <= 3.4028234e38f)) {
            // (the same for all threads of the row) Squares that 32 bits do not hold, or so small that they have lost bits: once more with the row divided by the power of two
            // of its largest value, or of sqrt(eps).
            auto each = [&](auto what) {
                if (HOLD) {
#pragma unroll
                    for (int it = 0; it < (HOLD ? HOLD : 1); ++it)
#pragma unroll
                        for (int i = 0; i < VEC; ++i) what(f[it][i], column(it) + i < A.cols);
                } else {
#pragma unroll 1
                    for (int it = 0; it < n_it; ++it) {
                        load(it, f[0]);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) what(f[0][i], true);
                    }
                }
            };
            const float root = sqrtf(A.eps);
            uint32_t most = __float_as_uint(root);
            each([&](float& y, bool) { most = max(most, __float_as_uint(y) & 0x7FFFFFFFu); });
            if (tpr > 32) __syncthreads();
            most = __float_as_uint(over_row(__uint_as_float(most), [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
            // (what is not finite: as the formula has it)
            if (most < 0x7F800000u) by = __uint_as_float((254u - min(max(most >> 23, 1u), 253u)) << 23);
            ss = 0.0f;
            each([&](float& y, bool) { ss = fmaf(y * by, y * by, ss); });
            if (tpr > 32) __syncthreads();
            ss = over_row(ss, add);
            inv = 1.0f / sqrtf(ss / (float)A.cols + root * by * (root * by));
            if (HOLD) {
                each([&](float& y, bool there) { y = there ? y * by * inv : 0.0f; });      // (zeros behind the last column whatever inv is)
                inv = 1.0f;
            }
        }
    }
    auto finish = [&](int it, float (&s)[VEC]) {
        const int64_t c = column(it);
        const bool there = row_there && c < A.cols;
        if (NORM && !HOLD && A.sum) put(static_cast<T*>(A.sum), c, s);
        if (NORM) {
            float w[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = 1.0f;
            if (there && A.weight) {
                if constexpr (SHIFT) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (c + i >= 0 && c + i < A.cols) w[i] = A.weight[c + i];
                } else if constexpr (VEC == 8) {
                    float lo[4], hi[4];
                    load_unit<float, 4>(A.weight + c, lo);
                    load_unit<float, 4>(A.weight + c + 4, hi);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { w[i] = lo[i]; w[4 + i] = hi[i]; }
                } else {
                    load_unit<float, VEC>(A.weight + c, w);
                }
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if (HOLD) s[i] = s[i] * inv * w[i];
                else s[i] = there ? s[i] * by * inv * w[i] : 0.0f;
            }
        }
        if constexpr (FMT >= SR_FORMAT_MX8) store_scaled<VEC, FMT>(A, row, c, s, largest(s), row_there);
        else put(static_cast<T*>(A.out), c, s);
    };
    if (HOLD) {
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : 1); ++it) finish(it, f[it]);
    } else {
        for (int it = 0; it < n_it; ++it) {
            load(it, f[0]);
            finish(it, f[0]);
        }
    }
}

// Quantisation of bf16 rows whose 16-byte units can be read as they lie: what the kernel above does, without a row's reduction, and with the largest magnitude
// taken from pairs of bf16.  A thread has two units, 256 columns apart.  Bound by instructions rather than memory: 8192 x 4096 to 4 bits 19.9 us (4.3 TB/s); 26 with the
// kernel above, which issues 162 instructions per 8 values.
template <int FMT>
__global__ void __launch_bounds__(256) sr_quantize_kernel(const __grid_constant__ RowArgs A, uint32_t strips)
{
    constexpr int UNITS = 2;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const uint32_t warp = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int64_t row = warp / strips;                 // a warp has a strip of 512 columns
    const uint32_t c0 = (warp - (uint32_t)row * strips) * (256 * UNITS) + lane * 8;
    if (row >= A.rows) return;
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(A.x) + row * A.x_stride;
    uint4 w[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) w[k] = c0 + 256 * k < A.cols ? *reinterpret_cast<const uint4*>(x + c0 + 256 * k) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const uint32_t in[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        uint32_t most = 0;
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            most = __vmaxu2(most, in[i] & 0x7FFF7FFFu);
            y[2 * i] = __uint_as_float(in[i] << 16);
            y[2 * i + 1] = __uint_as_float(in[i] & 0xFFFF0000u);
        }
        store_scaled<8, FMT>(A, row, c0 + 256 * k, y, max(most & 0xFFFF0000u, most << 16), true);
    }
}

template <typename T, int VEC, int HOLD, bool NORM, int FMT, bool SHIFT>
cudaError_t launch_one(const RowArgs& A, int tpr, cudaStream_t s)
{
    const int rpb = tpr == 32 ? 4 : 1;
    const int64_t blocks = (A.rows + rpb - 1) / rpb;
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)tpr, (unsigned)rpb);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sr_row_kernel<T, VEC, HOLD, NORM, FMT, SHIFT>, A);
}
// Threads of a row: as many as give each of them HOLD units.  One unit of 16 bytes is best as long as 1024 threads reach (16384 x 1024 of bf16 22 us, with four 31;
// 8 x 1024 2.2 and 4.6); single values want eight (16384 x 2001 of bf16 one by one 111, with four 126, with one 329).
template <typename T, int VEC, bool NORM, int FMT, bool SHIFT>
cudaError_t launch_rows(const RowArgs& A, cudaStream_t s)
{
    constexpr int FEW = VEC > 1 ? 1 : 8, MANY = VEC > 1 ? 4 : 16;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols;
    const int64_t units = (end + VEC - 1) / VEC + (SHIFT ? 1 : 0);
    for (const int hold : {FEW, MANY}) {
        int tpr = 32;
        while (tpr < 1024 && (int64_t)tpr * hold < units) tpr *= 2;
        if ((int64_t)tpr * hold >= units) return hold == FEW ? launch_one<T, VEC, FEW, NORM, FMT, SHIFT>(A, tpr, s) : launch_one<T, VEC, MANY, NORM, FMT, SHIFT>(A, tpr, s);
    }
    return launch_one<T, VEC, 0, NORM, FMT, SHIFT>(A, 1024, s);
}
template <typename T, int VEC>
cudaError_t launch_any(const RowArgs& A, bool norm, int fmt, cudaStream_t s)
{
    if constexpr (VEC != 8) {                          // (that is sr_quantize_kernel's)
        if (!norm) return fmt == SR_FORMAT_MX4 ? launch_rows<T, VEC, false, SR_FORMAT_MX4, false>(A, s) : launch_rows<T, VEC, false, SR_FORMAT_MX8, false>(A, s);
    }
    if (fmt == SR_FORMAT_MX4) return launch_rows<T, VEC, true, SR_FORMAT_MX4, false>(A, s);
    if (fmt == SR_FORMAT_MX8) return launch_rows<T, VEC, true, SR_FORMAT_MX8, false>(A, s);
    return launch_rows<T, VEC, true, SR_FORMAT_F32, false>(A, s);
}
// 16-byte accesses where every row of every buffer allows them, or all of them start equally far from where it would.
template <typename T>
cudaError_t launch(const RowArgs& A, bool norm, int fmt, cudaStream_t s)
{
    constexpr int el = sizeof(T), vec = 16 / el;
    auto fits = [&](const void* p, int64_t stride) { return !((uintptr_t)p & 15) && stride % vec == 0; };
    if (A.cols % vec == 0 && fits(A.x, A.x_stride) && (!A.residual || fits(A.residual, A.r_stride)) && !((uintptr_t)A.sum & 15) && !((uintptr_t)A.out & 15) &&
        !((uintptr_t)A.weight & 15))
        return launch_any<T, vec>(A, norm, fmt, s);
    auto like = [&](const void* p, int64_t stride) { return !p || (((uintptr_t)p ^ (uintptr_t)A.x) % 16 == 0 && (stride - A.x_stride) % vec == 0); };
    if (norm && fmt < SR_FORMAT_MX8 && like(A.residual, A.r_stride) && like(A.sum, A.cols) && like(A.out, A.cols)) return launch_rows<T, vec, true, SR_FORMAT_F32, true>(A, s);
    return launch_any<T, 1>(A, norm, fmt, s);
}
cudaError_t launch(const RowArgs& A, bool norm, int dtype, int fmt, cudaStream_t s)
{
    const int64_t strips = (A.tiles_g * 128 + 511) / 512, blocks = (A.rows * strips + 7) / 8;
    if (!norm && dtype == SR_DTYPE_BF16 && A.cols % 8 == 0 && !((uintptr_t)A.x & 15) && A.x_stride % 8 == 0) {
        if (blocks > 0x1FFFFFFF) return cudaErrorInvalidValue;       // (the warps' numbers have 32 bits; so many strips are more than a terabyte)
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)blocks);
        cfg.blockDim = dim3(256);
        cfg.stream = s;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        return fmt == SR_FORMAT_MX4 ? cudaLaunchKernelEx(&cfg, sr_quantize_kernel<SR_FORMAT_MX4>, A, (uint32_t)strips)
                                    : cudaLaunchKernelEx(&cfg, sr_quantize_kernel<SR_FORMAT_MX8>, A, (uint32_t)strips);
    }
    return dtype == SR_DTYPE_F32 ? launch<float>(A, norm, fmt, s) : launch<__nv_bfloat16>(A, norm, fmt, s);
}

// Two elements per thread.
template <int FMT>
__global__ void sr_values_kernel(const uint8_t* data, const uint8_t* scales, int64_t rows, int64_t cols, int64_t groups, int64_t tiles_g, float* out)
{
    const int64_t pairs = groups * 16, n = rows * pairs;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = i / pairs, c = (i - row * pairs) * 2;
        if (c >= cols) continue;
        const float s = sr_scale(scales[sr_scale_place(row, c >> 5, tiles_g)]);
        float lo, hi;
        if (FMT == SR_FORMAT_MX4) {
            const uint32_t b = data[i];
            lo = sr_e2m1_value(b & 15u);
            hi = sr_e2m1_value(b >> 4);
        } else {
            const uint32_t b = reinterpret_cast<const uint16_t*>(data)[i];
            lo = sr_e4m3_value(b & 255u);
            hi = sr_e4m3_value(b >> 8);
        }
        out[row * cols + c] = lo * s;
        if (c + 1 < cols) out[row * cols + c + 1] = hi * s;
    }
}

bool scaled_format(int f) { return f == SR_FORMAT_MX8 || f == SR_FORMAT_MX4; }
constexpr int64_t kMostRows = (int64_t)1 << 31, kMostCols = (int64_t)1 << 31;

}  // namespace

extern "C" {

sr_status sr_microscale_bytes(int64_t rows, int64_t cols, int format, size_t* data_bytes, size_t* scale_bytes)
{
    if (!data_bytes || !scale_bytes || !scaled_format(format) || rows < 0 || cols < 1 || rows >= kMostRows || cols >= kMostCols) return SR_ERR_INVALID_ARG;
    const SrScaled z = sr_scaled(rows, cols, format);
    *data_bytes = (size_t)rows * (size_t)z.row_bytes;
    *scale_bytes = (size_t)z.tiles_r * (size_t)z.tiles_g * 512;
    return SR_OK;
}

sr_status sr_microscale_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride, int format, void* data, void* scales,
                                 void* stream)
{
    if ((dtype != SR_DTYPE_F32 && dtype != SR_DTYPE_BF16) || !scaled_format(format) || rows < 0 || cols < 1 || rows >= kMostRows || cols >= kMostCols ||
        row_stride < 0)
        return SR_ERR_INVALID_ARG;
    if (!rows) return SR_OK;
    const int el = dtype == SR_DTYPE_F32 ? 4 : 2;
    if (!x || !data || !scales || (uintptr_t)x % el || ((uintptr_t)data & 15) || ((uintptr_t)scales & 15)) return SR_ERR_INVALID_ARG;
    const SrScaled z = sr_scaled(rows, cols, format);
    RowArgs A{};
    A.x = x;
    A.out = data;
    A.scales = static_cast<uint8_t*>(scales);
    A.rows = rows;
    A.cols = cols;
    A.x_stride = row_stride;
    A.tiles_g = z.tiles_g;
    A.groups = z.groups;
    return launch(A, false, dtype, format, static_cast<cudaStream_t>(stream)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_microscale_values(const void* data, const void* scales, int format, int64_t rows, int64_t cols, float* out, void* stream)
{
    if (!scaled_format(format) || rows < 0 || cols < 1 || rows >= kMostRows || cols >= kMostCols) return SR_ERR_INVALID_ARG;
    if (!rows) return SR_OK;
    if (!data || !scales || !out || ((uintptr_t)data & 15) || ((uintptr_t)scales & 15) || ((uintptr_t)out & 3)) return SR_ERR_INVALID_ARG;
    const SrScaled z = sr_scaled(rows, cols, format);
    const int64_t blocks = std::min<int64_t>((rows * z.groups * 16 + 255) / 256, 1 << 20);
    const uint8_t *d = static_cast<const uint8_t*>(data), *sc = static_cast<const uint8_t*>(scales);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (format == SR_FORMAT_MX4) sr_values_kernel<SR_FORMAT_MX4><<<(unsigned)blocks, 256, 0, s>>>(d, sc, rows, cols, z.groups, z.tiles_g, out);
    else sr_values_kernel<SR_FORMAT_MX8><<<(unsigned)blocks, 256, 0, s>>>(d, sc, rows, cols, z.groups, z.tiles_g, out);
    return cudaGetLastError() == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_rms_norm(const void* x, const void* residual, const float* weight, float eps, int dtype, int64_t rows, int64_t cols, int64_t x_stride,
                      int64_t residual_stride, void* sum, void* out, int out_format, void* scales, void* stream)
{
    if ((dtype != SR_DTYPE_F32 && dtype != SR_DTYPE_BF16) || rows < 0 || cols < 1 || rows >= kMostRows || cols >= kMostCols || x_stride < 0 ||
        (residual && residual_stride < 0) || !(eps >= 0.0f))
        return SR_ERR_INVALID_ARG;
    if (!scaled_format(out_format) && out_format != dtype) return SR_ERR_INVALID_ARG;
    if (!rows) return SR_OK;
    const int el = dtype == SR_DTYPE_F32 ? 4 : 2;
    if (!x || !out || (uintptr_t)x % el || (uintptr_t)residual % el || (uintptr_t)sum % el || (uintptr_t)weight % 4) return SR_ERR_INVALID_ARG;
    // in place: every element is read before it is written only where the two lie alike
    if (sum && ((sum == x && x_stride != cols && rows > 1) || (sum == residual && residual_stride != cols && rows > 1))) return SR_ERR_INVALID_ARG;
    RowArgs A{};
    if (scaled_format(out_format)) {
        if (!scales || ((uintptr_t)out & 15) || ((uintptr_t)scales & 15)) return SR_ERR_INVALID_ARG;
        const SrScaled z = sr_scaled(rows, cols, out_format);
        A.tiles_g = z.tiles_g;
        A.groups = z.groups;
        A.scales = static_cast<uint8_t*>(scales);
    } else if (scales || (uintptr_t)out % el) {
        return SR_ERR_INVALID_ARG;
    }
    A.x = x;
    A.residual = residual;
    A.weight = weight;
    A.sum = sum;
    A.out = out;
    A.rows = rows;
    A.cols = cols;
    A.x_stride = x_stride;
    A.r_stride = residual ? residual_stride : 0;
    A.eps = eps;
    return launch(A, true, dtype, out_format, static_cast<cudaStream_t>(stream)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
