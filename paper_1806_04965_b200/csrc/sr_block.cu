// The way out of a block and into the next one, one pass over rows:
//
//     h = residual + scale * act(gate) * rms(y) * weight_after,   out = rms(h) * weight_before,   rms(x) = x / sqrt(mean(x^2) + eps).
//
// Bound by memory: y, residual and gate in, h and out out, each once.  A row lies in the registers of the threads that share it through both reductions: y as floats, turned
// into h in place; residual and gate as they were read, ahead of the first reduction, so that their loads are under way during it.  Longer rows are read again (out of L2).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "sr_microscale.cuh"
#include "sr_ptx.cuh"
#include "sr_row.cuh"
#include "sr_selective.cuh"

namespace {

struct BlockArgs {
    const void *y, *residual, *gate;
    const float *after, *before;
    void *h, *out;
    uint8_t* scales;
    int64_t rows, cols, y_stride, r_stride, g_stride;
    int64_t tiles_g, groups;
    float scale, eps;
    int32_t norms, act;
};

// VEC elements as they lie in memory
template <typename T, int VEC>
struct Raw {
    uint4 bits;
    __device__ __forceinline__ void get(const T* p) { bits = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ float operator[](int i) const
    {
        const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
};
template <typename T>
struct Raw<T, 1> {
    T bits;
    __device__ __forceinline__ void get(const T* p) { bits = *p; }
    __device__ __forceinline__ float operator[](int) const { return (float)bits; }
};

template <int VEC>
__device__ __forceinline__ void load_weight(const float* w, int64_t c, float (&f)[VEC])
{
    if constexpr (VEC == 8) {
        float lo[4], hi[4];
        srx::load_unit<float, 4>(w + c, lo);
        srx::load_unit<float, 4>(w + c + 4, hi);
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[i] = lo[i]; f[4 + i] = hi[i]; }
    } else {
        srx::load_unit<float, VEC>(w + c, f);
    }
}

// HOLD: units of a thread that stay in registers; 0: rows of any length, read again.  FMT F32: the type of y.
template <typename T, int VEC, int HOLD, int FMT>
__global__ void __launch_bounds__(1024) sr_block_kernel(const __grid_constant__ BlockArgs A)
{
    constexpr int H = HOLD ? HOLD : 1;
    constexpr bool EXACT = sizeof(T) == 4;
    __shared__ float part[2][32];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const bool row_there = row < A.rows;
    const int64_t r0 = row_there ? row : 0;
    const T* y = static_cast<const T*>(A.y) + r0 * A.y_stride;
    const T* res = static_cast<const T*>(A.residual) + r0 * A.r_stride;
    const T* gate = A.gate ? static_cast<const T*>(A.gate) + r0 * A.g_stride : nullptr;
    const int tpr = blockDim.x, tid = threadIdx.x;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols;
    const int n_it = HOLD ? HOLD : (int)((end + (int64_t)tpr * VEC - 1) / ((int64_t)tpr * VEC));
    auto column = [&](int it) { return ((int64_t)it * tpr + tid) * VEC; };
    auto there = [&](int it) { return row_there && column(it) < A.cols; };

    float f[H][VEC];
    Raw<T, VEC> rr[H], gg[H];
    auto load_y = [&](int it, int k) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[k][i] = 0.0f;
        if (there(it)) srx::load_unit<T, VEC>(y + column(it), f[k]);
    };
    auto load_rest = [&](int it, int k) {
        if (!there(it)) return;
        rr[k].get(res + column(it));
        if (gate) gg[k].get(gate + column(it));
    };
    auto over_row = [&](float mine, int which, auto join) {       // over the row's threads; 0 joins nothing
#pragma unroll
        for (int d = 16; d; d /= 2) mine = join(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, d));
        if (tpr > 32) {                                // (one row per block)
            if (!(tid & 31)) part[which][tid >> 5] = mine;
            __syncthreads();
            mine = (tid & 31) < (tpr >> 5) ? part[which][tid & 31] : 0.0f;
#pragma unroll
            for (int d = 16; d; d /= 2) mine = join(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, d));
        }
        return mine;
    };
    // 1 / sqrt(mean(x^2) + eps) of the row that `unit` brings into f, as two factors: by is a power of two, 1 but where squares leave the range of 32 bits
    auto inverse = [&](int which, auto unit, float& by, float& inv) {
        auto add = [](float a, float b) { return a + b; };
        float ss = 0.0f;
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
            const int k = unit(it);
#pragma unroll
            for (int i = 0; i < VEC; ++i) ss = fmaf(f[k][i], f[k][i], ss);
        }
        ss = over_row(ss, which, add);
        const float mean = ss / (float)A.cols + A.eps;
        inv = 1.0f / sqrtf(mean);
        by = 1.0f;
        if (mean >= 0x1p-100f && ss <= 3.4028234e38f) return;
        // (the same for all threads of the row) once more, divided by the power of two of the largest value, or of sqrt(eps)
        const float root = sqrtf(A.eps);
        uint32_t most = __float_as_uint(root);
#pragma unroll 1
        for (int it = 0; it < n_it; ++it) {
            if (!HOLD) unit(it);
#pragma unroll
            for (int k = 0; k < H; ++k)
                if (!HOLD || k == it)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) most = max(most, __float_as_uint(f[k][i]) & 0x7FFFFFFFu);
        }
        if (tpr > 32) __syncthreads();
        most = __float_as_uint(over_row(__uint_as_float(most), which, [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
        // (what is not finite: as the formula has it)
        if (most < 0x7F800000u) by = __uint_as_float((254u - min(max(most >> 23, 1u), 253u)) << 23);
        ss = 0.0f;
#pragma unroll 1
        for (int it = 0; it < n_it; ++it) {
            if (!HOLD) unit(it);
#pragma unroll
            for (int k = 0; k < H; ++k)
                if (!HOLD || k == it)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) ss = fmaf(f[k][i] * by, f[k][i] * by, ss);
        }
        if (tpr > 32) __syncthreads();
        ss = over_row(ss, which, add);
        inv = 1.0f / sqrtf(ss / (float)A.cols + root * by * (root * by));
    };
    if (HOLD) {
#pragma unroll
        for (int k = 0; k < H; ++k) load_y(k, k);
#pragma unroll
        for (int k = 0; k < H; ++k) load_rest(k, k);
    }
    float by = 1.0f, inv = 1.0f;
    if (A.norms & SR_NORM_AFTER)
        inverse(0, [&](int it) {
            if (!HOLD) load_y(it, 0);
            return HOLD ? it : 0;
        }, by, inv);
    // y in f[k] becomes h
    auto join = [&](int it, int k) {
        if (!there(it)) return;
        float w[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = 1.0f;
        if ((A.norms & SR_NORM_AFTER) && A.after) load_weight<VEC>(A.after, column(it), w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float p = A.norms & SR_NORM_AFTER ? f[k][i] * by * inv * w[i] : f[k][i];
            if (gate) {
                const float x = gg[k][i];
                p *= A.act == 0 ? x : A.act == 1 ? srx::sigmoid<EXACT>(x) : srx::silu<EXACT>(x);
            }
            f[k][i] = fmaf(A.scale, p, rr[k][i]);
        }
    };
    auto make = [&](int it) {                          // (rows that are read again)
        load_y(it, 0);
        load_rest(it, 0);
        join(it, 0);
    };
#pragma unroll
    for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
        const int k = HOLD ? it : 0;
        if (HOLD) join(it, k);
        else make(it);
        if (there(it)) srx::store_unit<T, VEC>(static_cast<T*>(A.h) + row * A.cols + column(it), f[k]);
    }
    if (!(A.norms & SR_NORM_BEFORE)) return;
    float by2, inv2;
    inverse(1, [&](int it) {
        if (!HOLD) make(it);
        return HOLD ? it : 0;
    }, by2, inv2);
#pragma unroll
    for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
        const int k = HOLD ? it : 0;
        if (!HOLD) make(it);
        float w[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = 1.0f;
        if (there(it) && A.before) load_weight<VEC>(A.before, column(it), w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[k][i] = there(it) ? f[k][i] * by2 * inv2 * w[i] : 0.0f;
        if constexpr (FMT >= SR_FORMAT_MX8) srx::store_scaled<VEC, FMT>(A, row, column(it), f[k], srx::largest(f[k]), row_there);
        else if (there(it)) srx::store_unit<T, VEC>(static_cast<T*>(A.out) + row * A.cols + column(it), f[k]);
    }
}

template <typename T, int VEC, int HOLD, int FMT>
cudaError_t launch_one(const BlockArgs& A, int tpr, cudaStream_t s)
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
    return cudaLaunchKernelEx(&cfg, sr_block_kernel<T, VEC, HOLD, FMT>, A);
}
template <typename T, int VEC, int FMT>
cudaError_t launch_rows(const BlockArgs& A, cudaStream_t s)
{
    constexpr int FEW = VEC > 1 ? 1 : 8;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols, units = (end + VEC - 1) / VEC;
    int tpr = 32;
    while (tpr < 1024 && (int64_t)tpr * FEW < units) tpr *= 2;
    return (int64_t)tpr * FEW >= units ? launch_one<T, VEC, FEW, FMT>(A, tpr, s) : launch_one<T, VEC, 0, FMT>(A, 1024, s);
}
template <typename T, int VEC>
cudaError_t launch_any(const BlockArgs& A, int fmt, cudaStream_t s)
{
    return fmt == SR_FORMAT_MX4 ? launch_rows<T, VEC, SR_FORMAT_MX4>(A, s) : fmt == SR_FORMAT_MX8 ? launch_rows<T, VEC, SR_FORMAT_MX8>(A, s) : launch_rows<T, VEC, SR_FORMAT_F32>(A, s);
}
template <typename T>
cudaError_t launch(const BlockArgs& A, int fmt, cudaStream_t s)
{
    constexpr int vec = 16 / sizeof(T);
    auto fits = [&](const void* p, int64_t stride) { return !((uintptr_t)p & 15) && (stride % vec == 0 || A.rows < 2); };
    const bool wide = A.cols % vec == 0 && fits(A.y, A.y_stride) && fits(A.residual, A.r_stride) && fits(A.gate, A.gate ? A.g_stride : 0) &&
                      !(((uintptr_t)A.h | (uintptr_t)A.out | (uintptr_t)A.after | (uintptr_t)A.before) & 15);
    return wide ? launch_any<T, vec>(A, fmt, s) : launch_any<T, 1>(A, fmt, s);
}

}  // namespace

extern "C" sr_status sr_block_norm(const sr_block_desc* d, const void* y, const void* residual, const void* gate, const float* after, const float* before, void* h, void* out,
                                   void* scales, void* stream)
{
    constexpr int64_t kMost = (int64_t)1 << 31;
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || (d->norms & ~(SR_NORM_AFTER | SR_NORM_BEFORE)) || d->gate_act < 0 || d->gate_act > 2 || d->rows < 0 ||
        d->cols < 1 || d->rows >= kMost || d->cols >= kMost || d->y_stride < 0 || d->residual_stride < 0 || (gate && d->gate_stride < 0) || !(d->eps >= 0.0f))
        return SR_ERR_INVALID_ARG;
    const bool next = d->norms & SR_NORM_BEFORE, scaled = next && (d->out_format == SR_FORMAT_MX8 || d->out_format == SR_FORMAT_MX4);
    if (next && !scaled && d->out_format != d->dtype) return SR_ERR_INVALID_ARG;
    if (!d->rows) return SR_OK;
    const int el = d->dtype == SR_DTYPE_F32 ? 4 : 2;
    if (!y || !residual || !h || (uintptr_t)y % el || (uintptr_t)residual % el || (uintptr_t)gate % el || (uintptr_t)h % el || (uintptr_t)after % 4 || (uintptr_t)before % 4 ||
        h == y || h == residual || h == gate || (next ? !out || out == y || out == residual || out == gate || out == h : out != nullptr))
        return SR_ERR_INVALID_ARG;
    if (scaled ? !scales || ((uintptr_t)out & 15) || ((uintptr_t)scales & 15) : scales || (uintptr_t)out % el) return SR_ERR_INVALID_ARG;
    BlockArgs A{};
    if (scaled) {
        const SrScaled z = sr_scaled(d->rows, d->cols, d->out_format);
        A.tiles_g = z.tiles_g;
        A.groups = z.groups;
        A.scales = static_cast<uint8_t*>(scales);
    }
    A.y = y;
    A.residual = residual;
    A.gate = gate;
    A.after = after;
    A.before = before;
    A.h = h;
    A.out = out;
    A.rows = d->rows;
    A.cols = d->cols;
    A.y_stride = d->y_stride;
    A.r_stride = d->residual_stride;
    A.g_stride = gate ? d->gate_stride : 0;
    A.scale = d->scale;
    A.eps = d->eps;
    A.norms = d->norms;
    A.act = d->gate_act;
    const int fmt = scaled ? d->out_format : SR_FORMAT_F32;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return (d->dtype == SR_DTYPE_F32 ? launch<float>(A, fmt, s) : launch<__nv_bfloat16>(A, fmt, s)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}
