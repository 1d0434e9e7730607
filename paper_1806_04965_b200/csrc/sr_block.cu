// The way out of a block and into the next one, one pass over rows:
//
//     h = residual + scale * act(gate) * rms(y) * weight_after,   out = rms(h) * weight_before,   rms(x) = x / sqrt(mean(x^2) + eps).
//
// Bound by memory: y, residual and gate in, h and out out, each once.  A row lies in the registers of the threads that share it through both reductions, y turned
// into h in place.  Blocks go over many rows, with the weights in registers and the next row's loads under way while one is worked on.  Longer rows are read again (out of L2).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "sr_microscale.cuh"
#include "sr_operators.h"
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

using srx::Few;
using srx::Pair;

struct Times {
    __device__ __forceinline__ float operator()(float a, float b) const { return a * b; }
    __device__ __forceinline__ Pair operator()(Pair a, Pair b) const { return srx::mul2(a, b); }
};
struct By {
    float s;
    __device__ __forceinline__ float operator()(float a) const { return a * s; }
    __device__ __forceinline__ Pair operator()(Pair a) const { return srx::mul2(a, srx::pair(s, s)); }
};
struct TimesPlus {
    __device__ __forceinline__ float operator()(float a, float b, float c) const { return fmaf(a, b, c); }
    __device__ __forceinline__ Pair operator()(Pair a, Pair b, Pair c) const { return srx::fma2(a, b, c); }
};
template <bool EXACT>
struct Sigmoid {
    template <typename X>
    __device__ __forceinline__ X operator()(X x) const { return srx::sigmoid<EXACT>(x); }
};
template <bool EXACT>
struct Silu {
    template <typename X>
    __device__ __forceinline__ X operator()(X x) const { return srx::silu<EXACT>(x); }
};

// to = what(x, ...), element by element, two at a time where there are two.
template <int VEC, typename F, typename... X>
__device__ __forceinline__ void each_pair(F what, float (&to)[VEC], const X (&... x)[VEC])
{
    if constexpr (VEC == 1) {
        to[0] = what(x[0]...);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
            const float2 v = srx::split(what(srx::pair(x[i], x[i + 1])...));
            to[i] = v.x;
            to[i + 1] = v.y;
        }
    }
}

constexpr int kMostThreads = 512;                      // of a row: 128 registers each

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
__global__ void __launch_bounds__(kMostThreads) sr_block_kernel(const __grid_constant__ BlockArgs A)
{
    constexpr int H = HOLD ? HOLD : 1;
    constexpr bool EXACT = sizeof(T) == 4;
    __shared__ __align__(16) float part[2][2][32];                   // by reduction, and by row in turn: threads that are a row ahead do not touch what others still read
    int turn = 0;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int tpr = blockDim.x, tid = threadIdx.x;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols;
    const int n_it = HOLD ? HOLD : (int)((end + (int64_t)tpr * VEC - 1) / ((int64_t)tpr * VEC));
    // Unit `it` of a thread: of HOLD in a row a warp has all neighbouring ones, a fixed distance apart; of more it comes around with all threads.
    constexpr int NEXT = 32 * VEC;
    const int lane = tid & 31;
    const uint32_t at0 = HOLD ? (uint32_t)(tid >> 5) * (NEXT * H) + lane * VEC : (uint32_t)tid * VEC, around = (uint32_t)tpr * VEC;
    auto away = [&](int it) { return HOLD ? (uint32_t)(it * NEXT) : it * around; };
    auto column = [&](int it) { return at0 + away(it); };
    const uint32_t cols = (uint32_t)A.cols, have = at0 < cols ? cols - at0 : 0u;    // (31 bits)
    const int64_t rows_apart = (int64_t)gridDim.x * blockDim.y;
    int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    bool live = row < A.rows;
    auto there = [&](int it) { return away(it) < (live ? have : 0u); };

    float f[H][VEC];
    Few<T, VEC> yy[H], rr[H], gg[H];                   // the next row, and from its turn on this one's residual and gate
    const T *py, *pr, *pg;                             // the row that is loaded next
    auto to_row = [&](int64_t at) {
        py = static_cast<const T*>(A.y) + at * A.y_stride + at0;
        pr = static_cast<const T*>(A.residual) + at * A.r_stride + at0;
        pg = static_cast<const T*>(A.gate) + at * A.g_stride + at0;
    };
    auto load = [&](bool is, int it, int k) {
        if (!is) return;
        yy[k].get(py + away(it));
        rr[k].get(pr + away(it));
        if (A.gate) gg[k].get(pg + away(it));
    };
    auto weight = [&](const float* w, int it, float scale, float (&to)[VEC]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) to[i] = 1.0f;
        if (w && away(it) < have) load_weight<VEC>(w, column(it), to);
#pragma unroll
        for (int i = 0; i < VEC; ++i) to[i] *= scale;
    };
    float wa[H][VEC], wb[H][VEC];
    to_row(row);
    if (HOLD) {
#pragma unroll
        for (int k = 0; k < H; ++k) load(there(k), k, k);
#pragma unroll
        for (int k = 0; k < H; ++k) {
            weight(A.norms & SR_NORM_AFTER ? A.after : nullptr, k, A.scale, wa[k]);
            weight(A.before, k, 1.0f, wb[k]);
        }
    }
    const int warps = tpr >> 5;                        // of a row
    if (warps > 1 && tid < 64) part[tid >> 5][0][tid & 31] = part[tid >> 5][1][tid & 31] = 0.0f;
    if (warps > 1) __syncthreads();
    auto over_row = [&](float mine, int which, auto join) {       // over the row's threads; 0 joins nothing
#pragma unroll
        for (int d = 16; d; d /= 2) mine = join(mine, __shfl_xor_sync(0xFFFFFFFFu, mine, d));
        if (warps > 1) {                               // (one row per block)
            float(&of)[32] = part[which][turn];
            if (!(tid & 31)) of[tid >> 5] = mine;
            __syncthreads();
            const float4 v = *reinterpret_cast<const float4*>(of);
            mine = join(join(v.x, v.y), join(v.z, v.w));
            for (int w = 4; w < warps; w += 4) {
                const float4 v = *reinterpret_cast<const float4*>(of + w);
                mine = join(mine, join(join(v.x, v.y), join(v.z, v.w)));
            }
        }
        return mine;
    };
    // 1 / sqrt(mean(x^2) + eps) of the row that `unit` brings into f, as two factors: by is a power of two, 1 but where squares leave the range of 32 bits
    auto inverse = [&](int which, auto unit, float& by, float& inv) {
        auto add = [](float a, float b) { return a + b; };
        float ss = 0.0f;
        Pair s2 = srx::pair(0.0f, 0.0f);
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
            const int k = unit(it);
            if constexpr (VEC > 1) {
#pragma unroll
                for (int i = 0; i < VEC; i += 2) s2 = srx::fma2(srx::pair(f[k][i], f[k][i + 1]), srx::pair(f[k][i], f[k][i + 1]), s2);
            } else {
                ss = fmaf(f[k][0], f[k][0], ss);
            }
        }
        const float2 s = srx::split(s2);
        ss = over_row(ss + (s.x + s.y), which, add);
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
    // All threads of a block go around equally often: rows behind the last one are worked on as zeros.
    for (int64_t row0 = (int64_t)blockIdx.x * blockDim.y; row0 < A.rows; row0 += rows_apart, row += rows_apart, live = row < A.rows, turn ^= 1) {
        Few<T, VEC> res[H], gate[H];
        auto widen = [&](int it, int k) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[k][i] = there(it) ? yy[k][i] : 0.0f;
            res[k] = rr[k];
            gate[k] = gg[k];
        };
        if (HOLD) {
            const uint32_t next = row + rows_apart < A.rows ? have : 0u;
            to_row(row + rows_apart);
#pragma unroll
            for (int k = 0; k < H; ++k) {
                widen(k, k);
                load(away(k) < next, k, k);
            }
        } else {
            to_row(row);
        }
        auto bring = [&](int it) {                     // (rows that are read again)
            load(there(it), it, 0);
            widen(it, 0);
        };
        T* ph = static_cast<T*>(A.h) + row * A.cols + at0;
        T* po = static_cast<T*>(A.out) + row * A.cols + at0;
        float by = 1.0f, inv = 1.0f;
        if (A.norms & SR_NORM_AFTER)
            inverse(0, [&](int it) {
                if (!HOLD) bring(it);
                return HOLD ? it : 0;
            }, by, inv);
        // f[k] times by and inv, by being 1 for nearly all rows
        auto norm = [&](int k, float by, float inv) {
            if (by != 1.0f) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[k][i] *= by;
            }
            each_pair(By{inv}, f[k], f[k]);
        };
        // y in f[k] becomes h
        auto join = [&](int it, int k) {
            if (!there(it)) return;
            if (!HOLD) weight(A.norms & SR_NORM_AFTER ? A.after : nullptr, it, A.scale, wa[k]);
            norm(k, by, inv);
            float g[VEC];
            if (A.gate) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = gate[k][i];
                if (A.act == 1) each_pair(Sigmoid<EXACT>{}, g, g);
                if (A.act == 2) each_pair(Silu<EXACT>{}, g, g);
                each_pair(Times{}, g, g, wa[k]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = wa[k][i];
            }
            float r[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) r[i] = res[k][i];
            each_pair(TimesPlus{}, f[k], f[k], g, r);
        };
        auto make = [&](int it) {
            bring(it);
            join(it, 0);
        };
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
            const int k = HOLD ? it : 0;
            if (HOLD) join(it, k);
            else make(it);
            if (there(it)) srx::store_unit<T, VEC>(ph + away(it), f[k]);
        }
        if (!(A.norms & SR_NORM_BEFORE)) continue;
        float by2, inv2;
        inverse(1, [&](int it) {
            if (!HOLD) make(it);
            return HOLD ? it : 0;
        }, by2, inv2);
#pragma unroll
        for (int it = 0; it < (HOLD ? HOLD : n_it); ++it) {
            const int k = HOLD ? it : 0;
            if (!HOLD) {
                make(it);
                weight(A.before, it, 1.0f, wb[k]);
            }
            norm(k, by2, inv2);
            each_pair(Times{}, f[k], f[k], wb[k]);
            if (FMT >= SR_FORMAT_MX8 && !there(it)) {          // (whatever the row holds)
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[k][i] = 0.0f;
            }
            if constexpr (FMT >= SR_FORMAT_MX8) srx::store_scaled<VEC, FMT>(A, row, column(it), f[k], srx::largest(f[k]), live);
            else if (there(it)) srx::store_unit<T, VEC>(po + away(it), f[k]);
        }
    }
}

template <typename T, int VEC, int HOLD, int FMT>
cudaError_t launch_one(const BlockArgs& A, int tpr, cudaStream_t s)
{
    const int rpb = tpr == 32 ? 4 : 1, threads = tpr * rpb;
    static std::atomic<int> known[64][8];              // blocks that an SM takes, by device and threads
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return cudaErrorNoDevice;
    int size = 0;
    while (threads > 64 << size) ++size;
    int fit = dev < 64 ? known[dev][size].load(std::memory_order_relaxed) : 0;
    if (!fit) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, sr_block_kernel<T, VEC, HOLD, FMT>, threads, 0);
        if (e != cudaSuccess) return e;
        fit = std::max(fit, 1);
        if (dev < 64) known[dev][size].store(fit, std::memory_order_relaxed);
    }
    const int64_t blocks = std::min((A.rows + rpb - 1) / rpb, (int64_t)sr_device_sms() * fit);
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
// Two units of 16 bytes to a thread, whose part in a row's reductions is then the smaller (16384 x 2048 bf16 54.9 us, with one 79); one where each SM has a row at most and the
// time is that of a row (8 x 1024 2.2 us, with two 2.6).  Single values, eight: 8192 x 1999 bf16 68 us, with four 109.
template <typename T, int VEC, int FMT>
cudaError_t launch_rows(const BlockArgs& A, cudaStream_t s)
{
    constexpr int FEW = VEC > 1 ? 1 : 8, MANY = VEC > 1 ? 2 : 8;
    const int64_t end = FMT >= SR_FORMAT_MX8 ? A.tiles_g * 128 : A.cols, units = (end + VEC - 1) / VEC;
    for (const int hold : {FEW, MANY}) {
        if (hold != MANY && A.rows > sr_device_sms()) continue;
        int tpr = 32;
        while (tpr < kMostThreads && (int64_t)tpr * hold < units) tpr *= 2;
        if ((int64_t)tpr * hold >= units) return hold == FEW ? launch_one<T, VEC, FEW, FMT>(A, tpr, s) : launch_one<T, VEC, MANY, FMT>(A, tpr, s);
    }
    return launch_one<T, VEC, 0, FMT>(A, kMostThreads, s);
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
