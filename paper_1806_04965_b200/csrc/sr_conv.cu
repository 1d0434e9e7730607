// Causal convolution of every channel over the last frames: out[t, c] = act(bias[c] + sum_j weight[c, j] x[t - (W - 1) + j, c]).
//
// Bound by memory: x once, out once.  A thread has VEC neighbouring channels and goes over a segment of frames with the last W - 1 of them in registers, so that only
// the W - 1 frames ahead of a segment are read twice; eight frames are loaded at a time.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/sr_rollout.h"
#include "sr_operators.h"
#include "sr_pair.cuh"
#include "sr_ptx.cuh"
#include "sr_row.cuh"
#include "sr_selective.cuh"
#include "sr_spans.cuh"

namespace {

struct ConvArgs {
    const void* x;
    const float *weight, *bias;
    const int64_t* offsets;
    const void* state_in;
    void *state_out, *out;
    int64_t frames, segment;
    int32_t batch, channels, act, tiles;               // tiles: CTAs side by side over the channels
    sr_frame_strides sx, so;
};

constexpr int kThreads = 128, kAhead = 8;

template <typename T, int VEC, int W>
struct Taps {
    float w[W][VEC], bias[VEC];
    __device__ __forceinline__ Taps(const ConvArgs& A, int64_t c)
    {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            bias[e] = A.bias ? A.bias[c + e] : 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][e] = A.weight[(c + e) * W + j];
        }
    }
    // seen: W frames, oldest first
    template <typename F>
    __device__ __forceinline__ void apply(const ConvArgs& A, F seen, float (&y)[VEC]) const
    {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                srx::Pair s = srx::pair(bias[e], bias[e + 1]);
#pragma unroll
                for (int j = 0; j < W; ++j) s = srx::fma2(srx::pair(w[j][e], w[j][e + 1]), srx::pair(seen(j)[e], seen(j)[e + 1]), s);
                const float2 v = srx::split(s);
                y[e] = v.x;
                y[e + 1] = v.y;
            }
        } else {
            y[0] = bias[0];
#pragma unroll
            for (int j = 0; j < W; ++j) y[0] = fmaf(w[j][0], seen(j)[0], y[0]);
        }
        if (A.act) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = srx::silu<sizeof(T) == 4>(y[e]);
        }
    }
};

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kThreads) sr_conv_run_kernel(const __grid_constant__ ConvArgs A)
{
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t slot = blockIdx.x / A.tiles;
    int b;
    int64_t seg;
    find_slot(A.offsets, A.frames, A.batch, A.segment, slot, b, seg);
    const int64_t c = ((int64_t)(blockIdx.x % A.tiles) * kThreads + threadIdx.x) * VEC;
    if (b < 0 || c >= A.channels) return;
    const FrameSpan span = frame_span(A.offsets, A.frames, b);
    const int64_t t0 = seg * A.segment, n = min(A.segment, span.n - t0);
    const T* x = static_cast<const T*>(A.x) + span.first * A.sx.frame + span.b * A.sx.sequence + c;
    T* out = static_cast<T*>(A.out) + (span.first + t0) * A.so.frame + span.b * A.so.sequence + c;
    const int64_t old = (int64_t)b * (W - 1) * A.channels + c;       // the sequence's state
    auto frame = [&](int64_t t, float (&f)[VEC]) {     // one of the sequence's, or of its state's
        if (t >= 0) {
            srx::load_unit<T, VEC>(x + t * A.sx.frame, f);
        } else if (A.state_in) {
            srx::load_unit<T, VEC>(static_cast<const T*>(A.state_in) + old + (W - 1 + t) * A.channels, f);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = 0.0f;
        }
    };
    const Taps<T, VEC, W> taps(A, c);
    float seen[W - 1 + kAhead][VEC];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) frame(t0 - (W - 1) + j, seen[j]);
    const T* px = x + t0 * A.sx.frame;
    for (int64_t t = 0; t < n; t += kAhead) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (t + k < n) srx::load_unit<T, VEC>(px, seen[W - 1 + k]);
            px += A.sx.frame;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float y[VEC];
            taps.apply(A, [&](int j) -> const float(&)[VEC] { return seen[k + j]; }, y);
            if (t + k < n) srx::store_unit<T, VEC>(out, y);
            out += A.so.frame;
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e) seen[j][e] = seen[j + kAhead][e];
    }
    // The thread that has read the old state writes the new one, so that they may be the same: place i then holds what frame n - (W - 1) + i was, read from place n + i at
    // the earliest.
    if (seg == 0 && A.state_out) {
        T* to = static_cast<T*>(A.state_out) + old;
        for (int i = 0; i < W - 1; ++i) {
            float f[VEC];
            frame(span.n - (W - 1) + i, f);
            srx::store_unit<T, VEC>(to + (int64_t)i * A.channels, f);
        }
    }
}

template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kThreads) sr_conv_step_kernel(const __grid_constant__ ConvArgs A)
{
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t b = blockIdx.x / A.tiles;
    const int64_t c = ((int64_t)(blockIdx.x % A.tiles) * kThreads + threadIdx.x) * VEC;
    if (c >= A.channels) return;
    T* state = static_cast<T*>(A.state_out) + b * (W - 1) * A.channels + c;
    float seen[W][VEC];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) srx::load_unit<T, VEC>(state + (int64_t)j * A.channels, seen[j]);
    srx::load_unit<T, VEC>(static_cast<const T*>(A.x) + b * A.sx.sequence + c, seen[W - 1]);
    const Taps<T, VEC, W> taps(A, c);
    float y[VEC];
    taps.apply(A, [&](int j) -> const float(&)[VEC] { return seen[j]; }, y);
    srx::store_unit<T, VEC>(static_cast<T*>(A.out) + b * A.so.sequence + c, y);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) srx::store_unit<T, VEC>(state + (int64_t)j * A.channels, seen[j + 1]);
}

template <typename F>
cudaError_t start(F* kernel, int64_t blocks, ConvArgs A, cudaStream_t s)
{
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, A);
}

template <typename T, int VEC, int W>
cudaError_t launch(ConvArgs A, bool step, cudaStream_t s)
{
    A.tiles = (int32_t)((A.channels + (int64_t)kThreads * VEC - 1) / (kThreads * VEC));
    if (step) return start(sr_conv_step_kernel<T, VEC, W>, (int64_t)A.batch * A.tiles, A, s);
    A.segment = 32;
    const int64_t slots = A.offsets ? A.frames / A.segment + A.batch : A.batch * segments_of(A.frames, A.segment);
    return start(sr_conv_run_kernel<T, VEC, W>, slots * A.tiles, A, s);
}
template <typename T, int VEC>
cudaError_t launch(const ConvArgs& A, int width, bool step, cudaStream_t s)
{
    switch (width) {
        case 1: return launch<T, VEC, 1>(A, step, s);
        case 2: return launch<T, VEC, 2>(A, step, s);
        case 3: return launch<T, VEC, 3>(A, step, s);
        case 4: return launch<T, VEC, 4>(A, step, s);
        case 5: return launch<T, VEC, 5>(A, step, s);
        case 6: return launch<T, VEC, 6>(A, step, s);
        case 7: return launch<T, VEC, 7>(A, step, s);
        default: return launch<T, VEC, 8>(A, step, s);
    }
}
// 16 bytes at a time where every row of every tensor allows it.
template <typename T>
cudaError_t launch(const ConvArgs& A, int width, bool step, cudaStream_t s)
{
    constexpr int vec = 16 / sizeof(T);
    auto fits = [&](const void* p, const sr_frame_strides& st) {
        return !((uintptr_t)p & 15) && (step || st.frame % vec == 0) && (A.offsets || A.batch < 2 || st.sequence % vec == 0);
    };
    const bool wide = A.channels % vec == 0 && fits(A.x, A.sx) && fits(A.out, A.so) && !(((uintptr_t)A.state_in | (uintptr_t)A.state_out) & 15);
    return wide ? launch<T, vec>(A, width, step, s) : launch<T, 1>(A, width, step, s);
}

sr_status check(const sr_conv_desc* d)
{
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || d->batch < 0 || d->channels < 1 || d->width < 1 || d->frames < 0 || (d->act != 0 && d->act != 1) ||
        d->x.frame < 0 || d->x.sequence < 0 || d->out.frame < 0 || d->out.sequence < 0)
        return SR_ERR_INVALID_ARG;
    return d->width > 8 ? SR_ERR_UNSUPPORTED : SR_OK;
}
bool aligned(const void* p, int dtype) { return !((uintptr_t)p & (dtype == SR_DTYPE_F32 ? 3 : 1)); }

sr_status call(const sr_conv_desc* d, const void* x, const float* weight, const float* bias, const int64_t* offsets, const void* state_in, void* state_out, void* out,
               bool step, cudaStream_t s)
{
    if (!x || !weight || !out || !aligned(x, d->dtype) || !aligned(out, d->dtype) || ((uintptr_t)weight & 3) || ((uintptr_t)bias & 3) || out == x) return SR_ERR_INVALID_ARG;
    ConvArgs A{};
    A.x = x;
    A.weight = weight;
    A.bias = bias;
    A.offsets = offsets;
    A.state_in = d->width > 1 ? state_in : nullptr;
    A.state_out = d->width > 1 ? state_out : nullptr;
    A.out = out;
    A.frames = d->frames;
    A.batch = d->batch;
    A.channels = d->channels;
    A.act = d->act;
    A.sx = d->x;
    A.so = d->out;
    return (d->dtype == SR_DTYPE_F32 ? launch<float>(A, d->width, step, s) : launch<__nv_bfloat16>(A, d->width, step, s)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // namespace

extern "C" {

sr_status sr_causal_conv_run(const sr_conv_desc* d, const void* x, const float* weight, const float* bias, const int64_t* offsets, const void* state_in, void* state_out,
                             void* out, void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if (!aligned(state_in, d->dtype) || !aligned(state_out, d->dtype) || ((uintptr_t)offsets & 7)) return SR_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!d->frames) {                                  // (there need not be any tensors then)
        const size_t bytes = (size_t)d->batch * (d->width - 1) * d->channels * (d->dtype == SR_DTYPE_F32 ? 4 : 2);
        if (!state_out || !bytes || state_in == state_out) return SR_OK;
        const cudaError_t e = state_in ? cudaMemcpyAsync(state_out, state_in, bytes, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(state_out, 0, bytes, s);
        return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
    }
    return call(d, x, weight, bias, offsets, state_in, state_out, out, false, s);
}

sr_status sr_causal_conv_step(const sr_conv_desc* d, const void* x, const float* weight, const float* bias, void* state, void* out, void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if ((!state && d->width > 1) || !aligned(state, d->dtype)) return SR_ERR_INVALID_ARG;
    return call(d, x, weight, bias, nullptr, nullptr, state, out, true, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
