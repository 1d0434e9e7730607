// Causal convolution of every channel over the last frames: out[t, c] = act(bias[c] + sum_j weight[c, j] x[t - (W - 1) + j, c]).
//
// Bound by memory: x once, out once.  A thread has VEC neighbouring channels and goes over a segment of frames with the last W - 1 of them in registers, so that only
// the W - 1 frames ahead of a segment are read twice.  Units of 16 bytes come through a ring in shared memory that is the thread's own, so that nothing waits for others; narrower
// ones through registers, the next eight under way while eight are worked on.  64 sequences of 128 frames, 4096 channels, four taps, bf16: 30 us (4.6 TB/s), 26 without the
// activation, 512 frames 94 (5.7 TB/s): beginning and end of a launch, and the activation's exponentials and reciprocals (15 us of the special function units).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

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

constexpr int kThreads = 128, kRing = 3;
// Frames that a thread loads at a time, and batches of them: in its ring in shared memory (16-byte units), or two in registers.
__host__ __device__ constexpr int ahead_of(int bytes) { return bytes == 16 ? 4 : 8; }

// The weights of a thread's channels.  VEC > 1: through shared memory, where a thread's units of 16 bytes lie an odd number of them from the next thread's; read straight from
// global memory every load would touch as many lines as there are lanes (64 sequences of 128 frames, 4096 channels, four taps: 64 us).
template <typename T, int VEC, int W>
struct Taps {
    static constexpr int UNITS = VEC * W / 4, STRIDE = UNITS | 1, SHARED = VEC > 2 ? kThreads * STRIDE : 1;
    float w[W][VEC], bias[VEC];
    __device__ __forceinline__ void get(const ConvArgs& A, int64_t c0, float4* shared)          // c0: the block's first channel
    {
        const int64_t c = c0 + (int64_t)threadIdx.x * VEC;
        const bool there = c < A.channels;
        if constexpr (VEC > 2) {
            const int units = (int)min((int64_t)kThreads * UNITS, (A.channels - c0) * W / 4);      // (VEC > 2: the channels are a multiple of 4)
            const float4* from = reinterpret_cast<const float4*>(A.weight + c0 * W);
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                const int m = i * kThreads + threadIdx.x;
                if (m < units) shared[m / UNITS * STRIDE + m % UNITS] = from[m];
            }
            __syncthreads();
            float flat[VEC * W];
#pragma unroll
            for (int i = 0; i < UNITS; ++i) *reinterpret_cast<float4*>(&flat[4 * i]) = shared[threadIdx.x * STRIDE + i];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
#pragma unroll
                for (int j = 0; j < W; ++j) w[j][e] = flat[e * W + j];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
#pragma unroll
                for (int j = 0; j < W; ++j) w[j][e] = there ? A.weight[(c + e) * W + j] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) bias[e] = there && A.bias ? A.bias[c + e] : 0.0f;
    }
    // seen: the last W frames, oldest first
    __device__ __forceinline__ void apply(bool act, const float (&seen)[W][VEC], float (&y)[VEC]) const
    {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                srx::Pair s = srx::pair(bias[e], bias[e + 1]);
#pragma unroll
                for (int j = 0; j < W; ++j) s = srx::fma2(srx::pair(w[j][e], w[j][e + 1]), srx::pair(seen[j][e], seen[j][e + 1]), s);
                if (act) s = srx::silu<sizeof(T) == 4>(s);
                const float2 v = srx::split(s);
                y[e] = v.x;
                y[e + 1] = v.y;
            }
        } else {
            y[0] = bias[0];
#pragma unroll
            for (int j = 0; j < W; ++j) y[0] = fmaf(w[j][0], seen[j][0], y[0]);
            if (act) y[0] = srx::silu<sizeof(T) == 4>(y[0]);
        }
    }
};
// `next` becomes the last of W frames.
template <typename T, int VEC, int W>
__device__ __forceinline__ void see(float (&seen)[W][VEC], const srx::Few<T, VEC>& next)
{
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) seen[j][e] = seen[j + 1][e];
#pragma unroll
    for (int e = 0; e < VEC; ++e) seen[W - 1][e] = next[e];
}

// Single values: eight blocks to an SM, six of more than four taps (16 packed sequences, 1111 channels, three taps, fp32: 16.4 us, with as many registers as wanted 17.9).
// Four blocks as long as weights and frames of units all but fit 128 registers (24 bytes of spills with four and five taps): with eight channels up to five taps (64 sequences of 128 frames,
// 4096 channels, eight taps: 44 us with two blocks, 139 with four; six taps 37 and 46).
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(kThreads, VEC * sizeof(T) == 16 ? (VEC * W > 40 ? 2 : 4) : W > 4 ? 6 : 8) sr_conv_run_kernel(const __grid_constant__ ConvArgs A)
{
    using srx::Few;
    constexpr int kAhead = ahead_of(VEC * (int)sizeof(T));
    __shared__ float4 shared[Taps<T, VEC, W>::SHARED];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t slot = blockIdx.x / A.tiles;
    int b;
    int64_t seg;
    if (A.offsets) packed_slot(A.offsets, A.frames, A.batch, A.segment, slot, b, seg);
    else find_slot(nullptr, A.frames, A.batch, A.segment, slot, b, seg);
    if (b < 0) return;
    const int64_t c0 = (int64_t)(blockIdx.x % A.tiles) * kThreads * VEC, c = c0 + threadIdx.x * VEC;
    const FrameSpan span = frame_span(A.offsets, A.frames, b);
    const int64_t t0 = seg * A.segment, n = min(A.segment, span.n - t0);
    if (span.n == 0 && !A.state_out) return;
    Taps<T, VEC, W> taps;
    taps.get(A, c0, shared);
    if (c >= A.channels) return;
    const T* x = static_cast<const T*>(A.x) + span.first * A.sx.frame + span.b * A.sx.sequence + c;
    T* out = static_cast<T*>(A.out) + (span.first + t0) * A.so.frame + span.b * A.so.sequence + c;
    const int64_t old = (int64_t)b * (W - 1) * A.channels + c;       // the sequence's state
    auto frame = [&](int64_t t, Few<T, VEC>& f) {      // one of the sequence's, or of its state's
        if (t >= 0) {
            f.get(x + t * A.sx.frame);
        } else if (A.state_in) {
            f.get(static_cast<const T*>(A.state_in) + old + (W - 1 + t) * A.channels);
        } else {
#pragma unroll
            for (int e = 0; e < Few<T, VEC>::WORDS; ++e) f.w[e] = 0;
        }
    };
    float seen[W][VEC] = {};
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        Few<T, VEC> f;
        frame(t0 - (W - 1) + j, f);
        see<T, VEC, W>(seen, f);
    }
    // kAhead frames at a time: of 16-byte units kRing - 1 times as many are on their way to places in shared memory that are the thread's own, of others as many in registers
    constexpr bool ASYNC = VEC * sizeof(T) == 16;
    constexpr int UNIT = VEC * (int)sizeof(T);
    extern __shared__ __align__(16) uint8_t memory[];
    uint8_t* mine = memory + threadIdx.x * UNIT;
    Few<T, VEC> next[ASYNC ? 1 : kAhead], held[ASYNC ? 1 : kAhead];
    const T* px = x + t0 * A.sx.frame;
    auto load = [&](int64_t t, int place) {            // the kAhead frames from t on
        const int there = (int)min(n - t, (int64_t)kAhead);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (k < there) {
                if constexpr (ASYNC) srx::copy_16(mine + (place * kAhead + k) * kThreads * UNIT, px + k * A.sx.frame);
                else next[k].get(px + k * A.sx.frame);
            }
        }
        px += kAhead * A.sx.frame;
        if (ASYNC) asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto work = [&](auto usual, int left, int place) { // usual: all kAhead frames, with their activation
        constexpr bool USUAL = decltype(usual)::value;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            Few<T, VEC> in;
            if constexpr (ASYNC) in.get(reinterpret_cast<const T*>(mine + (place * kAhead + k) * kThreads * UNIT));
            else in = held[k];
            see<T, VEC, W>(seen, in);
            float y[VEC];
            taps.apply(USUAL || A.act, seen, y);
            Few<T, VEC> o;
            o.set(y);
            if (USUAL || k < left) o.put(out + k * A.so.frame);
        }
    };
    constexpr int RING = ASYNC ? kRing : 1;
#pragma unroll
    for (int i = 0; i < (ASYNC ? RING - 1 : 1); ++i) load(i * kAhead, i);
    int place = 0;
    for (int64_t t = 0; t < n; t += kAhead) {
        if constexpr (!ASYNC) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) held[k] = next[k];
            if (t + kAhead < n) load(t + kAhead, 0);
        }
        if constexpr (ASYNC) {
            load(t + (RING - 1) * kAhead, place ? place - 1 : RING - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
        }
        const int left = (int)min(n - t, (int64_t)kAhead);
        if (left == kAhead && A.act) work(std::true_type{}, left, place);
        else work(std::false_type{}, left, place);
        out += kAhead * A.so.frame;
        place = place + 1 == RING ? 0 : place + 1;
    }
    // The thread that has read the old state writes the new one, so that they may be the same: place i then holds what frame n - (W - 1) + i was, read from place n + i at
    // the earliest.
    if (seg == 0 && A.state_out) {
        T* to = static_cast<T*>(A.state_out) + old;
        for (int i = 0; i < W - 1; ++i) {
            Few<T, VEC> f;
            frame(span.n - (W - 1) + i, f);
            f.put(to + (int64_t)i * A.channels);
        }
    }
}

// A thread goes over SEQ sequences with the same weights.
template <typename T, int VEC, int W, int SEQ>
__global__ void __launch_bounds__(kThreads) sr_conv_step_kernel(const __grid_constant__ ConvArgs A)
{
    using srx::Few;
    __shared__ float4 shared[Taps<T, VEC, W>::SHARED];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t b0 = (int64_t)(blockIdx.x / A.tiles) * SEQ;
    const int64_t c0 = (int64_t)(blockIdx.x % A.tiles) * kThreads * VEC, c = c0 + threadIdx.x * VEC;
    const bool there = c < A.channels;
    Few<T, VEC> in[SEQ][W];
#pragma unroll
    for (int s = 0; s < SEQ; ++s) {
        if (!there || b0 + s >= A.batch) continue;
        const T* state = static_cast<const T*>(A.state_out) + (b0 + s) * (W - 1) * A.channels + c;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) in[s][j].get(state + (int64_t)j * A.channels);
        in[s][W - 1].get(static_cast<const T*>(A.x) + (b0 + s) * A.sx.sequence + c);
    }
    Taps<T, VEC, W> taps;
    taps.get(A, c0, shared);
#pragma unroll
    for (int s = 0; s < SEQ; ++s) {
        if (!there || b0 + s >= A.batch) continue;
        float y[VEC], seen[W][VEC];
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e) seen[j][e] = in[s][j][e];
        taps.apply(A.act, seen, y);
        Few<T, VEC> o;
        o.set(y);
        o.put(static_cast<T*>(A.out) + (b0 + s) * A.so.sequence + c);
        T* state = static_cast<T*>(A.state_out) + (b0 + s) * (W - 1) * A.channels + c;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) in[s][j + 1].put(state + (int64_t)j * A.channels);
    }
}

template <typename F>
cudaError_t start(F* kernel, int64_t blocks, int shared, ConvArgs A, cudaStream_t s)
{
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)shared;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, A);
}

template <typename T, int VEC, int W>
cudaError_t launch(ConvArgs A, bool step, cudaStream_t s)
{
    constexpr bool RUNS = VEC == 1 || VEC * sizeof(T) == 16, STEPS = VEC * sizeof(T) < 16;
    A.tiles = (int32_t)((A.channels + (int64_t)kThreads * VEC - 1) / (kThreads * VEC));
    const int sms = sr_device_sms();
    if constexpr (STEPS) {
        if (step) {
            if (A.batch >= 32) return start(sr_conv_step_kernel<T, VEC, W, 4>, (A.batch + 3) / 4 * (int64_t)A.tiles, 0, A, s);
            return start(sr_conv_step_kernel<T, VEC, W, 1>, (int64_t)A.batch * A.tiles, 0, A, s);
        }
    }
    if constexpr (RUNS) {
        // as long segments as leave three blocks to an SM (64 sequences of 128 frames, 4096 channels: 29.9 us with 64 frames, 30.2 with 32, 31.3 with 16)
        A.segment = 64;
        while (A.segment > 8 && (A.offsets ? A.frames / A.segment : A.batch * segments_of(A.frames, A.segment)) * A.tiles < 3 * sms) A.segment /= 2;
        const int64_t slots = A.offsets ? A.frames / A.segment + A.batch : A.batch * segments_of(A.frames, A.segment);
        constexpr int bytes = VEC * sizeof(T) == 16 ? kRing * ahead_of(16) * kThreads * VEC * (int)sizeof(T) : 0;
        static SrSharedLimit limit;
        const cudaError_t e = bytes ? limit.raise(sr_conv_run_kernel<T, VEC, W>, bytes) : cudaSuccess;
        return e == cudaSuccess ? start(sr_conv_run_kernel<T, VEC, W>, slots * A.tiles, bytes, A, s) : e;
    }
    return cudaErrorInvalidValue;
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
// 16 bytes at a time where every row of every tensor allows it.  Single frames: 8 bytes, for more threads (256 sequences of 4096 channels 4.6 us, with 16 bytes 5.3), and where there
// are few sequences pairs of bf16 (one of 4096 channels 1.6, with 16 bytes 2.1).
template <typename T>
cudaError_t launch(const ConvArgs& A, int width, bool step, cudaStream_t s)
{
    constexpr int vec = 16 / sizeof(T);
    auto fits = [&](int vec) {
        auto lies = [&](const void* p, const sr_frame_strides& st) {
            return (uintptr_t)p % (vec * sizeof(T)) == 0 && (step || st.frame % vec == 0) && (A.offsets || A.batch < 2 || st.sequence % vec == 0);
        };
        return A.channels % vec == 0 && lies(A.x, A.sx) && lies(A.out, A.so) && ((uintptr_t)A.state_in | (uintptr_t)A.state_out) % (vec * sizeof(T)) == 0;
    };
    if constexpr (sizeof(T) == 2) {
        if (step && (int64_t)A.batch * A.channels <= (int64_t)sr_device_sms() * kThreads * 4 && fits(2)) return launch<T, 2>(A, width, step, s);
    }
    if (step && !((uintptr_t)A.weight & 15) && fits(vec / 2)) return launch<T, vec / 2>(A, width, step, s);
    return !step && !((uintptr_t)A.weight & 15) && fits(vec) ? launch<T, vec>(A, width, step, s) : launch<T, 1>(A, width, step, s);
}

sr_status check(const sr_conv_desc* d)
{
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || d->batch < 0 || d->batch > kMostSequences || d->channels < 1 || d->width < 1 ||
        d->frames < 0 || (d->act != 0 && d->act != 1) || d->x.frame < 0 || d->x.sequence < 0 || d->out.frame < 0 || d->out.sequence < 0)
        return SR_ERR_INVALID_ARG;
    if ((double)d->frames * d->channels > 0x1p45 || (double)d->batch * d->channels * d->width > 0x1p45) return SR_ERR_INVALID_ARG;          // (no memory holds them)
    return d->width > 8 ? SR_ERR_UNSUPPORTED : SR_OK;
}
bool aligned(const void* p, int dtype) { return !((uintptr_t)p & (dtype == SR_DTYPE_F32 ? 3 : 1)); }

sr_status call(const sr_conv_desc* d, const void* x, const float* weight, const float* bias, const int64_t* offsets, const void* state_in, void* state_out, void* out,
               bool step, cudaStream_t s)
{
    if (!x || !weight || !out || !aligned(x, d->dtype) || !aligned(out, d->dtype) || ((uintptr_t)weight & 3) || ((uintptr_t)bias & 3) || out == x ||
        frames_overlap(d->out.frame, d->out.sequence, step ? 1 : d->frames, offsets ? 1 : d->batch, d->channels))
        return SR_ERR_INVALID_ARG;
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
