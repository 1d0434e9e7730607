// Linear attention with a decay for each head:  S_t = exp(g_t) S_{t-1} + k_t v_t^T,  out_t = scale * q_t S_t.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "sr_memory.h"
#include "sr_operators.h"
#include "sr_pair.cuh"
#include "sr_ptx.cuh"

namespace {

// ------------------------------------------------------------------------------------------ whole clips, any sizes
// CUDA cores, everything in 32 bits: fp32 clips, and what the tensor-core kernel does not take (heads of more than 128, rows that TMA cannot copy, a few
// frames).  The same chunks, of 16 frames:  out_i = scale * (exp(G_i) q_i S + sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j),
// S' = exp(G_last) S + sum_j exp(G_last - G_j) k_j v_j^T, so that a state's value costs two fused multiply-adds per frame (q S and k v^T) and one product per chunk.
// A CTA has 64 columns of a group's state: thread (row group, column group) ROWS x 4 values of it in registers, so that a frame's 2 * 4 * ROWS multiply-adds take
// 2 * ROWS / 4 + 1 loads of 16 bytes from shared memory.  Bound by the latency of those in few
// warps (issue slots 31 % used with one CTA to an SM).  500 frames of 5 sequences, 6 heads of 40 and 72 on 3: 72 us; frame by frame, with a column per thread, 320.
// Two CTAs to an SM, 128 registers, where there are more CTAs than SMs, segments always: 512 frames of 32 sequences, 8 heads of 64 248 -> 181 us, 16384 frames, 8 heads
// of 128 755 -> 660; otherwise one, unlimited, since the time is that of one CTA: 512 frames of 16 sequences, 16 heads on 4 of 128 597, with two 800.
// The partial sums of q S over the row groups of a warp are added with a shuffle, those of the warps in shared memory.
constexpr int kFrames = 16, kRunCols = 64, kRunThreads = 256;

template <int DK>
struct FramesShared {
    float k[kFrames][DK], q[kFrames][DK], v[kFrames][kRunCols];
    float part[8][kFrames][kRunCols];
    float p[kFrames][kFrames + 1];                     // weights of the frames before
    double g[kFrames];                                 // log decay since the chunk's start
    float near[kFrames], rest[kFrames];                // exp(G_i), exp(G_last - G_j)
    float whole;                                       // exp(G_last)
};

// DK: rows of the state, padded; MODE as in the tensor-core kernel: 0 whole, 1 sums of segments, 2 their outputs; HELD: CTAs of an SM
template <typename T, int DK, int MODE, int HELD>
__global__ void __launch_bounds__(kRunThreads, HELD) sr_attention_frames_kernel(const __grid_constant__ SegmentArgs C)
{
    constexpr int ROWS = DK / 16;                      // of a thread
    constexpr bool OUT = MODE != 1;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    FramesShared<DK>& M = *reinterpret_cast<FramesShared<DK>*>(smem_raw);
    const AttentionArgs& A = C.A;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const AttentionItem it = attention_item(C, MODE != 0, kRunCols);
    if (!it.there || (MODE == 1 && it.last)) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cg = tid & 15, rg = tid >> 4;
    const int64_t sequence = it.span.b;
    const T* k = static_cast<const T*>(A.k) + sequence * A.sk.sequence + (int64_t)it.g * A.sk.head;
    const T* v = static_cast<const T*>(A.v) + sequence * A.sv.sequence + (int64_t)it.g * A.sv.head + it.c0;
    const float* d = A.decay + sequence * A.sd.sequence + (int64_t)it.g * A.sd.head;
    const int64_t state_at = ((int64_t)it.b * A.groups + it.g) * A.dk, slot_at = ((int64_t)it.slot * A.groups + it.g) * A.dk;
    const int64_t f0 = it.span.first + it.t0;
    const int cols = min(kRunCols, A.dv - it.c0);
    // row r of a thread: neighbouring fours of the row groups lie side by side, so that a warp's two row groups read different banks
    auto row_of = [&](int r) { return (r >> 2) * 64 + rg * 4 + (r & 3); };
    constexpr int R4 = ROWS < 4 ? 1 : ROWS / 4;
    auto row = [&](int r) { return ROWS < 4 ? rg * ROWS + r : row_of(r); };
    // four of a thread's rows of a frame's queries or keys
    auto rows_of = [&](const float* from, int r4, float (&y)[4]) {
        if constexpr (ROWS >= 4) {
            const float4 z = *reinterpret_cast<const float4*>(from + row(4 * r4));
            y[0] = z.x; y[1] = z.y; y[2] = z.z; y[3] = z.w;
        } else {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) y[r] = from[row(r)];
        }
    };
    using srx::Pair;
    using srx::pair;
    Pair S[ROWS][2];
    {
        const float* from = MODE == 1 ? nullptr : MODE == 2 ? C.sums + slot_at * A.dv : A.state_in ? A.state_in + state_at * A.dv : nullptr;
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                float y[2];
#pragma unroll
                for (int z = 0; z < 2; ++z)
                    y[z] = from && row(r) < A.dk && cg * 4 + e + z < cols ? from[(int64_t)row(r) * A.dv + it.c0 + cg * 4 + e + z] : 0.0f;
                S[r][e / 2] = pair(y[0], y[1]);
            }
    }
    double carry = 0.0, log_whole = 0.0;               // (thread 0) what the decays of whole chunks have lost by rounding, relative; the logarithm of all
    const int steps = OUT ? A.share : 1;
    // A chunk's frames are in registers while the one before is worked on.
    const T* q0 = static_cast<const T*>(A.q) + sequence * A.sq.sequence + (int64_t)it.g * A.share * A.sq.head;
    T k_next[ROWS], q_next[ROWS], v_next[4];
    float d_next = 0.0f;
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int x = 0; x < ROWS; ++x) {
            const int t = (tid + x * kRunThreads) / DK, c = (tid + x * kRunThreads) % DK;
            const bool there = t0 + t < it.n && c < A.dk;
            k_next[x] = there ? k[(f0 + t0 + t) * A.sk.frame + c] : (T)0.0f;
            if (OUT) q_next[x] = there ? q0[(f0 + t0 + t) * A.sq.frame + c] : (T)0.0f;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int t = (tid + x * kRunThreads) / kRunCols, c = (tid + x * kRunThreads) % kRunCols;
            v_next[x] = t0 + t < it.n && c < cols ? v[(f0 + t0 + t) * A.sv.frame + c] : (T)0.0f;
        }
        if (warp == 7) d_next = lane < kFrames && t0 + lane < it.n ? d[(f0 + t0 + lane) * A.sd.frame] : 0.0f;
    };
    fetch(0);
    for (int64_t t0 = 0; t0 < it.n; t0 += kFrames) {
        const int n = (int)min((int64_t)kFrames, it.n - t0);
        const int64_t f = f0 + t0;
        __syncthreads();                               // (the chunk before has been read)
#pragma unroll
        for (int x = 0; x < ROWS; ++x) {
            (&M.k[0][0])[tid + x * kRunThreads] = (float)k_next[x];
            if (OUT) (&M.q[0][0])[tid + x * kRunThreads] = (float)q_next[x];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) (&M.v[0][0])[tid + x * kRunThreads] = (float)v_next[x];
        if (warp == 7) {
            float x = d_next;
            if (x < -128.0f) x = -128.0f;              // (exp(-128) is zero in 32 bits; sums of infinities would be NaN)
            double g = (double)x;
#pragma unroll
            for (int m = 1; m < kFrames; m *= 2) {
                const double up = __shfl_up_sync(0xFFFFFFFFu, g, m);
                if (lane >= m) g += up;
            }
            const double last = __shfl_sync(0xFFFFFFFFu, g, kFrames - 1);
            if (lane < kFrames) {
                M.g[lane] = g;
                M.near[lane] = expf((float)g);
                M.rest[lane] = expf((float)(last - g));
            }
            if (lane == 0) {
                const double exact = exp(last) * (1.0 + carry);
                const float rounded = (float)exact;
                M.whole = rounded;
                carry = rounded > 1e-30f ? exact / (double)rounded - 1.0 : 0.0;
                log_whole += last;
            }
        }
        for (int h = 0; h < steps; ++h) {
            if (h > 0) {
                const T* q = q0 + h * A.sq.head;
                for (int x = tid; x < kFrames * DK; x += kRunThreads) {
                    const int t = x / DK, c = x % DK;
                    M.q[t][c] = t < n && c < A.dk ? (float)q[(f + t) * A.sq.frame + c] : 0.0f;
                }
            }
            __syncthreads();
            if (h == 0) fetch(t0 + kFrames);
            if (!OUT) break;
            {   // weights: thread (i, j)
                const int i = tid >> 4, j = tid & 15;
                float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (j <= i) {
#pragma unroll 4
                    for (int c = 0; c < DK; c += 4) {
                        // (every thread starts at another place: rows lie a multiple of 128 bytes apart)
                        const int at = (c + 4 * j) % DK;
                        const float4 a = *reinterpret_cast<const float4*>(&M.q[i][at]), b = *reinterpret_cast<const float4*>(&M.k[j][at]);
                        x[0] = fmaf(a.x, b.x, x[0]);
                        x[1] = fmaf(a.y, b.y, x[1]);
                        x[2] = fmaf(a.z, b.z, x[2]);
                        x[3] = fmaf(a.w, b.w, x[3]);
                    }
                }
                M.p[i][j] = j <= i ? ((x[0] + x[1]) + (x[2] + x[3])) * expf((float)(M.g[i] - M.g[j])) : 0.0f;
            }
#pragma unroll
            for (int t = 0; t < kFrames; ++t) {        // q S over the thread's rows
                Pair o[2] = {0, 0};
#pragma unroll
                for (int r4 = 0; r4 < R4; ++r4) {
                    float y[4];
                    rows_of(&M.q[t][0], r4, y);
#pragma unroll
                    for (int r = 0; r < (ROWS < 4 ? ROWS : 4); ++r) {
                        o[0] = srx::fma2(pair(y[r], y[r]), S[4 * r4 + r][0], o[0]);
                        o[1] = srx::fma2(pair(y[r], y[r]), S[4 * r4 + r][1], o[1]);
                    }
                }
                const float2 o0 = srx::split(o[0]), o1 = srx::split(o[1]);
                float z[4] = {o0.x, o0.y, o1.x, o1.y};
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] += __shfl_xor_sync(0xFFFFFFFFu, z[e], 16);
                if (lane < 16) *reinterpret_cast<float4*>(&M.part[warp][t][cg * 4]) = make_float4(z[0], z[1], z[2], z[3]);
            }
            __syncthreads();
            {   // outputs: thread (frame, four columns)
                const int t = tid >> 4;
                float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const float4 z = *reinterpret_cast<const float4*>(&M.part[w][t][cg * 4]);
                    o[0] += z.x; o[1] += z.y; o[2] += z.z; o[3] += z.w;
                }
                const float near = M.near[t];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] *= near;
                for (int j = 0; j <= t; ++j) {
                    const float p = M.p[t][j];
                    const float4 z = *reinterpret_cast<const float4*>(&M.v[j][cg * 4]);
                    o[0] = fmaf(p, z.x, o[0]);
                    o[1] = fmaf(p, z.y, o[1]);
                    o[2] = fmaf(p, z.z, o[2]);
                    o[3] = fmaf(p, z.w, o[3]);
                }
                if (t < n) {
                    T* out = static_cast<T*>(A.out) + sequence * A.so.sequence + (f + t) * A.so.frame + ((int64_t)it.g * A.share + h) * A.so.head + it.c0;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (cg * 4 + e < cols) out[cg * 4 + e] = (T)(A.scale * o[e]);
                }
            }
            __syncthreads();
        }
        const Pair whole = pair(M.whole, M.whole);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            S[r][0] = srx::mul2(S[r][0], whole);
            S[r][1] = srx::mul2(S[r][1], whole);
        }
#pragma unroll
        for (int t = 0; t < kFrames; ++t) {
            const float w = M.rest[t];
            const float4 z = *reinterpret_cast<const float4*>(&M.v[t][cg * 4]);
            const Pair x0 = srx::mul2(pair(w, w), pair(z.x, z.y)), x1 = srx::mul2(pair(w, w), pair(z.z, z.w));
#pragma unroll
            for (int r4 = 0; r4 < R4; ++r4) {
                float y[4];
                rows_of(&M.k[t][0], r4, y);
#pragma unroll
                for (int r = 0; r < (ROWS < 4 ? ROWS : 4); ++r) {
                    S[4 * r4 + r][0] = srx::fma2(pair(y[r], y[r]), x0, S[4 * r4 + r][0]);
                    S[4 * r4 + r][1] = srx::fma2(pair(y[r], y[r]), x1, S[4 * r4 + r][1]);
                }
            }
        }
    }
    if (MODE == 1 && tid == 7 * 32 && it.c0 == 0) C.decays[(int64_t)it.slot * A.groups + it.g] = (float)exp(log_whole);
    float* to = MODE == 1 ? C.sums + slot_at * A.dv : it.last && A.state_out ? A.state_out + state_at * A.dv : nullptr;
    if (to)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float2 lo = srx::split(S[r][0]), hi = srx::split(S[r][1]);
            const float y[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (row(r) < A.dk && cg * 4 + e < cols) to[(int64_t)row(r) * A.dv + it.c0 + cg * 4 + e] = y[e];
        }
}

template <typename T, int DK, int MODE, int HELD>
cudaError_t launch_frames(const SegmentArgs& C, cudaStream_t s)
{
    constexpr int smem = (int)sizeof(FramesShared<DK>);
    static SrSharedLimit limit;
    const cudaError_t e = limit.raise(sr_attention_frames_kernel<T, DK, MODE, HELD>, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((MODE ? (int64_t)C.slots : (int64_t)C.A.batch) * C.A.groups * C.v_tiles));
    cfg.blockDim = dim3(kRunThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sr_attention_frames_kernel<T, DK, MODE, HELD>, C);
}
template <typename T, int DK>
cudaError_t launch_frames_cut(const SegmentArgs& C, cudaStream_t s)
{
    constexpr int HELD = DK <= 128 ? 2 : 1;
    if (!C.segment && (int64_t)C.A.batch * C.A.groups * C.v_tiles <= sr_device_sms()) return launch_frames<T, DK, 0, 1>(C, s);
    if (!C.segment) return launch_frames<T, DK, 0, HELD>(C, s);
    cudaError_t e = launch_frames<T, DK, 1, HELD>(C, s);
    if (e == cudaSuccess) e = sr_segments_launch(C, s);
    return e == cudaSuccess ? launch_frames<T, DK, 2, HELD>(C, s) : e;
}
template <typename T>
cudaError_t launch_frames_any(const SegmentArgs& C, cudaStream_t s)
{
    if (C.A.dk <= 32) return launch_frames_cut<T, 32>(C, s);
    if (C.A.dk <= 64) return launch_frames_cut<T, 64>(C, s);
    if (C.A.dk <= 128) return launch_frames_cut<T, 128>(C, s);
    return launch_frames_cut<T, 256>(C, s);
}
// Segments for this kernel, by the same reasoning as for the other one: two CTAs to an SM, a piece of 128 frames at least, and about 160 frames' time for the two
// launches more and the states' way.
AttentionCut frames_cut(const sr_attention_desc* d, bool packed, int sms)
{
    AttentionCut cut{0, 0};
    const int64_t per_slot = (int64_t)d->groups * ((d->dv + kRunCols - 1) / kRunCols), held = 2 * std::max(1, sms);
    if (d->batch < 1 || d->frames < 1 || (int64_t)d->batch * d->groups > 65535) return cut;
    const double share = (double)(d->heads / d->groups);
    const double total = packed ? (double)d->frames : (double)d->frames * d->batch, mean = total / d->batch;
    const double longest = packed ? std::min(total, 3.0 * mean) : mean;
    const double waves = (double)(((int64_t)d->batch * per_slot + held - 1) / held);
    const int64_t want = std::max<int64_t>(1, held / per_slot);
    const int64_t each = packed ? (int64_t)(total / (double)want) : (d->frames + std::max<int64_t>(1, want / d->batch) - 1) / std::max<int64_t>(1, want / d->batch);
    const int64_t length = std::max<int64_t>(128, (each + kFrames - 1) / kFrames * kFrames);
    if (length >= d->frames) return cut;
    const int64_t slots = packed ? d->batch + d->frames / length : d->batch * ((d->frames + length - 1) / length);
    const double pieces = packed ? total / (double)length + 0.5 * d->batch : (double)slots;
    if (std::ceil(pieces * (double)per_slot / (double)held) * (double)length * (share + 0.5) + 160.0 > 0.9 * std::max(longest, waves * mean) * share) return cut;
    if (slots * per_slot > 0x7FFFFFFF) return cut;
    cut.segment = length;
    cut.slots = slots;
    return cut;
}

// ------------------------------------------------------------------------------------------ one frame
// Bound by the states: 8 bytes per element, read and written once.  A block of 256 threads has 32 columns of a group's state, so that a row of
// it is a whole line, and few sequences still make many blocks.  VEC columns per thread.  Six blocks to an SM (40 registers): 256 sequences, 16 heads of 128
// 92 us, 5.8 TB/s; with what the compiler takes by itself 104, with eight 110 (spills).
constexpr int kStepCols = 32, kStepHeads = 8;

template <typename T, int VEC, int ROWS>               // ROWS: rows of a thread
__global__ void __launch_bounds__(256, ROWS <= 8 ? 6 : 1) sr_attention_step_kernel(const __grid_constant__ AttentionArgs A)
{
    constexpr int CT = kStepCols / VEC, RL = 256 / CT; // threads per row; rows side by side
    __shared__ float part[kStepHeads][8][kStepCols];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int b = blockIdx.x / A.groups, g = blockIdx.x % A.groups;
    const int tc = threadIdx.x % CT, rl = threadIdx.x / CT, j = blockIdx.y * kStepCols + tc * VEC;
    const bool there = j < A.dv;
    float* state = A.state_out + ((int64_t)b * A.groups + g) * A.dk * A.dv + j;
    float S[ROWS][VEC];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int i = rl + r * RL;
#pragma unroll
        for (int e = 0; e < VEC; ++e) S[r][e] = 0.0f;
        if (there && i < A.dk) {
            if constexpr (VEC == 4) {
                const float4 y = *reinterpret_cast<const float4*>(state + (int64_t)i * A.dv);
                S[r][0] = y.x; S[r][1] = y.y; S[r][2] = y.z; S[r][3] = y.w;
            } else {
                S[r][0] = state[(int64_t)i * A.dv];
            }
        }
    }
    const T* k = static_cast<const T*>(A.k) + (int64_t)b * A.sk.sequence + (int64_t)g * A.sk.head;
    const T* v = static_cast<const T*>(A.v) + (int64_t)b * A.sv.sequence + (int64_t)g * A.sv.head + j;
    const float decay = expf(A.decay[(int64_t)b * A.sd.sequence + (int64_t)g * A.sd.head]);
    float x[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = there ? (float)v[e] : 0.0f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int i = rl + r * RL;
        const float y = i < A.dk ? (float)k[i] : 0.0f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) S[r][e] = fmaf(decay, S[r][e], y * x[e]);
        if (there && i < A.dk) {
            if constexpr (VEC == 4) *reinterpret_cast<float4*>(state + (int64_t)i * A.dv) = make_float4(S[r][0], S[r][1], S[r][2], S[r][3]);
            else state[(int64_t)i * A.dv] = S[r][0];
        }
    }
    for (int h0 = 0; h0 < A.share; h0 += kStepHeads) {
        const int n = min(kStepHeads, A.share - h0);
        for (int h = 0; h < n; ++h) {
            const T* q = static_cast<const T*>(A.q) + (int64_t)b * A.sq.sequence + ((int64_t)g * A.share + h0 + h) * A.sq.head;
            float o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = 0.0f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int i = rl + r * RL;
                const float y = i < A.dk ? (float)q[i] : 0.0f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = fmaf(y, S[r][e], o[e]);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e)
#pragma unroll
                for (int m = CT; m < 32; m *= 2) o[e] += __shfl_xor_sync(0xFFFFFFFFu, o[e], m);
            if ((threadIdx.x & 31) < CT)
#pragma unroll
                for (int e = 0; e < VEC; ++e) part[h][threadIdx.x >> 5][tc * VEC + e] = o[e];
        }
        __syncthreads();
        const int h = threadIdx.x >> 5, c = threadIdx.x & 31, jo = blockIdx.y * kStepCols + c;
        if (h < n && jo < A.dv) {
            float o = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) o += part[h][w][c];
            static_cast<T*>(A.out)[(int64_t)b * A.so.sequence + ((int64_t)g * A.share + h0 + h) * A.so.head + jo] = (T)(A.scale * o);
        }
        __syncthreads();
    }
}

template <typename T, int VEC, int ROWS>
cudaError_t launch_step_rows(const AttentionArgs& A, cudaStream_t s)
{
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(A.batch * A.groups), (unsigned)((A.dv + kStepCols - 1) / kStepCols));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sr_attention_step_kernel<T, VEC, ROWS>, A);
}
template <typename T, int VEC>
cudaError_t launch_step(const AttentionArgs& A, cudaStream_t s)
{
    constexpr int RL = 256 / (kStepCols / VEC);
    const int rows = (A.dk + RL - 1) / RL;
    if (rows <= 2) return launch_step_rows<T, VEC, 2>(A, s);
    if (rows <= 4) return launch_step_rows<T, VEC, 4>(A, s);
    if (rows <= 8) return launch_step_rows<T, VEC, 8>(A, s);
    return launch_step_rows<T, VEC, 32>(A, s);
}
template <typename T>
cudaError_t launch_step_any(const AttentionArgs& A, cudaStream_t s)
{
    return A.dv % 4 == 0 && !((uintptr_t)A.state_out & 15) ? launch_step<T, 4>(A, s) : launch_step<T, 1>(A, s);
}

// ------------------------------------------------------------------------------------------ checks
bool strides_fit(const sr_attention_strides& s) { return s.frame >= 0 && s.sequence >= 0 && s.head >= 0; }

sr_status check(const sr_attention_desc* d)
{
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || d->batch < 0 || d->heads < 1 || d->groups < 1 || d->heads % d->groups ||
        d->dk < 1 || d->dv < 1 || d->frames < 0 || !strides_fit(d->q) || !strides_fit(d->k) || !strides_fit(d->v) || !strides_fit(d->out) ||
        !strides_fit(d->log_decay))
        return SR_ERR_INVALID_ARG;
    if ((int64_t)d->batch * d->groups > 0x7FFFFFFF || d->dv > 65535 * kStepCols ||
        (int64_t)d->batch * d->groups * ((d->dv + kRunCols - 1) / kRunCols) > 0x7FFFFFFF)
        return SR_ERR_INVALID_ARG;
    if (d->dk > 256 || d->heads / d->groups > 128) return SR_ERR_UNSUPPORTED;
    return SR_OK;
}
// (overlaps of other kinds are the caller's to avoid)
bool apart(const void* out, const void* q, const void* k, const void* v) { return !out || (out != q && out != k && out != v); }
bool aligned(const void* p, int dtype) { return !((uintptr_t)p & (dtype == SR_DTYPE_F32 ? 3 : 1)); }

AttentionArgs arguments(const sr_attention_desc* d, const void* q, const void* k, const void* v, const float* decay, void* out)
{
    AttentionArgs A{};
    A.q = q;
    A.k = k;
    A.v = v;
    A.decay = decay;
    A.out = out;
    A.frames = d->frames;
    A.batch = d->batch;
    A.groups = d->groups;
    A.share = d->heads / d->groups;
    A.dk = d->dk;
    A.dv = d->dv;
    A.scale = d->scale;
    A.sq = d->q;
    A.sk = d->k;
    A.sv = d->v;
    A.so = d->out;
    A.sd = d->log_decay;
    return A;
}

}  // namespace

extern "C" {

sr_status sr_linear_attention_workspace_bytes(const sr_attention_desc* d, int packed, size_t* bytes)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!bytes) return SR_ERR_INVALID_ARG;
    // (whether the tensor-core kernel can take the tensors is known when they are)
    const int sms = sr_device_sms();
    *bytes = std::max(sr_chunks_wanted(d) ? sr_cut_bytes(d, sr_chunks_cut(d, packed != 0, sms)) : 0, sr_cut_bytes(d, frames_cut(d, packed != 0, sms)));
    return SR_OK;
}

sr_status sr_linear_attention_plan(const sr_attention_desc* d, int packed, int sms, sr_attention_plan* plan)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!plan || sms < 0) return SR_ERR_INVALID_ARG;
    if (!sms) sms = sr_device_sms();
    if (sms < 1) return SR_ERR_CUDA;
    const bool chunks = sr_chunks_wanted(d);
    const AttentionCut cut = chunks ? sr_chunks_cut(d, packed != 0, sms) : frames_cut(d, packed != 0, sms);
    *plan = sr_attention_plan{chunks ? 128 : kFrames, cut.segment, cut.slots};
    return SR_OK;
}

sr_status sr_linear_attention_run(const sr_attention_desc* d, const void* q, const void* k, const void* v, const float* decay, const int64_t* offsets,
                                  const float* state_in, float* state_out, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if (((uintptr_t)state_in & 3) || ((uintptr_t)state_out & 3) || ((uintptr_t)offsets & 7)) return SR_ERR_INVALID_ARG;
    if (d->frames && (!q || !k || !v || !decay || !out || !aligned(q, d->dtype) || !aligned(k, d->dtype) || !aligned(v, d->dtype) || !aligned(out, d->dtype) ||
                      ((uintptr_t)decay & 3) || !apart(out, q, k, v)))
        return SR_ERR_INVALID_ARG;
    const bool chunks = sr_chunks_wanted(d) && sr_chunks_fit(d, offsets != nullptr, q, k, v);
    const int sms = sr_device_sms();
    const AttentionCut cut = chunks ? sr_chunks_cut(d, offsets != nullptr, sms) : frames_cut(d, offsets != nullptr, sms);
    const size_t needed = sr_cut_bytes(d, cut);
    if (needed && (!workspace || workspace_bytes < needed || ((uintptr_t)workspace & 255))) return SR_ERR_INVALID_ARG;
    AttentionArgs A = arguments(d, q, k, v, decay, out);
    A.offsets = offsets;
    A.state_in = state_in;
    A.state_out = state_out;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (chunks) {
        e = sr_chunks_launch(A, d, cut, workspace, s);
    } else {
        const SegmentArgs C = sr_segment_args(A, cut, kRunCols, workspace);
        e = d->dtype == SR_DTYPE_F32 ? launch_frames_any<float>(C, s) : launch_frames_any<__nv_bfloat16>(C, s);
    }
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_linear_attention_step(const sr_attention_desc* d, const void* q, const void* k, const void* v, const float* decay, float* state, void* out,
                                   void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if (!q || !k || !v || !decay || !state || !out || !aligned(q, d->dtype) || !aligned(k, d->dtype) || !aligned(v, d->dtype) ||
        !aligned(out, d->dtype) || ((uintptr_t)decay & 3) || ((uintptr_t)state & 3) || !apart(out, q, k, v))
        return SR_ERR_INVALID_ARG;
    AttentionArgs A = arguments(d, q, k, v, decay, out);
    A.state_out = state;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d->dtype == SR_DTYPE_F32 ? launch_step_any<float>(A, s) : launch_step_any<__nv_bfloat16>(A, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
