// Selective scan: per channel i and state n    h <- exp(r a[i, n]) h + r u b[n],    out = (sum_n c[n] h + d u) * silu(z),    r = softplus(dt + bias).
//
// Every state of every frame costs an exponential (16 a clock and SM on the special function units), two products and two multiply-adds, and nothing of it can be shared: decays
// differ in channel, state and frame.  With 16 states, and the four exponentials and reciprocals of a step and a gate, that is 20 of those units' operations for 8 bytes of bf16: 37 us
// for 8.4 million of them (32 sequences of 128 frames, 2048 channels), three times what memory takes.  63 us measured: 132 instructions for the 160 cycles of a warp's frame.
// Exponentials as polynomials on the multiply-add units for some of the states took as long (two of 16) or longer, since those and the issue of instructions have no more to give.
//
// A thread holds K states of a channel in registers over all its frames, L threads of a warp share a channel (state n: thread n / 4 % L, so that the L threads' loads of b and c lie
// side by side).  Steps and inputs are computed once: of L frames each of the L threads takes one, hands r and r u to the others by shuffles, and has that frame's output
// after an exchange of the partial sums (L - 1 shuffles for L frames).  Frames come in stages of eight through shared memory, by copies a stage ahead; loads into registers that are
// under way during the frames' work hold up every other wait of the warp.  Two channels to a thread, which would save the doubling of r and r u for paired products, leave too
// few warps (82 us).
//
// Drift.  The approximate exponential is low by 2e-8 in the mean, which a state that loses a thousandth of itself per frame makes 2e-5 of.  So a state is carried over in chunks of
// 32 frames, by one exponential of their steps' sum that has no bias, and what comes in during a chunk is summed apart: `local`.  That costs a multiply-add for a state and frame and
// takes the error of states from 2e-6 to 3e-7.  A segment whose states nobody asks for (what enters the next comes from the segments' sums) goes without where its outputs are rounded to
// bf16: over 1024 frames the bias comes to 2e-5 of a state at most, half a step of bf16 is 4e-3 (a sequence of 16384 frames of 1024 channels: 202 us, with the carry 212).
//
// Long sequences are cut into segments: their sums (without outputs), the states that enter them, their outputs.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
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

using srx::Few;
using srx::Pair;

struct ScanArgs {
    const void *u, *dt, *z, *b, *c;
    const float *a, *d, *bias;
    const int64_t *offsets, *longest;                  // longest: packed sequences', where they are many
    const float* state_in;
    float* state_out;
    void* out;
    float* sums;                                       // [slot][channels][states]: states after a segment that none enter, then those that enter it
    float* steps;                                      // [slot][channels]: sum of r over a segment
    int64_t frames, segment, whole, count;             // segment 0: whole sequences; whole: packed sequences are not cut where none is longer; count: segments of each of others
    int32_t batch, channels, states, groups, share, softplus, tiles;      // share: channels of a group; tiles: CTAs side by side over them
    sr_frame_strides su, sdt, sz, so;
    sr_attention_strides sb, sc;
    bool units, quads;                                 // b and c can be copied 16 bytes at a time; states and decays, too
};

constexpr int kBlock = 8;                              // frames of a stage
constexpr int kChunk = 32;                             // frames that a state is carried over at once
constexpr int kUncarried = 1024;                       // frames that a segment of bf16 outputs may have without that
enum { kWhole = 0, kSums = 1, kOutputs = 2 };          // whole sequences; sums of segments; outputs of segments, from the states that enter them
// A block's threads share b and c, whose widening is the more to do the more states there are; fewer make the work of SMs more even.
__host__ __device__ constexpr int threads_of(int lanes) { return lanes < 4 ? 32 : 128; }
// Of an SM, so 128 registers.  With 12 warps and 168: 16 packed sequences, 1024 channels of 64 states 630 us instead of 616, side by side with 300 frames each 138 instead of 129, of 128 states 224
// instead of 232.
constexpr int kWarps = 16;

// Frames of a segment of this run.  Blocks look for the longest of a few packed sequences themselves.  They are as many as the sequences, though, and all together look at the square of them: of
// more than kFew one block does, ahead of the others (sequences of 64 frames, 64 channels of 16 states: 64 of them 34.5 us by themselves, 36 with the block ahead; 256 46 either way; 1024 80 and
// 67, 4096 331 and 169).
constexpr int kFew = 256;
__device__ __forceinline__ int64_t segment_of(const ScanArgs& A)
{
    return A.offsets && (A.longest ? *A.longest : longest_span(A.offsets, A.frames, A.batch, threadIdx.x & 31, 32)) <= A.whole ? A.whole : A.segment;
}
constexpr int kLongestThreads = 1024;
__global__ void __launch_bounds__(kLongestThreads) sr_scan_longest_kernel(const int64_t* offsets, int64_t frames, int batch, int64_t* longest)
{
    __shared__ int64_t of[kLongestThreads / 32];
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t mine = longest_span(offsets, frames, batch, threadIdx.x, kLongestThreads);
    if (!(threadIdx.x & 31)) of[threadIdx.x >> 5] = mine;
    __syncthreads();
    if (threadIdx.x < 32) {
        const int64_t most = most_of_warp(of[threadIdx.x]);
        if (!threadIdx.x) *longest = most;
    }
}

// Sum over the L threads of a channel, whose lanes are SIDE apart: thread p gets frame p's.
template <int L, int SIDE>
__device__ __forceinline__ float exchange(float (&y)[L], int p)
{
#pragma unroll
    for (int half = L / 2; half; half /= 2) {
        const bool up = p & half;
#pragma unroll
        for (int i = 0; i < half; ++i) {
            const float give = up ? y[i] : y[i + half], keep = up ? y[i + half] : y[i];
            y[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, half * SIDE);
        }
    }
    return y[0];
}

__device__ __forceinline__ void copy_4(void* dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(srx::smem_u32(dst)), "l"(src) : "memory");
}
// A stage's rows of a tensor, `cols` of COLS elements in each, into shared memory, by THREADS threads: 16 bytes at a time (UNITS), or an element.  What is behind the last
// column or frame stays what it was.
template <typename T, int COLS, int THREADS, bool UNITS>
struct Rows {
    static constexpr int UNIT = UNITS ? 16 / (int)sizeof(T) : 1, PER_ROW = COLS / UNIT > 0 ? COLS / UNIT : 1;
    static constexpr int AT_ONCE = THREADS / PER_ROW, COPIES = AT_ONCE ? (kBlock + AT_ONCE - 1) / (AT_ONCE ? AT_ONCE : 1) : kBlock * (PER_ROW / THREADS);
    static_assert(AT_ONCE || PER_ROW % THREADS == 0);
    // The thread's first place; its copy e; whether that is one of `left` rows' and `cols` columns'.
    __device__ __forceinline__ static int frame(int e, int tid) { return AT_ONCE ? e * AT_ONCE + tid / PER_ROW : e / (PER_ROW / THREADS ? PER_ROW / THREADS : 1); }
    __device__ __forceinline__ static int col(int e, int tid)
    {
        return (AT_ONCE ? tid % PER_ROW : e % (PER_ROW / THREADS ? PER_ROW / THREADS : 1) * THREADS + tid) * UNIT;
    }
    __device__ __forceinline__ static bool there(int e, int tid, int cols, int left)
    {
        return (!AT_ONCE || THREADS % PER_ROW == 0 || tid < AT_ONCE * PER_ROW) && (kBlock % (AT_ONCE ? AT_ONCE : 1) == 0 || frame(e, tid) < kBlock) && frame(e, tid) < left && col(e, tid) < cols;
    }
    __device__ __forceinline__ static int64_t start(int tid, int64_t stride) { return frame(0, tid) * stride + col(0, tid); }
    __device__ __forceinline__ static int64_t away(int e, int tid, int64_t stride) { return (frame(e, tid) - frame(0, tid)) * stride + (col(e, tid) - col(0, tid)); }
    // from: the thread's first place
    __device__ __forceinline__ static void copy(T (*to)[COLS], const T* from, int64_t stride, int cols, int left, int tid)
    {
#pragma unroll
        for (int e = 0; e < COPIES; ++e) {
            if (!there(e, tid, cols, left)) continue;
            T* place = &to[frame(e, tid)][col(e, tid)];
            if constexpr (UNITS) srx::copy_16(place, from + away(e, tid, stride));
            else if constexpr (sizeof(T) == 4) copy_4(place, from + away(e, tid, stride));
            else *place = from[away(e, tid, stride)];
        }
    }
};

// What lies in shared memory: two stages as they come in, b and c of the one that is worked on as floats, its outputs, and the states at the chunk's start.
template <typename T, int K, int L, int THREADS, bool OUT>
struct ScanShared {
    static constexpr int NP = K * L, CHANNELS = THREADS / L, OUTS = OUT ? 2 : 1;
    T u[2][kBlock][CHANNELS], dt[2][kBlock][CHANNELS], z[OUTS][kBlock][CHANNELS], out[OUT ? kBlock : 1][CHANNELS];
    T b[2][kBlock][NP], c[OUTS][kBlock][NP];
    float bf[kBlock][NP], cf[OUT ? kBlock : 1][NP];
    float2 carried[K / 2][THREADS];
};

template <typename T, int K, int L, int MODE, bool WIDE>
__global__ void __launch_bounds__(threads_of(L), kWarps * 32 / threads_of(L)) sr_scan_kernel(const __grid_constant__ ScanArgs A)
{
    constexpr int THREADS = threads_of(L), NP = K * L, SIDE = 32 / L, CHANNELS = THREADS / L, N = kBlock / L;
    constexpr bool EXACT = sizeof(T) == 4, OUT = MODE != kSums;
    using Shared = ScanShared<T, K, L, THREADS, OUT>;
    static_assert(kBlock % L == 0 && kChunk % kBlock == 0);
    extern __shared__ __align__(16) uint8_t memory[];
    Shared& S = *reinterpret_cast<Shared*>(memory);
    srx::let_successor_start();
    srx::wait_for_predecessor();

    const int tile = blockIdx.x % A.tiles, rest = blockIdx.x / A.tiles, g = rest % A.groups;
    const int64_t slot = rest / A.groups;
    int b = (int)slot;
    int64_t seg = 0;
    const int64_t segment = MODE == kWhole ? 0 : segment_of(A);
    if (MODE != kWhole) {
        if (A.offsets) {
            packed_slot(A.offsets, A.frames, A.batch, segment, slot, b, seg);
            if (b < 0) return;
        } else {
            b = (int)((uint32_t)slot / (uint32_t)A.count);         // (there are not more slots than blocks)
            seg = slot - b * A.count;
        }
    }
    const FrameSpan span = frame_span(A.offsets, A.frames, b);
    const int64_t t0 = seg * segment, n = MODE == kWhole ? span.n : min(segment, span.n - t0);
    const bool last = t0 + n >= span.n;
    if (MODE == kSums && last) return;                 // (nobody asks for them)

    const int tid = threadIdx.x, lane = tid & 31, p = lane / SIDE, col = (tid >> 5) * SIDE + lane % SIDE;
    const int channels = min(A.share - tile * CHANNELS, CHANNELS), ch0 = g * A.share + tile * CHANNELS;
    const bool there = col < channels;
    const int ch = ch0 + (there ? col : 0);
    const int64_t first = span.first + t0;
    const bool gated = OUT && A.z;
    auto sync = [] {
        if (THREADS == 32) __syncwarp();
        else __syncthreads();
    };

    // ---- copies
    using Wide = Rows<T, CHANNELS, THREADS, WIDE>;
    using Some = Rows<T, NP, THREADS, false>;
    using Units = Rows<T, NP, THREADS, NP * sizeof(T) % 16 == 0>;
    constexpr bool CAN = NP * sizeof(T) % 16 == 0;     // rows of b and c in whole units
    const T* gu = static_cast<const T*>(A.u) + first * A.su.frame + span.b * A.su.sequence + ch0 + Wide::start(tid, A.su.frame);
    const T* gdt = static_cast<const T*>(A.dt) + first * A.sdt.frame + span.b * A.sdt.sequence + ch0 + Wide::start(tid, A.sdt.frame);
    const T* gz = gated ? static_cast<const T*>(A.z) + first * A.sz.frame + span.b * A.sz.sequence + ch0 + Wide::start(tid, A.sz.frame) : nullptr;
    const T* gb = static_cast<const T*>(A.b) + first * A.sb.frame + span.b * A.sb.sequence + g * A.sb.head;
    const T* gc = static_cast<const T*>(A.c) + first * A.sc.frame + span.b * A.sc.sequence + g * A.sc.head;
    const bool units = CAN && A.units;
    gb += units ? Units::start(tid, A.sb.frame) : Some::start(tid, A.sb.frame);
    gc += units ? Units::start(tid, A.sc.frame) : Some::start(tid, A.sc.frame);
    auto frames_from = [&](int64_t at) { return (int)max(min(n - at, (int64_t)kBlock), (int64_t)0); };
    auto fetch = [&](int half, int left) {
        Wide::copy(S.u[half], gu, A.su.frame, channels, left, tid);
        Wide::copy(S.dt[half], gdt, A.sdt.frame, channels, left, tid);
        gu += kBlock * A.su.frame;
        gdt += kBlock * A.sdt.frame;
        if (gated) {
            Wide::copy(S.z[OUT ? half : 0], gz, A.sz.frame, channels, left, tid);
            gz += kBlock * A.sz.frame;
        }
        if (units) {
            if constexpr (CAN) {
                Units::copy(S.b[half], gb, A.sb.frame, A.states, left, tid);
                if (OUT) Units::copy(S.c[OUT ? half : 0], gc, A.sc.frame, A.states, left, tid);
            }
        } else {
            Some::copy(S.b[half], gb, A.sb.frame, A.states, left, tid);
            if (OUT) Some::copy(S.c[OUT ? half : 0], gc, A.sc.frame, A.states, left, tid);
        }
        gb += kBlock * A.sb.frame;
        gc += kBlock * A.sc.frame;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    auto widen = [&](int half, int left) {             // b and c as floats: a thread's neighbouring states, all of a frame; zeros behind the last frame and state
        constexpr int MOST = kBlock * NP / THREADS, PART = MOST >= 8 && NP % 8 == 0 ? 8 : MOST > 2 && NP % 4 == 0 ? 4 : MOST == 2 ? 2 : 1, PER = NP / PART;
#pragma unroll
        for (int i = tid; i < kBlock * PER; i += THREADS) {
            const int f = i / PER, c = i % PER * PART;
            Few<T, PART> v;
            float y[PART];
            Few<float, PART> to;
            v.get(&S.b[half][f][c]);
#pragma unroll
            for (int e = 0; e < PART; ++e) y[e] = f < left && c + e < A.states ? v[e] : 0.0f;
            to.set(y);
            to.put(&S.bf[f][c]);
            if (OUT) {
                v.get(&S.c[OUT ? half : 0][f][c]);
#pragma unroll
                for (int e = 0; e < PART; ++e) y[e] = f < left && c + e < A.states ? v[e] : 0.0f;
                to.set(y);
                to.put(&S.cf[OUT ? f : 0][c]);
            }
        }
    };
    T* go = OUT ? static_cast<T*>(A.out) + first * A.so.frame + span.b * A.so.sequence + ch0 + Wide::start(tid, A.so.frame) : nullptr;
    auto put = [&](int left) {                         // a stage's outputs
#pragma unroll
        for (int e = 0; e < Wide::COPIES; ++e) {
            if (!Wide::there(e, tid, channels, left)) continue;
            T* to = go + Wide::away(e, tid, A.so.frame);
            const T* place = &S.out[OUT ? Wide::frame(e, tid) : 0][Wide::col(e, tid)];
            if constexpr (WIDE) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(place);
            else *to = *place;
        }
        go += kBlock * A.so.frame;
    };
    const float bias = A.bias ? A.bias[ch] : 0.0f, skip = OUT && A.d ? A.d[ch] : 0.0f;

    fetch(0, frames_from(0));
    // ---- the thread's states and decays; local: what the states are without those at the chunk's start
    Pair h[K / 2], local[K / 2], a2[K / 2];
    auto four = [&](const float* of, int i) {          // of a channel's states; zeros behind the last one
        if (A.quads) return i < A.states ? *reinterpret_cast<const float4*>(of + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto one = [&](int i) { return i < A.states ? of[i] : 0.0f; };
        return make_float4(one(i), one(i + 1), one(i + 2), one(i + 3));
    };
    {
        const int64_t entering = seg ? slot - 1 : slot + (A.offsets ? segments_of(span.n, segment) : A.count) - 1;       // (see sr_scan_join_kernel)
        const float* from = MODE == kSums ? nullptr : MODE == kOutputs && !(seg == 0 && last) ? A.sums + (entering * A.channels + ch) * A.states
                                                    : A.state_in ? A.state_in + ((int64_t)b * A.channels + ch) * A.states : nullptr;
        const float* a = A.a + (int64_t)ch * A.states;
#pragma unroll
        for (int k = 0; k < K; k += 4) {
            const int i = ((k / 4) * L + p) * 4;
            const float4 d = four(a, i), v = from ? four(from, i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            a2[k / 2] = srx::pair(srx::decay_base2(d.x), srx::decay_base2(d.y));
            a2[k / 2 + 1] = srx::pair(srx::decay_base2(d.z), srx::decay_base2(d.w));
            h[k / 2] = srx::pair(v.x, v.y);
            h[k / 2 + 1] = srx::pair(v.z, v.w);
            S.carried[k / 2][tid] = make_float2(v.x, v.y);
            S.carried[k / 2 + 1][tid] = make_float2(v.z, v.w);
            local[k / 2] = local[k / 2 + 1] = srx::pair(0.0f, 0.0f);
        }
    }

    double total = 0.0;                                // of r
    float since = 0.0f;                                // of r, from the chunk's start on
    int half = 0;
    auto all_frames = [&](auto carry) {
        constexpr bool CARRY = decltype(carry)::value;
        for (int64_t at = 0; at < n; at += kBlock, half ^= 1) {
            const int left = frames_from(at);
            asm volatile("cp.async.wait_all;" ::: "memory");
            sync();                                    // the stage has landed, and the one before is done with
            if (at + kBlock < n) fetch(half ^ 1, frames_from(at + kBlock));
            widen(half, left);
            sync();
#pragma unroll(EXACT ? 4 : 2)                     // (fp32: two at a time cost 7 % more; bf16 gains nothing from four)
            for (int q = 0; q < N; ++q) {
                // of L frames each of the channel's threads prepares one
                const int mine = q * L + p;
                const float s = (float)S.dt[half][mine][col] + bias, u = (float)S.u[half][mine][col], plus = srx::softplus<EXACT>(s);
                const float r = mine >= left ? 0.0f : A.softplus ? plus : s;         // (a frame behind the last one changes nothing)
                const float x = mine >= left ? 0.0f : r * u;
                float y[L];
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    const int f = q * L + i;
                    const float rr = L > 1 ? __shfl_sync(0xFFFFFFFFu, r, i * SIDE + lane % SIDE) : r;
                    const float xx = L > 1 ? __shfl_sync(0xFFFFFFFFu, x, i * SIDE + lane % SIDE) : x;
                    if (CARRY) since += rr;
                    const Pair r2 = srx::pair(rr, rr), x2 = srx::pair(xx, xx);
                    Pair y2 = srx::pair(0.0f, 0.0f);
#pragma unroll
                    for (int k = 0; k < K; k += 4) {
                        const float4 bv = *reinterpret_cast<const float4*>(&S.bf[f][((k / 4) * L + p) * 4]);
                        const float2 e0 = srx::split(srx::mul2(r2, a2[k / 2])), e1 = srx::split(srx::mul2(r2, a2[k / 2 + 1]));
                        const Pair d0 = srx::pair(srx::ex2(e0.x), srx::ex2(e0.y)), d1 = srx::pair(srx::ex2(e1.x), srx::ex2(e1.y));
                        const Pair i0 = srx::mul2(x2, srx::pair(bv.x, bv.y)), i1 = srx::mul2(x2, srx::pair(bv.z, bv.w));
                        if (CARRY) {
                            local[k / 2] = srx::fma2(d0, local[k / 2], i0);
                            local[k / 2 + 1] = srx::fma2(d1, local[k / 2 + 1], i1);
                        }
                        if (OUT) {
                            h[k / 2] = srx::fma2(d0, h[k / 2], i0);
                            h[k / 2 + 1] = srx::fma2(d1, h[k / 2 + 1], i1);
                            const float4 cv = *reinterpret_cast<const float4*>(&S.cf[OUT ? f : 0][((k / 4) * L + p) * 4]);
                            y2 = k ? srx::fma2(srx::pair(cv.x, cv.y), h[k / 2], y2) : srx::mul2(srx::pair(cv.x, cv.y), h[k / 2]);
                            y2 = srx::fma2(srx::pair(cv.z, cv.w), h[k / 2 + 1], y2);
                        }
                    }
                    const float2 v = srx::split(y2);
                    y[i] = v.x + v.y;
                }
                if (OUT) {
                    const float o = fmaf(skip, u, exchange<L, SIDE>(y, p)), gate = srx::silu<EXACT>((float)S.z[OUT ? half : 0][mine][col]);
                    S.out[OUT ? mine : 0][col] = (T)(gated ? o * gate : o);
                }
            }
            if (CARRY && ((at + kBlock) % kChunk == 0 || at + kBlock >= n)) {
                const Pair s2 = srx::pair(since, since);
#pragma unroll
                for (int k = 0; k < K / 2; ++k) {
                    const float2 v = S.carried[k][tid];
                    h[k] = srx::fma2(srx::exp2_exact(srx::mul2(s2, a2[k])), srx::pair(v.x, v.y), local[k]);
                    S.carried[k][tid] = srx::split(h[k]);
                    local[k] = srx::pair(0.0f, 0.0f);
                }
                total += (double)since;
                since = 0.0f;
            }
            if (OUT) {
                sync();
                put(left);
            }
        }
    };
    if (MODE == kOutputs && !EXACT && !last && n <= kUncarried) all_frames(std::false_type{});
    else all_frames(std::true_type{});

    float* to = MODE == kSums ? A.sums + (slot * A.channels + ch) * A.states : A.state_out && last ? A.state_out + ((int64_t)b * A.channels + ch) * A.states : nullptr;
    if (to && there) {
#pragma unroll
        for (int k = 0; k < K; k += 4) {
            const int i = ((k / 4) * L + p) * 4;
            const float2 v = S.carried[k / 2][tid], w = S.carried[k / 2 + 1][tid];
            if (A.quads) {
                if (i < A.states) *reinterpret_cast<float4*>(to + i) = make_float4(v.x, v.y, w.x, w.y);
            } else {
                if (i < A.states) to[i] = v.x;
                if (i + 1 < A.states) to[i + 1] = v.y;
                if (i + 2 < A.states) to[i + 2] = w.x;
                if (i + 3 < A.states) to[i + 3] = w.y;
            }
        }
    }
    if (MODE == kSums && there && p == 0) A.steps[slot * A.channels + ch] = (float)total;
}

// The states that enter the segments of sequences that have several, from their sums, one thread for VEC states of a channel.  What enters a segment takes the place of the sum before it,
// what enters the first that of the last one's, which is not made (state_in may be state_out, which the last segment writes).  Bound by the latency of a load for every AHEAD segments, or, where
// there are so many states that blocks come in several rounds, by what a block does before its first load: then four states to a thread (16 packed sequences of 1024 channels of 64 states, the
// whole run: 613 us, with one 629; one sequence of 16384 frames, 1024 channels of 16 states: 209, with one state and 16 segments ahead 198).  Warps that shared a
// state's segments took 24 us instead of 5 for 16 segments of 66660 states, and less (40, not 64) only for 512 of 16384, which no run is cut into.
constexpr int kJoinThreads = 128;
template <int VEC, int AHEAD>
__global__ void __launch_bounds__(kJoinThreads) sr_scan_join_kernel(const __grid_constant__ ScanArgs A)
{
    __shared__ int64_t count_of, slot0_of;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t per = (int64_t)A.channels * A.states, mine = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) * VEC, i = min(mine, per - VEC);
    const int64_t ch = per <= 0xFFFFFFFF ? (uint32_t)i / (uint32_t)A.states : i / A.states;
    Few<float, VEC> a, h, sum[AHEAD];
    a.get(A.a + i);
    for (int b = blockIdx.y; b < A.batch; b += gridDim.y) {
        if (A.offsets) {
            if (threadIdx.x < 32) {
                const int64_t segment = segment_of(A), n = segments_of(frame_span(A.offsets, A.frames, b).n, segment), slot0 = packed_first(A.offsets, A.frames, segment, b);
                if (threadIdx.x == 0) {
                    count_of = n;
                    slot0_of = slot0;
                }
            }
            __syncthreads();
        }
        const int64_t count = A.offsets ? count_of : A.count, slot0 = A.offsets ? slot0_of : b * A.count;
        if (A.offsets) __syncthreads();
        if (count < 2) continue;
        float now[VEC] = {};
        if (A.state_in) {
            h.get(A.state_in + b * per + i);
#pragma unroll
            for (int e = 0; e < VEC; ++e) now[e] = h[e];
        }
        float* at = A.sums + slot0 * per + i;
        const float* steps = A.steps + slot0 * A.channels + ch;
        h.set(now);
        if (mine < per) h.put(at + (count - 1) * per);
        for (int64_t s = 0; s < count - 1; s += AHEAD) {           // (the last segment's sums are not made)
            const int left = (int)min(count - 1 - s, (int64_t)AHEAD);
            float step[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (k < left) {
                    sum[k].get(at + k * per);
                    step[k] = steps[k * A.channels];
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (k < left) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) now[e] = fmaf(srx::exp2_exact(srx::decay_base2(a[e]) * step[k]), now[e], sum[k][e]);
                    h.set(now);
                    if (mine < per) h.put(at + k * per);
                }
            }
            at += AHEAD * per;
            steps += AHEAD * A.channels;
        }
    }
}

// ------------------------------------------------------------------------------------------ single frames
// One frame: the states are read and written once.  L threads have VEC states each of a channel (more where L is 32 already: PIECES), the warp's other threads the next
// channels; a block goes over `per` sequences with the same decays, the loads of AHEAD of them under way.  UNITS: b and c can be read VEC at a time.  Bound by memory where there are
// many sequences, but not far from the issue of its instructions, of which most are for a channel and not for a state: hence eight states to a thread.
template <typename T, int VEC, int PIECES, int AHEAD, bool UNITS>
__global__ void __launch_bounds__(128, 4) sr_scan_step_kernel(const __grid_constant__ ScanArgs A, int L, int per)
{
    constexpr bool EXACT = sizeof(T) == 4;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int p = threadIdx.x % L;                     // (L: a power of two)
    const int64_t ch0 = (int64_t)blockIdx.x * (128 / L) + threadIdx.x / L;
    const bool there = ch0 < A.channels;
    const int ch = there ? (int)ch0 : 0, g = A.groups > 1 ? ch / A.share : 0, b0 = (int)blockIdx.y * per, seqs = min(A.batch - b0, per);
    const int64_t apart = (int64_t)A.channels * A.states;
    const T* pu = static_cast<const T*>(A.u) + b0 * A.su.sequence + ch;
    const T* pdt = static_cast<const T*>(A.dt) + b0 * A.sdt.sequence + ch;
    const T* pz = A.z ? static_cast<const T*>(A.z) + b0 * A.sz.sequence + ch : nullptr;
    const T* pb = static_cast<const T*>(A.b) + b0 * A.sb.sequence + g * A.sb.head + p * VEC;
    const T* pc = static_cast<const T*>(A.c) + b0 * A.sc.sequence + g * A.sc.head + p * VEC;
    const float* from = A.state_out + b0 * apart + (int64_t)ch * A.states + p * VEC;
    float* to = A.state_out + b0 * apart + (int64_t)ch * A.states + p * VEC;
    T* out = static_cast<T*>(A.out) + b0 * A.so.sequence + ch;
    auto is = [&](int k) { return there && (k * L + p) * VEC < A.states; };         // (VEC 4, 8: the states are a multiple of it)
    struct Item {
        T u, dt, z;
        Few<float, VEC> h[PIECES];
        Few<T, VEC> b[PIECES], c[PIECES];
    } items[AHEAD];
    auto get = [&](Few<T, VEC>& v, const T* of) {
        if constexpr (UNITS || VEC == 1) {
            v.get(of);
        } else {
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = (float)of[e];
            v.set(f);
        }
    };
    auto load = [&](Item& item) {
        item.u = *pu;
        item.dt = *pdt;
        if (pz) item.z = *pz;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (!is(k)) continue;
            item.h[k].get(from + k * L * VEC);
            get(item.b[k], pb + k * L * VEC);
            get(item.c[k], pc + k * L * VEC);
        }
        pu += A.su.sequence;
        pdt += A.sdt.sequence;
        if (pz) pz += A.sz.sequence;
        pb += A.sb.sequence;
        pc += A.sc.sequence;
        from += apart;
    };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
        if (j < seqs) load(items[j]);
    const float bias = A.bias ? A.bias[ch] : 0.0f, skip = A.d ? A.d[ch] : 0.0f;
    float a2[PIECES][VEC];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        Few<float, VEC> a = {};
        if (is(k)) a.get(A.a + (int64_t)ch * A.states + (k * L + p) * VEC);
#pragma unroll
        for (int e = 0; e < VEC; ++e) a2[k][e] = srx::decay_base2(a[e]);
    }
    auto work = [&](const Item& item) {
        const float s = (float)item.dt + bias, r = A.softplus ? srx::softplus<EXACT>(s) : s, u = (float)item.u, x = r * u;
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            if (!is(k)) continue;
            float h[VEC];
            if constexpr (VEC > 1) {
                Pair sum = srx::pair(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const Pair decay = srx::exp2_exact(srx::mul2(srx::pair(r, r), srx::pair(a2[k][e], a2[k][e + 1])));
                    const Pair v = srx::fma2(decay, srx::pair(item.h[k][e], item.h[k][e + 1]), srx::mul2(srx::pair(x, x), srx::pair(item.b[k][e], item.b[k][e + 1])));
                    sum = srx::fma2(srx::pair(item.c[k][e], item.c[k][e + 1]), v, sum);
                    const float2 f = srx::split(v);
                    h[e] = f.x;
                    h[e + 1] = f.y;
                }
                const float2 f = srx::split(sum);
                y += f.x + f.y;
            } else {
                h[0] = fmaf(srx::exp2_exact(r * a2[k][0]), item.h[k][0], x * item.b[k][0]);
                y = fmaf(item.c[k][0], h[0], y);
            }
            Few<float, VEC> o;
            o.set(h);
            o.put(to + k * L * VEC);
        }
        to += apart;
#pragma unroll 1
        for (int d = 1; d < L; d *= 2) y += __shfl_xor_sync(0xFFFFFFFFu, y, d);
        float o = fmaf(skip, u, y);
        if (pz) o *= srx::silu<EXACT>((float)item.z);
        if (p == 0 && there) *out = (T)o;
        out += A.so.sequence;
    };
#pragma unroll 1
    for (int s = 0; s < seqs; s += AHEAD) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (s + j >= seqs) break;
            work(items[j]);
            if (s + j + AHEAD < seqs) load(items[j]);
        }
    }
}

// ------------------------------------------------------------------------------------------ launches
// early: while the kernel before drains.
template <typename F, typename... Args>
cudaError_t start(F* kernel, bool early, dim3 grid, int threads, int shared, cudaStream_t s, Args... args)
{
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)shared;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename F, typename... Args>
cudaError_t start(F* kernel, bool early, int64_t blocks, int threads, int shared, cudaStream_t s, Args... args)
{
    return blocks > 0x7FFFFFFF ? cudaErrorInvalidValue : start(kernel, early, dim3((unsigned)blocks), threads, shared, s, args...);
}

// How a run is cut.
struct ScanCut {
    int held, lanes;
    int64_t segment, slots, whole;                     // segment 0: whole sequences
};
// Cycles that cutting costs besides: two launches, the latency of the join's loads, and the segments' states, which are written, joined and read (16 bytes each).
double joining(const sr_scan_desc* d, int64_t count) { return 16000.0 + count / 8 * 2000.0 + (double)d->batch * count * d->channels * d->states / 200; }
// Cycles that `warps` warps, spread over all schedulers, take for a frame; measured for 16 states in bf16 (fp32: 1.5 times as many).  Rounds of four follow each other without a gap, and what one
// SM is behind in one another makes up for in the next (8192 frames of 8192 channels: 778 us in one round, 736 in two, 697 in four).
double cycles_of(double warps, int64_t schedulers)
{
    constexpr double kOf[5] = {0, 427, 545, 705, 880};
    const double each = std::ceil(warps / schedulers), rounds = std::floor(each / 4);
    return (rounds * kOf[4] + kOf[(int)(each - 4 * rounds)]) * (each > 4 ? 0.92 + 0.32 / each : 1.0);
}
// Whole sequences where their channels fill the schedulers; otherwise segments, whose sums cost 0.7 of their outputs, and two launches more.
// Side by side: of the numbers of segments that just give every scheduler one to four warps, or rounds of four, the one with the smallest estimate (5 sequences of 500 frames, 1111 channels, fp32:
// 46 us with segments of 40 frames, 50 with 32).
// Packed: only the GPU knows the lengths.  There are segments of a third of the frames that there are for each scheduler's warp (16 sequences, 1024 channels of 64 states: 619 us, of half of them 637,
// all 731), but not below 72 where there are as many (7500 frames, 700 channels of 12: 76 us, with 32 frames 92), where some sequence has more than 1.75 times those, that is, would
// take longer than all of them in segments; else, as the kernels find, no sequence is cut.
ScanCut scan_cut(const sr_scan_desc* d, bool packed, int sms)
{
    ScanCut c{};
    int padded = 4;
    while (padded < d->states) padded *= 2;
    c.held = std::min(padded, 16);
    c.lanes = padded / c.held;
    if (c.held == 16 && c.lanes <= 2 && d->states <= 12 * c.lanes) c.held = 12;
    c.slots = d->batch;
    if (d->frames <= kChunk || !d->batch) return c;
    const int64_t per = threads_of(c.lanes) / c.lanes, tiles = (d->channels / d->groups + per - 1) / per;
    const int64_t warps = d->groups * tiles * (threads_of(c.lanes) / 32), schedulers = 4 * (int64_t)std::max(sms, 1);          // of a sequence
    auto whole_chunks = [](int64_t frames) { return std::max<int64_t>((frames + kChunk - 1) / kChunk, 1) * kChunk; };
    if (packed) {
        const int64_t even = (int64_t)std::min((double)d->frames * warps / (schedulers * 4), 1e12);
        c.whole = whole_chunks(even * 7 / 4);
        if (c.whole >= d->frames) return c;
        c.segment = std::max<int64_t>((std::max(even / 3, std::min<int64_t>(even, 72)) + kBlock - 1) / kBlock * kBlock, kChunk);
        c.slots = d->frames / c.segment + d->batch;
        return c;
    }
    const int64_t at_once = warps * d->batch;
    auto cycles_for = [&](int64_t frames, int64_t count) { return frames * cycles_of((double)at_once * count, schedulers); };
    double best = cycles_for(d->frames, 1);
    for (int each = 1; each <= 64; each += each < 4 ? 1 : 4) {
        const int64_t most = each * schedulers / at_once;
        if (most < 2) continue;
        const int64_t segment = std::max<int64_t>((d->frames + kBlock * most - 1) / (kBlock * most) * kBlock, kChunk), count = segments_of(d->frames, segment);
        if (count < 2) continue;
        const double cycles = cycles_for(segment, count) + 0.7 * cycles_for(segment, count - 1) + joining(d, count);
        if (cycles < best) {
            best = cycles;
            c.segment = segment;
            c.slots = d->batch * count;
        }
    }
    return c;
}
size_t cut_bytes(const sr_scan_desc* d, const ScanCut& c)
{
    return c.segment ? (size_t)c.slots * d->channels * ((size_t)d->states * 4 + 4) + 256 : 0;
}

template <typename T, int K, int L, int MODE, bool WIDE>
cudaError_t launch_mode(const ScanArgs& A, int64_t grid, cudaStream_t s)
{
    static SrSharedLimit limit;
    constexpr int bytes = (int)sizeof(ScanShared<T, K, L, threads_of(L), MODE != kSums>);
    if (bytes > 48 << 10) {
        const cudaError_t e = limit.raise(sr_scan_kernel<T, K, L, MODE, WIDE>, bytes);
        if (e != cudaSuccess) return e;
    }
    // Blocks that come while others drain go where those have left room: unless they nearly fill the SMs anyway some of these get more than their part, and the time is theirs (512 frames of
    // 16 sequences, 2048 channels: 196 us, one after the other 150).
    const int64_t most = (int64_t)sr_device_sms() * kWarps / (threads_of(L) / 32) * 3 / 4;
    return start(sr_scan_kernel<T, K, L, MODE, WIDE>, grid >= most || grid <= sr_device_sms(), grid, threads_of(L), bytes, s, A);
}
template <typename T, int K, int L, bool WIDE>
cudaError_t launch_scan(const ScanArgs& A, const ScanCut& c, cudaStream_t s)
{
    const int64_t grid = c.slots * A.groups * A.tiles;
    if (!c.segment) return launch_mode<T, K, L, kWhole, WIDE>(A, grid, s);
    cudaError_t e = A.longest ? start(sr_scan_longest_kernel, true, dim3(1), kLongestThreads, 0, s, A.offsets, A.frames, A.batch, const_cast<int64_t*>(A.longest)) : cudaSuccess;
    if (e == cudaSuccess) e = launch_mode<T, K, L, kSums, WIDE>(A, grid, s);
    if (e == cudaSuccess) {
        const int64_t states = (int64_t)A.channels * A.states;
        auto join = [&](auto* kernel, int vec) {
            const int64_t blocks = (states / vec + kJoinThreads - 1) / kJoinThreads;
            return blocks > 0x7FFFFFFF ? cudaErrorInvalidValue : start(kernel, true, dim3((unsigned)blocks, (unsigned)std::min(A.batch, 65535)), kJoinThreads, 0, s, A);
        };
        const bool many = (double)states * A.batch >= 4096.0 * sr_device_sms();
        e = A.quads && many ? join(sr_scan_join_kernel<4, 8>, 4) : join(sr_scan_join_kernel<1, 16>, 1);
    }
    if (e == cudaSuccess) e = launch_mode<T, K, L, kOutputs, WIDE>(A, grid, s);
    return e;
}
template <typename T, bool WIDE>
cudaError_t launch_scan(const ScanArgs& A, const ScanCut& c, cudaStream_t s)
{
    if (c.held == 4) return launch_scan<T, 4, 1, WIDE>(A, c, s);
    if (c.held == 8) return launch_scan<T, 8, 1, WIDE>(A, c, s);
    if (c.held == 12) return c.lanes == 1 ? launch_scan<T, 12, 1, WIDE>(A, c, s) : launch_scan<T, 12, 2, WIDE>(A, c, s);
    if (c.lanes == 1) return launch_scan<T, 16, 1, WIDE>(A, c, s);
    if (c.lanes == 2) return launch_scan<T, 16, 2, WIDE>(A, c, s);
    if (c.lanes == 4) return launch_scan<T, 16, 4, WIDE>(A, c, s);
    return launch_scan<T, 16, 8, WIDE>(A, c, s);
}
// 16 bytes at a time where the rows of a tensor start on them.
template <typename T>
cudaError_t launch_scan(ScanArgs A, const ScanCut& c, cudaStream_t s)
{
    constexpr int vec = 16 / sizeof(T);
    const bool one = A.offsets || A.batch < 2;         // (no strides between sequences)
    auto fits = [&](const void* p, const sr_frame_strides& st) { return !((uintptr_t)p & 15) && (A.frames < 2 || st.frame % vec == 0) && (one || st.sequence % vec == 0); };
    auto units = [&](const void* p, const sr_attention_strides& st) { return A.states % vec == 0 && fits(p, sr_frame_strides{st.frame, st.sequence}) && (A.groups < 2 || st.head % vec == 0); };
    A.units = units(A.b, A.sb) && units(A.c, A.sc);
    A.quads = A.states % 4 == 0 && !(((uintptr_t)A.a | (uintptr_t)A.state_in | (uintptr_t)A.state_out) & 15);
    const bool wide = A.share % vec == 0 && fits(A.u, A.su) && fits(A.dt, A.sdt) && fits(A.z, A.sz) && fits(A.out, A.so);
    return wide ? launch_scan<T, true>(A, c, s) : launch_scan<T, false>(A, c, s);
}

template <typename T, int VEC, int PIECES, int AHEAD, bool UNITS>
cudaError_t launch_step(const ScanArgs& A, int per, cudaStream_t s)
{
    const int units = (A.states + VEC - 1) / VEC;
    int L = 1;
    while (L < 32 && L < units) L *= 2;
    const int64_t parts = ((int64_t)A.channels + 128 / L - 1) / (128 / L);
    per = std::max(per, (A.batch + 65534) / 65535);
    return start(sr_scan_step_kernel<T, VEC, PIECES, AHEAD, UNITS>, true, dim3((unsigned)parts, (unsigned)((A.batch + per - 1) / per)), 128, 0, s, A, L, per);
}
template <typename T>
cudaError_t launch_step(const ScanArgs& A, cudaStream_t s)
{
    auto units = [&](int vec) {
        auto lies = [&](const void* p, const sr_attention_strides& st) {
            return (uintptr_t)p % std::min<size_t>(16, vec * sizeof(T)) == 0 && (A.batch < 2 || st.sequence % vec == 0) && (A.groups < 2 || st.head % vec == 0);
        };
        return lies(A.b, A.sb) && lies(A.c, A.sc);
    };
    // 256 sequences of 4096 channels with 16 states: 28.4 us (5.0 TB/s); with the loads of one sequence ahead 30.3, with four states to a thread and four sequences at once 45
    constexpr int AHEAD = sizeof(T) == 2 ? 3 : 2;
    const int per = std::max(1, std::min(16, A.batch / 16));
    if (A.states % 4 || ((uintptr_t)A.state_out & 15) || ((uintptr_t)A.a & 15))
        return A.states <= 32 ? launch_step<T, 1, 1, AHEAD, false>(A, per, s) : launch_step<T, 1, 4, 1, false>(A, per, s);
    if (A.batch >= 16 && A.states % 8 == 0 && units(8)) return launch_step<T, 8, 1, AHEAD, true>(A, per, s);
    return units(4) ? launch_step<T, 4, 1, AHEAD, true>(A, per, s) : launch_step<T, 4, 1, AHEAD, false>(A, per, s);
}

// ------------------------------------------------------------------------------------------ checks
bool fits(const sr_frame_strides& s) { return s.frame >= 0 && s.sequence >= 0; }
bool fits(const sr_attention_strides& s) { return s.frame >= 0 && s.sequence >= 0 && s.head >= 0; }

sr_status check(const sr_scan_desc* d)
{
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || d->batch < 0 || d->batch > kMostSequences || d->channels < 1 || d->states < 1 ||
        d->groups < 1 || d->channels % d->groups || d->frames < 0 || (d->softplus != 0 && d->softplus != 1) || !fits(d->u) || !fits(d->dt) || !fits(d->z) || !fits(d->out) || !fits(d->b) ||
        !fits(d->c))
        return SR_ERR_INVALID_ARG;
    if (d->states > 128) return SR_ERR_UNSUPPORTED;
    if ((double)d->frames * d->channels > 0x1p45 || (double)d->batch * d->channels * d->states > 0x1p45) return SR_ERR_INVALID_ARG;          // (no memory holds them)
    return SR_OK;
}
bool aligned(const void* p, int dtype) { return !((uintptr_t)p & (dtype == SR_DTYPE_F32 ? 3 : 1)); }

// The tensors of a call; false: one is missing, misaligned or lies where the outputs go.
bool tensors(const sr_scan_desc* d, ScanArgs& A, const void* u, const void* dt, const float* a, const void* b, const void* c, const float* skip, const void* z,
             const float* bias, void* out)
{
    if (!u || !dt || !a || !b || !c || !out || !aligned(u, d->dtype) || !aligned(dt, d->dtype) || !aligned(z, d->dtype) || !aligned(b, d->dtype) || !aligned(c, d->dtype) ||
        !aligned(out, d->dtype) || ((uintptr_t)a & 3) || ((uintptr_t)skip & 3) || ((uintptr_t)bias & 3) || out == u || out == dt || out == z || out == b || out == c)
        return false;
    A.u = u;
    A.dt = dt;
    A.a = a;
    A.b = b;
    A.c = c;
    A.d = skip;
    A.z = z;
    A.bias = bias;
    A.out = out;
    A.frames = d->frames;
    A.batch = d->batch;
    A.channels = d->channels;
    A.states = d->states;
    A.groups = d->groups;
    A.share = d->channels / d->groups;
    A.softplus = d->softplus;
    A.su = d->u;
    A.sdt = d->dt;
    A.sz = d->z;
    A.so = d->out;
    A.sb = d->b;
    A.sc = d->c;
    return true;
}

}  // namespace

extern "C" {

sr_status sr_selective_scan_workspace_bytes(const sr_scan_desc* d, int packed, size_t* bytes)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!bytes) return SR_ERR_INVALID_ARG;
    *bytes = cut_bytes(d, scan_cut(d, packed != 0, sr_device_sms()));
    return SR_OK;
}

sr_status sr_selective_scan_plan(const sr_scan_desc* d, int packed, int sms, sr_scan_plan* plan)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!plan || sms < 0) return SR_ERR_INVALID_ARG;
    if (!sms) sms = sr_device_sms();
    if (sms < 1) return SR_ERR_CUDA;
    const ScanCut c = scan_cut(d, packed != 0, sms);
    *plan = sr_scan_plan{c.held, c.lanes, c.segment, c.slots};
    return SR_OK;
}

sr_status sr_selective_scan_run(const sr_scan_desc* d, const void* u, const void* dt, const float* a, const void* b, const void* c, const float* skip, const void* z,
                                const float* bias, const int64_t* offsets, const float* state_in, float* state_out, void* out, void* workspace, size_t workspace_bytes,
                                void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if (((uintptr_t)state_in & 3) || ((uintptr_t)state_out & 3) || ((uintptr_t)offsets & 7)) return SR_ERR_INVALID_ARG;
    ScanArgs A{};
    if (d->frames ? !tensors(d, A, u, dt, a, b, c, skip, z, bias, out) : !state_out) return d->frames ? SR_ERR_INVALID_ARG : SR_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!d->frames) {                                  // (there need not be any tensors then)
        const size_t bytes = (size_t)d->batch * d->channels * d->states * 4;
        const cudaError_t e = state_in == state_out ? cudaSuccess : state_in ? cudaMemcpyAsync(state_out, state_in, bytes, cudaMemcpyDeviceToDevice, s)
                                                                               : cudaMemsetAsync(state_out, 0, bytes, s);
        return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
    }
    if (frames_overlap(d->out.frame, d->out.sequence, d->frames, offsets ? 1 : d->batch, d->channels)) return SR_ERR_INVALID_ARG;
    const ScanCut cut = scan_cut(d, offsets != nullptr, sr_device_sms());
    const size_t needed = cut_bytes(d, cut);
    if (needed && (!workspace || workspace_bytes < needed || ((uintptr_t)workspace & 255))) return SR_ERR_INVALID_ARG;
    A.offsets = offsets;
    A.state_in = state_in;
    A.state_out = state_out;
    A.segment = cut.segment;
    A.whole = cut.whole;
    A.count = cut.segment ? segments_of(d->frames, cut.segment) : 1;
    A.sums = static_cast<float*>(workspace);
    A.steps = A.sums + cut.slots * d->channels * d->states;
    if (cut.segment && offsets && d->batch > kFew) A.longest = reinterpret_cast<int64_t*>(static_cast<uint8_t*>(workspace) + ((needed - 16) & ~(size_t)7));     // (behind the steps)
    const int per = threads_of(cut.lanes) / cut.lanes;
    A.tiles = (A.share - 1) / per + 1;
    const cudaError_t e = d->dtype == SR_DTYPE_F32 ? launch_scan<float>(A, cut, s) : launch_scan<__nv_bfloat16>(A, cut, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_selective_scan_step(const sr_scan_desc* d, const void* u, const void* dt, const float* a, const void* b, const void* c, const float* skip, const void* z,
                                 const float* bias, float* state, void* out, void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    ScanArgs A{};
    if (!tensors(d, A, u, dt, a, b, c, skip, z, bias, out) || !state || ((uintptr_t)state & 3) || frames_overlap(0, d->out.sequence, 1, d->batch, d->channels))
        return SR_ERR_INVALID_ARG;
    A.state_out = state;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d->dtype == SR_DTYPE_F32 ? launch_step<float>(A, s) : launch_step<__nv_bfloat16>(A, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
