// Selective scan: per channel i and state n    h <- exp(r a[i, n]) h + r u b[n],    out = (sum_n c[n] h + d u) * silu(z),    r = softplus(dt + bias).
//
// Every state of every frame costs an exponential (16 a clock and SM on the special function units), two products and two multiply-adds, and nothing of it can be shared: decays
// differ in channel, state and frame.  With 16 states that is three times what memory takes for u, dt, z and out, so the kernel is built around the issue of those.
//
// A thread holds K states of a channel in registers over all its frames, L threads of a warp share a channel (state n: thread n / 4 % L, so that the L threads' loads of b and c lie
// side by side).  Steps and inputs are computed once: of L frames each of the L threads takes one, hands r and r u to the others by shuffles, and has that frame's output
// after an exchange of the partial sums (L - 1 shuffles for L frames).  b and c of a piece of frames lie in shared memory as floats, in two buffers; u, dt and z come
// straight into registers, a block of frames ahead.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/sr_rollout.h"
#include "sr_operators.h"
#include "sr_pair.cuh"
#include "sr_ptx.cuh"
#include "sr_selective.cuh"
#include "sr_spans.cuh"

namespace {

using srx::Pair;

struct ScanArgs {
    const void *u, *dt, *z, *b, *c;
    const float *a, *d, *bias;
    const int64_t* offsets;
    const float* state_in;
    float* state_out;
    void* out;
    float* sums;                                       // [slot][channels][states]: states after a segment that none enter, then those that enter it
    float* steps;                                      // [slot][channels]: sum of r over a segment
    int64_t frames, segment;                           // segment 0: whole sequences
    int32_t batch, channels, states, groups, share, softplus, tiles;      // share: channels of a group; tiles: CTAs side by side over them
    sr_frame_strides su, sdt, sz, so;
    sr_attention_strides sb, sc;
};

constexpr int kThreads = 128, kBlock = 8;              // frames that are loaded ahead
enum { kWhole = 0, kSums = 1, kOutputs = 2 };          // whole sequences; sums of segments; outputs of segments, from the states that enter them

template <int K, int L>
struct ScanTile {
    static constexpr int NP = K * L;                   // states, with those that pad them
    static constexpr int PIECE = NP >= 128 ? kBlock : 1024 / NP;          // frames of b and c in a buffer
    static constexpr int SIDE = 32 / L;                // channels of a warp
    static constexpr int CHANNELS = kThreads / L;
};

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

template <typename T, int K, int L, int MODE>
__global__ void __launch_bounds__(kThreads) sr_scan_kernel(const __grid_constant__ ScanArgs A)
{
    using Tile = ScanTile<K, L>;
    constexpr int NP = Tile::NP, PIECE = Tile::PIECE, SIDE = Tile::SIDE, Q = kBlock / L, EACH = PIECE * NP / kThreads;
    constexpr bool EXACT = sizeof(T) == 4;
    static_assert(kBlock % L == 0 && PIECE % kBlock == 0 && PIECE * NP % kThreads == 0);
    __shared__ __align__(16) float sb[2][PIECE][NP], sc[MODE == kSums ? 1 : 2][MODE == kSums ? 1 : PIECE][NP];
    srx::let_successor_start();
    srx::wait_for_predecessor();

    const int tile = blockIdx.x % A.tiles, rest = blockIdx.x / A.tiles, g = rest % A.groups;
    const int64_t slot = rest / A.groups;
    int b = (int)slot;
    int64_t seg = 0;
    if (MODE != kWhole) find_slot(A.offsets, A.frames, A.batch, A.segment, slot, b, seg);
    if (b < 0) return;
    const FrameSpan span = frame_span(A.offsets, A.frames, b);
    const int64_t t0 = MODE == kWhole ? 0 : seg * A.segment, n = MODE == kWhole ? span.n : min(A.segment, span.n - t0);
    const bool last = t0 + n >= span.n;
    if (MODE == kSums && last) return;                 // (nobody asks for them)

    const int lane = threadIdx.x & 31, p = lane / SIDE, in_tile = (threadIdx.x >> 5) * SIDE + lane % SIDE, in_group = tile * Tile::CHANNELS + in_tile;
    const bool there = in_group < A.share;
    const int ch = g * A.share + (there ? in_group : 0);
    const int64_t first = span.first + t0;

    // the thread's states and decays
    Pair h[K / 2], a2[K / 2];
    {
        const float* from = MODE == kWhole ? (A.state_in ? A.state_in + ((int64_t)b * A.channels + ch) * A.states : nullptr)
                                           : MODE == kOutputs ? A.sums + (slot * A.channels + ch) * A.states : nullptr;
        const float* a = A.a + (int64_t)ch * A.states;
#pragma unroll
        for (int k = 0; k < K; k += 2) {
            const int i = ((k / 4) * L + p) * 4 + k % 4;
            const bool lo = i < A.states, hi = i + 1 < A.states;
            a2[k / 2] = srx::pair(lo ? srx::kLog2e * a[i] : 0.0f, hi ? srx::kLog2e * a[i + 1] : 0.0f);
            h[k / 2] = srx::pair(from && lo ? from[i] : 0.0f, from && hi ? from[i + 1] : 0.0f);
        }
    }
    const float bias = A.bias ? A.bias[ch] : 0.0f, skip = A.d ? A.d[ch] : 0.0f;

    // where the thread's frames lie: every L-th, from p on
    const T* pu = static_cast<const T*>(A.u) + (first + p) * A.su.frame + span.b * A.su.sequence + ch;
    const T* pdt = static_cast<const T*>(A.dt) + (first + p) * A.sdt.frame + span.b * A.sdt.sequence + ch;
    const T* pz = A.z && MODE != kSums ? static_cast<const T*>(A.z) + (first + p) * A.sz.frame + span.b * A.sz.sequence + ch : nullptr;
    T* po = MODE == kSums ? nullptr : static_cast<T*>(A.out) + (first + p) * A.so.frame + span.b * A.so.sequence + ch;
    const int64_t du = L * A.su.frame, ddt = L * A.sdt.frame, dz = L * A.sz.frame, dout = L * A.so.frame;
    T un[Q], dn[Q], zn[Q];
    auto load = [&](int64_t at) {                      // the block of frames from `at` on
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const bool in = at + q * L + p < n;
            un[q] = in ? *pu : (T)0.0f;
            dn[q] = in ? *pdt : (T)0.0f;
            if (MODE != kSums) zn[q] = in && pz ? *pz : (T)0.0f;
            pu += du;
            pdt += ddt;
            if (MODE != kSums && pz) pz += dz;
        }
    };
    // b and c of a piece of frames, as they lie in memory
    const T* gb = static_cast<const T*>(A.b) + first * A.sb.frame + span.b * A.sb.sequence + g * A.sb.head;
    const T* gc = static_cast<const T*>(A.c) + first * A.sc.frame + span.b * A.sc.sequence + g * A.sc.head;
    T bn[EACH], cn[EACH];
    auto load_piece = [&](int64_t at) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int x = e * kThreads + threadIdx.x, i = x % NP;
            const int64_t t = at + x / NP;
            const bool in = t < n && i < A.states;
            bn[e] = in ? gb[t * A.sb.frame + i] : (T)0.0f;
            if (MODE != kSums) cn[e] = in ? gc[t * A.sc.frame + i] : (T)0.0f;
        }
    };
    auto keep_piece = [&](int to) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int x = e * kThreads + threadIdx.x;
            sb[to][x / NP][x % NP] = (float)bn[e];
            if (MODE != kSums) sc[to][x / NP][x % NP] = (float)cn[e];
        }
    };

    load_piece(0);
    load(0);
    keep_piece(0);
    __syncthreads();
    double total = 0.0;                                // of r
    int buffer = 0;
    for (int64_t at = 0; at < n; at += PIECE) {
        if (at + PIECE < n) load_piece(at + PIECE);
#pragma unroll 1
        for (int in_piece = 0; in_piece < PIECE && at + in_piece < n; in_piece += kBlock) {
            float r[Q], x[Q], u[Q], z[Q];
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const float s = (float)dn[q] + bias;
                r[q] = A.softplus ? srx::softplus(s) : s;
                u[q] = (float)un[q];
                x[q] = r[q] * u[q];
                if (MODE != kSums) z[q] = (float)zn[q];
            }
            const int64_t t = at + in_piece;
            const int left = (int)min(n - t, (int64_t)kBlock);
            if (t + kBlock < n) load(t + kBlock);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                float y[L];
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    const int f = q * L + i;
                    const float rr = L > 1 ? __shfl_sync(0xFFFFFFFFu, r[q], i * SIDE + lane % SIDE) : r[q];
                    const float xx = L > 1 ? __shfl_sync(0xFFFFFFFFu, x[q], i * SIDE + lane % SIDE) : x[q];
                    y[i] = 0.0f;
                    if (f < left) {
                        const Pair r2 = srx::pair(rr, rr), x2 = srx::pair(xx, xx);
                        Pair y2 = srx::pair(0.0f, 0.0f);
#pragma unroll
                        for (int k = 0; k < K; k += 4) {
                            const float4 bv = *reinterpret_cast<const float4*>(&sb[buffer][in_piece + f][((k / 4) * L + p) * 4]);
                            const float2 e0 = srx::split(srx::mul2(r2, a2[k / 2])), e1 = srx::split(srx::mul2(r2, a2[k / 2 + 1]));
                            h[k / 2] = srx::fma2(srx::pair(srx::ex2(e0.x), srx::ex2(e0.y)), h[k / 2], srx::mul2(x2, srx::pair(bv.x, bv.y)));
                            h[k / 2 + 1] = srx::fma2(srx::pair(srx::ex2(e1.x), srx::ex2(e1.y)), h[k / 2 + 1], srx::mul2(x2, srx::pair(bv.z, bv.w)));
                            if (MODE != kSums) {
                                const float4 cv = *reinterpret_cast<const float4*>(&sc[buffer][in_piece + f][((k / 4) * L + p) * 4]);
                                y2 = srx::fma2(srx::pair(cv.x, cv.y), h[k / 2], y2);
                                y2 = srx::fma2(srx::pair(cv.z, cv.w), h[k / 2 + 1], y2);
                            }
                        }
                        const float2 s = srx::split(y2);
                        y[i] = s.x + s.y;
                    }
                }
                const bool mine = q * L + p < left;
                if (MODE == kSums) {
                    if (mine) total += (double)r[q];
                } else {
                    float o = exchange<L, SIDE>(y, p);
                    o = fmaf(skip, u[q], o);
                    if (pz) o *= srx::silu<EXACT>(z[q]);
                    if (mine && there) *po = (T)o;
                    po += dout;
                }
            }
        }
        if (at + PIECE < n) keep_piece(buffer ^ 1);
        __syncthreads();
        buffer ^= 1;
    }

    float* to = MODE == kSums ? A.sums + (slot * A.channels + ch) * A.states : A.state_out && last ? A.state_out + ((int64_t)b * A.channels + ch) * A.states : nullptr;
    if (to && there) {
#pragma unroll
        for (int k = 0; k < K; k += 2) {
            const int i = ((k / 4) * L + p) * 4 + k % 4;
            const float2 v = srx::split(h[k / 2]);
            if (i < A.states) to[i] = v.x;
            if (i + 1 < A.states) to[i + 1] = v.y;
        }
    }
    if (MODE == kSums) {
#pragma unroll
        for (int s = SIDE; s < 32; s *= 2) total += __shfl_xor_sync(0xFFFFFFFFu, total, s);
        if (there && p == 0) A.steps[slot * A.channels + ch] = (float)total;
    }
}

// The states that enter the segments, from their sums: one thread for a state of a channel of a sequence, over its segments.
__global__ void __launch_bounds__(128) sr_scan_join_kernel(const __grid_constant__ ScanArgs A)
{
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int64_t per = (int64_t)A.channels * A.states, parts = (per + 127) / 128;
    const int b = (int)(blockIdx.x / parts);
    const int64_t slot0 = first_slot(A.offsets, A.frames, A.segment, b), count = segments_of(frame_span(A.offsets, A.frames, b).n, A.segment);
    const int64_t i = (blockIdx.x - b * parts) * 128 + threadIdx.x;
    if (i >= per) return;
    const int64_t ch = i / A.states;
    const float a2 = srx::kLog2e * A.a[i];
    float h = A.state_in ? A.state_in[b * per + i] : 0.0f;
    float* at = A.sums + slot0 * per + i;
    const float* steps = A.steps + slot0 * A.channels + ch;
    constexpr int AHEAD = 8;
    for (int64_t s = 0; s < count; s += AHEAD) {
        float sum[AHEAD], step[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {              // (the last segment's sums are not made)
            const bool in = s + k < count - 1;
            sum[k] = in ? at[k * per] : 0.0f;
            step[k] = in ? steps[k * A.channels] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (s + k >= count) break;
            at[k * per] = h;
            h = fmaf(srx::ex2(a2 * step[k]), h, sum[k]);
        }
        at += AHEAD * per;
        steps += AHEAD * A.channels;
    }
}

// ------------------------------------------------------------------------------------------ single frames
// One frame: the states are read and written once.  L threads have VEC states each of a channel (more where L is 32 already), the warp's other threads the next
// channels; a thread goes over SEQ sequences with the same decays.
template <typename T, int VEC, int SEQ>
__global__ void __launch_bounds__(128) sr_scan_step_kernel(const __grid_constant__ ScanArgs A, int L, int pieces)
{
    constexpr bool EXACT = sizeof(T) == 4;
    srx::let_successor_start();
    srx::wait_for_predecessor();
    const int p = threadIdx.x % L;
    const int parts = (A.channels + 128 / L - 1) / (128 / L);
    const int64_t ch0 = (int64_t)(blockIdx.x % parts) * (128 / L) + threadIdx.x / L;
    const bool there = ch0 < A.channels;
    const int64_t ch = there ? ch0 : 0;
    const int g = (int)(ch / A.share);
    const int b0 = (int)(blockIdx.x / parts) * SEQ;
    const float bias = A.bias ? A.bias[ch] : 0.0f, skip = A.d ? A.d[ch] : 0.0f;
    float u[SEQ], r[SEQ], z[SEQ], y[SEQ];
#pragma unroll
    for (int s = 0; s < SEQ; ++s) {
        const int64_t b = min(b0 + s, A.batch - 1);
        u[s] = (float)static_cast<const T*>(A.u)[b * A.su.sequence + ch];
        r[s] = (float)static_cast<const T*>(A.dt)[b * A.sdt.sequence + ch];
        z[s] = A.z ? (float)static_cast<const T*>(A.z)[b * A.sz.sequence + ch] : 0.0f;
        y[s] = 0.0f;
    }
    for (int k = 0; k < pieces; ++k) {
        const int i = (k * L + p) * VEC;
        const bool in = there && i < A.states;         // (VEC 4: the states are a multiple of 4)
        float a[VEC], h[SEQ][VEC], bv[SEQ][VEC], cv[SEQ][VEC];
        if constexpr (VEC == 4) {
            const float4 v = in ? *reinterpret_cast<const float4*>(A.a + ch * A.states + i) : make_float4(0, 0, 0, 0);
            a[0] = v.x; a[1] = v.y; a[2] = v.z; a[3] = v.w;
        } else {
            a[0] = in ? A.a[ch * A.states + i] : 0.0f;
        }
#pragma unroll
        for (int s = 0; s < SEQ; ++s) {
            const bool is = in && b0 + s < A.batch;
            const int64_t b = min(b0 + s, A.batch - 1);
            const float* state = A.state_out + (b * A.channels + ch) * A.states + i;
            if constexpr (VEC == 4) {
                const float4 v = is ? *reinterpret_cast<const float4*>(state) : make_float4(0, 0, 0, 0);
                h[s][0] = v.x; h[s][1] = v.y; h[s][2] = v.z; h[s][3] = v.w;
            } else {
                h[s][0] = is ? state[0] : 0.0f;
            }
            const T* pb = static_cast<const T*>(A.b) + b * A.sb.sequence + g * A.sb.head + i;
            const T* pc = static_cast<const T*>(A.c) + b * A.sc.sequence + g * A.sc.head + i;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                bv[s][e] = is ? (float)pb[e] : 0.0f;
                cv[s][e] = is ? (float)pc[e] : 0.0f;
            }
        }
        if (k == 0) {
#pragma unroll
            for (int s = 0; s < SEQ; ++s) r[s] = A.softplus ? srx::softplus(r[s] + bias) : r[s] + bias;
        }
#pragma unroll
        for (int s = 0; s < SEQ; ++s) {
            const float x = r[s] * u[s];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                h[s][e] = fmaf(srx::ex2(r[s] * (srx::kLog2e * a[e])), h[s][e], x * bv[s][e]);
                y[s] = fmaf(cv[s][e], h[s][e], y[s]);
            }
            if (in && b0 + s < A.batch) {
                float* state = A.state_out + ((int64_t)(b0 + s) * A.channels + ch) * A.states + i;
                if constexpr (VEC == 4) *reinterpret_cast<float4*>(state) = make_float4(h[s][0], h[s][1], h[s][2], h[s][3]);
                else state[0] = h[s][0];
            }
        }
    }
#pragma unroll
    for (int s = 0; s < SEQ; ++s) {
        for (int d = 1; d < L; d *= 2) y[s] += __shfl_xor_sync(0xFFFFFFFFu, y[s], d);
        float o = fmaf(skip, u[s], y[s]);
        if (A.z) o *= srx::silu<EXACT>(z[s]);
        if (there && p == 0 && b0 + s < A.batch) static_cast<T*>(A.out)[(int64_t)(b0 + s) * A.so.sequence + ch] = (T)o;
    }
}

// ------------------------------------------------------------------------------------------ launches
template <typename F, typename... Args>
cudaError_t start(F* kernel, int64_t blocks, int threads, cudaStream_t s, Args... args)
{
    if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// How a run is cut.
struct ScanCut {
    int held, lanes;
    int64_t segment, slots;                            // 0: whole sequences
};
ScanCut scan_cut(const sr_scan_desc* d, bool packed, int sms)
{
    ScanCut c{};
    int padded = 4;
    while (padded < d->states) padded *= 2;
    c.held = padded < 8 ? 4 : padded > 64 ? 16 : 8;
    c.lanes = padded / c.held;
    (void)packed;
    (void)sms;
    c.slots = d->batch;
    return c;
}
size_t cut_bytes(const sr_scan_desc* d, const ScanCut& c)
{
    return c.segment ? (size_t)c.slots * d->channels * ((size_t)d->states * 4 + 4) + 256 : 0;
}

template <typename T, int K, int L>
cudaError_t launch_scan(const ScanArgs& A, const ScanCut& c, cudaStream_t s)
{
    const int64_t grid = c.slots * A.groups * A.tiles;
    if (!c.segment) return start(sr_scan_kernel<T, K, L, kWhole>, grid, kThreads, s, A);
    cudaError_t e = start(sr_scan_kernel<T, K, L, kSums>, grid, kThreads, s, A);
    if (e == cudaSuccess) e = start(sr_scan_join_kernel, ((int64_t)A.channels * A.states + 127) / 128 * A.batch, 128, s, A);
    if (e == cudaSuccess) e = start(sr_scan_kernel<T, K, L, kOutputs>, grid, kThreads, s, A);
    return e;
}
template <typename T>
cudaError_t launch_scan(const ScanArgs& A, const ScanCut& c, cudaStream_t s)
{
    if (c.held == 4) return launch_scan<T, 4, 1>(A, c, s);
    if (c.held == 16) return launch_scan<T, 16, 8>(A, c, s);
    if (c.lanes == 1) return launch_scan<T, 8, 1>(A, c, s);
    if (c.lanes == 2) return launch_scan<T, 8, 2>(A, c, s);
    if (c.lanes == 4) return launch_scan<T, 8, 4>(A, c, s);
    return launch_scan<T, 8, 8>(A, c, s);
}

template <typename T, int VEC>
cudaError_t launch_step(const ScanArgs& A, cudaStream_t s)
{
    const int units = (A.states + VEC - 1) / VEC;
    int L = 1;
    while (L < 32 && L < units) L *= 2;
    const int pieces = (units + L - 1) / L;
    const int64_t x = (A.channels + 128 / L - 1) / (128 / L);
    if (A.batch >= 16 && VEC == 4) return start(sr_scan_step_kernel<T, VEC, 4>, x * ((A.batch + 3) / 4), 128, s, A, L, pieces);
    return start(sr_scan_step_kernel<T, VEC, 1>, x * A.batch, 128, s, A, L, pieces);
}
template <typename T>
cudaError_t launch_step(const ScanArgs& A, cudaStream_t s)
{
    return A.states % 4 == 0 && !((uintptr_t)A.state_out & 15) && !((uintptr_t)A.a & 15) ? launch_step<T, 4>(A, s) : launch_step<T, 1>(A, s);
}

// ------------------------------------------------------------------------------------------ checks
bool fits(const sr_frame_strides& s) { return s.frame >= 0 && s.sequence >= 0; }
bool fits(const sr_attention_strides& s) { return s.frame >= 0 && s.sequence >= 0 && s.head >= 0; }

sr_status check(const sr_scan_desc* d)
{
    if (!d || (d->dtype != SR_DTYPE_F32 && d->dtype != SR_DTYPE_BF16) || d->batch < 0 || d->channels < 1 || d->states < 1 || d->groups < 1 ||
        d->channels % d->groups || d->frames < 0 || (d->softplus != 0 && d->softplus != 1) || !fits(d->u) || !fits(d->dt) || !fits(d->z) || !fits(d->out) || !fits(d->b) ||
        !fits(d->c))
        return SR_ERR_INVALID_ARG;
    if (d->states > 128) return SR_ERR_UNSUPPORTED;
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
    const ScanCut cut = scan_cut(d, offsets != nullptr, sr_device_sms());
    const size_t needed = cut_bytes(d, cut);
    if (needed && (!workspace || workspace_bytes < needed || ((uintptr_t)workspace & 255))) return SR_ERR_INVALID_ARG;
    A.offsets = offsets;
    A.state_in = state_in;
    A.state_out = state_out;
    A.segment = cut.segment;
    A.sums = static_cast<float*>(workspace);
    A.steps = A.sums + cut.slots * d->channels * d->states;
    const int per = kThreads / cut.lanes;
    A.tiles = (A.share + per - 1) / per;
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
    if (!tensors(d, A, u, dt, a, b, c, skip, z, bias, out) || !state || ((uintptr_t)state & 3)) return SR_ERR_INVALID_ARG;
    A.state_out = state;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d->dtype == SR_DTYPE_F32 ? launch_step<float>(A, s) : launch_step<__nv_bfloat16>(A, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
