// Linear attention over whole clips in bf16, chunk by chunk of 128 frames on the tensor cores.
//
// With G_i the sum of the log decays from a chunk's start up to frame i of it, S the state that enters the chunk and i, j frames of the chunk,
//     out_i = scale * ( exp(G_i) q_i S + sum_{j <= i} exp(G_i - G_j) (q_i . k_j) v_j ),
//     S'    = exp(G_last) S + sum_j k_j (exp(G_last - G_j) v_j)^T:
// four matrix products per chunk and group of 64 columns of v (the last one a CTA's: it holds DK x 64 values of a state), all of them tcgen05.mma
// with M = 128:
//   scores  Q K^T              128 frames x 128 frames, both from shared memory                       (TMEM columns 0 .. 127)
//   near    (P_hi + P_lo) V    P = scores * decays, lower triangle, in two bf16 parts, back in TMEM as the A operand (columns 448 .. 511 and 256 .. 319, sums
//                              in 384 .. 447)
//   far     Q (S_hi + S_lo)    the state in two bf16 parts for this product                           (columns 320 .. 383)
//   state   K^T V', V' = V exp(G_last - G_j) in three bf16 parts, 24 bits: the state itself is as exact as 32 bits make it.  Two accumulators side by
//                              side (columns 128 .. 255), the decayed state with the first parts' sums and the sums of the others, added up once per chunk
// Sums of segments, whose state nothing reads, leave it alone until the end: their chunks go from the last to the first, values weighted by all the decays behind them.
// They have three accumulators, one to each part, and one MMA for all of them.
// K is read along both of its sides from the same tile.  Nothing but the outputs is rounded to bf16 once: two parts hold a factor to 2^-16 of itself, so that the outputs are as far
// off as their own rounding makes them (1.7e-3 of their size; with one part each 2.3e-3).  Us with one part each / two: 32 clips of 128 frames, 8 heads of 64 16.4 / 17.8; packed 16 of 3000,
// 16 heads on 4 of 128 301 / 324; one of 32768, 8 heads of 128 153 / 170; 1024 frames x 37, 8 heads on 2 of 128 67 / 84.
// Decays never exceed one: exp(G_i - G_j) is a product of exp(G_i - G_e) and exp(G_e - G_j) with e the last frame of j's 32, where i lies behind them, and
// one exponential where it does not.  G is summed in 64 bits and held in two floats, so that a frame that forgets everything costs the ones behind it nothing.
//
// A chunk of DK = 128 is 96 KiB of loads and stores and 2.9k cycles of MMAs per CTA, 2.2k cycles' worth of memory with every SM at it, and takes 6.6k (4096 frames, 148 CTAs:
// 112 us, 2.8 TB/s; without the MMAs of the second parts 99, without its stores 108); further heads of the chunk about 2 us each (1024 frames x 37, 8 heads on 2: 84 us; 79 and 79).  What bounds it is the
// chain from scores over weights to outputs, which workers (four warps to a scheduler, kept in step by the barriers) and MMAs go along in turn; two CTAs to an SM do not fit (209 KiB of tiles, all
// of TMEM).  Not faster, with one part each: roles of their own for the workers (128 us instead of 91), the state in registers instead of TMEM (91); persistent CTAs gained only where sequences are
// a chunk long (32 clips of 128 frames 14.8 -> 13.7; packed sequences 90 -> 124, 116 -> 194).
// Roles: warp 0 copies, 1 MMAs, 2 decays, 3 TMEM; sixteen workers for everything between the MMAs.
// What is not finite stays where the formula has it: scores behind the diagonal are replaced, not multiplied; a value of v that is not finite is taken out of
// the near product (whose zeros would spread it to earlier frames) and added where the outputs are stored; rows behind a sequence's last frame are zeroed.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>

#include "sr_memory.h"
#include "sr_operators.h"
#include "sr_pair.cuh"
#include "sr_ptx.cuh"

namespace {
using namespace srx;

constexpr int kChunk = 128, kCols = 64, kDecays = 4;
constexpr int kWorkers = 16, kThreads = 128 + 32 * kWorkers;
constexpr uint32_t kScores = 0, kState = 128, kRest = 256, kFar = 320, kNear = 384, kWeights = 448;      // TMEM columns
constexpr float kLn2 = 0.6931471805599453f;

struct ChunkArgs {
    CUtensorMap q_map, k_map, v_map;
    SegmentArgs S;
    int32_t out_align;                                 // bytes on which a row's pieces of 16 outputs start: 32, 16 or 0 (any)
    int* error;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float exp2_two(double x)   // 2^x, x as two floats
{
    const float hi = (float)x, lo = (float)(x - (double)hi);
    const float y = exp2_fast(hi);
    return fmaf(y, lo * kLn2, y);
}
// What rounding a pair to bf16 left over, rounded, and the halves of a word of bf16 that are finite
__device__ __forceinline__ uint32_t left_bf16(Pair y, uint32_t rounded) { return round_bf16(fma2(widen_bf16(rounded), pair(-1.0f, -1.0f), y)); }
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) { return ((w & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u); }
__device__ __forceinline__ void store_32_bytes(void* to, const uint32_t (&z)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "r"(z[0]), "r"(z[1]), "r"(z[2]), "r"(z[3]), "r"(z[4]), "r"(z[5]), "r"(z[6]), "r"(z[7]) : "memory");
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

struct alignas(16) Decays {                            // of a chunk (read four at a time); G in units of log 2
    float hi[kChunk], lo[kChunk];                      // G_j in two floats
    float col[kChunk];                                 // exp(G_e - G_j), e the last frame of j's 32
    float rest[kChunk];                                // exp(G_last - G_j)
    float row[kChunk];                                 // exp(G_i)
    float whole;                                       // exp(G_last)
    uint32_t odd;                                      // 1: some of the chunk's values are not finite
};
static_assert(sizeof(Decays) % 16 == 0, "read as 16-byte words");

// What follows is out of line: it is rarely run, and the loop that every chunk goes through has to stay small.

// 16 outputs of row i of a chunk, one by one.  odd: values that are not finite have been left out of the chunk's near product; their terms as the formula has
// them go on top of the stored outputs (what comes out is not finite, so the outputs' rounding does not matter).
__device__ __noinline__ void store_row(const AttentionArgs& A, const Decays& D, const AttentionItem& it, int64_t f0, int i, int h, int c0, bool odd, uint4 lo, uint4 hi)
{
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + it.span.b * A.so.sequence + (f0 + i) * A.so.frame + ((int64_t)it.g * A.share + h) * A.so.head + c0;
    const uint32_t z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (c0 + e < A.dv) out[e] = __ushort_as_bfloat16((unsigned short)(e & 1 ? z[e / 2] >> 16 : z[e / 2] & 0xFFFFu));
    if (!odd) return;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(A.q) + it.span.b * A.sq.sequence + (f0 + i) * A.sq.frame + ((int64_t)it.g * A.share + h) * A.sq.head;
#pragma unroll 1
    for (int j = 0; j <= i; ++j) {
        const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(A.v) + it.span.b * A.sv.sequence + (f0 + j) * A.sv.frame + (int64_t)it.g * A.sv.head + c0;
        const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(A.k) + it.span.b * A.sk.sequence + (f0 + j) * A.sk.frame + (int64_t)it.g * A.sk.head;
        float p = 0.0f;
        bool have = false;
#pragma unroll 1
        for (int e = 0; e < 16 && c0 + e < A.dv; ++e) {
            const float value = __bfloat162float(v[e]);
            if (finite(value)) continue;
            if (!have) {
                for (int t = 0; t < A.dk; ++t) p = fmaf(__bfloat162float(q[t]), __bfloat162float(k[t]), p);
                p *= exp2_fast((D.hi[i] - D.hi[j]) + (D.lo[i] - D.lo[j])) * A.scale;
                have = true;
            }
            out[e] = __float2bfloat16(__bfloat162float(out[e]) + p * value);
        }
    }
}
// Takes what is not finite out of a thread's 16 values.
__device__ __noinline__ void clear_odd(uint4* first, uint4* second)
{
#pragma unroll 1
    for (int e = 0; e < 16; ++e) {
        uint16_t* p = reinterpret_cast<uint16_t*>(e < 8 ? first : second) + (e & 7);
        if ((*p & 0x7F80u) == 0x7F80u) *p = 0;
    }
}
// 16 values of a state's row between global memory and two TMEM lanes' registers.
__device__ __noinline__ void load_state(const float* from, int j0, int dv, uint32_t taddr)
{
    uint32_t x[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = from && j0 + e < dv ? __float_as_uint(from[j0 + e]) : 0u;
    __syncwarp();
    tc_st(taddr, x);
}
template <int ACCS>
__device__ __noinline__ void store_state(float* to, int j0, int dv, uint32_t taddr)
{
    uint32_t x0[16], x1[16], x2[16];
    if constexpr (ACCS == 3) tc_ld(taddr, taddr + kCols, taddr + 2 * kCols, x0, x1, x2);
    else tc_ld(taddr, taddr + kCols, x0, x1);
    if (!to) return;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float more = ACCS == 3 ? __uint_as_float(x1[e]) + __uint_as_float(x2[e]) : __uint_as_float(x1[e]);
        x0[e] = __float_as_uint(__uint_as_float(x0[e]) + more);
    }
    if (j0 + 16 <= dv && !((uintptr_t)(to + j0) & 15)) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(to + j0 + e) = make_uint4(x0[e], x0[e + 1], x0[e + 2], x0[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (j0 + e < dv) to[j0 + e] = __uint_as_float(x0[e]);
    }
}

template <int DK, int MODE>
constexpr int kKeySlots = DK == 64 || MODE == 1 ? 2 : 1;

// MODE 0: whole sequences; 1: sums of segments; 2: outputs of segments.
template <int DK, int MODE>
__global__ void __launch_bounds__(kThreads, 1) sr_chunks_kernel(const __grid_constant__ ChunkArgs C)
{
    constexpr bool OUT = MODE != 1;                    // outputs are wanted
    constexpr int NK = kKeySlots<DK, MODE>, NW = OUT ? 1 : 2;          // slots for keys, for the parts of values
    constexpr int KT = DK * 256, VT = kCols * 256, ST = DK * 128;        // bytes of a tile of K or Q, of V (or outputs), of the state
    constexpr int SQ = DK / 32;                        // quarters of the TMEM lanes with rows of the state
    extern __shared__ uint8_t smem_raw[];
    __shared__ Decays decays[kDecays];
    __shared__ uint64_t bars[32];
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_flag;
    const AttentionArgs& A = C.S.A;
    volatile int* gave_up = &gave_up_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wait_for_predecessor();
    const AttentionItem it = attention_item(C.S, MODE != 0, kCols);
    if (!it.there || (MODE == 1 && it.last)) return;
    const int64_t state_at = ((int64_t)it.b * A.groups + it.g) * A.dk;
    const int64_t slot_at = ((int64_t)it.slot * A.groups + it.g) * A.dk;
    if (it.n == 0) {                                   // an empty sequence hands its state through
        if (A.state_out && MODE != 1)
            for (int i = threadIdx.x; i < A.dk * kCols; i += kThreads) {
                const int r = i / kCols, j = it.c0 + i % kCols;
                if (j < A.dv) A.state_out[(state_at + r) * A.dv + j] = A.state_in ? A.state_in[(state_at + r) * A.dv + j] : 0.0f;
            }
        return;
    }
    const int chunks = (int)((it.n + kChunk - 1) / kChunk);
    const int share = OUT ? A.share : 1;

    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t k_tiles = base, v_tiles = k_tiles + NK * KT, q_tiles = v_tiles + 2 * VT, w_tiles = q_tiles + (OUT ? 2 * KT : 0), s_tiles = w_tiles + 3 * VT;
    uint8_t* const k_mem = smem_raw + (base - smem_u32(smem_raw));
    uint8_t *const v_mem = k_mem + NK * KT, *const w_first = v_mem + 2 * VT + (OUT ? 2 * KT : 0), *const s_mem = w_first + 3 * VT;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    const uint32_t k_full = bar(0), k_empty = bar(2), v_full = bar(4), v_empty = bar(6), q_full = bar(8), q_empty = bar(10), d_full = bar(12), d_empty = bar(16);
    const uint32_t scored = bar(20), weighed = bar(21), answered = bar(22), taken = bar(24);
    const uint32_t cleaned = bar(26);
    // The sums alone, which no state goes through, are a chunk ahead: two of each of these in turn.
    auto parted = [&](int c) { return bar(!OUT && (c & 1) ? 29 : 25); };
    auto summed = [&](int c) { return bar(!OUT && (c & 1) ? 30 : 27); };
    auto turn = [](int c) { return (uint32_t)(OUT ? c : c >> 1) & 1u; };
    if (threadIdx.x == 0) {
        gave_up_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(k_empty + 8 * i, 1);
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_empty + 8 * i, 1);
            mbar_init(q_full + 8 * i, 1);
            mbar_init(q_empty + 8 * i, 1);
        }
        for (int i = 0; i < kDecays; ++i) {
            mbar_init(d_full + 8 * i, 1);
            mbar_init(d_empty + 8 * i, kWorkers);
        }
        mbar_init(scored, 1);                          // scores are in TMEM
        mbar_init(weighed, kWorkers);                  // P is in TMEM
        mbar_init(answered, 1);                        // the last step's outputs are in TMEM
        mbar_init(taken, kWorkers);                    // a step's outputs have been read
        mbar_init(bar(25), kWorkers);                  // V' is in shared memory, V is fit for the near product, the state in TMEM has decayed
        mbar_init(bar(27), 1);                         // the chunk's sums are on top of the state, V' has been read
        mbar_init(bar(29), kWorkers);
        mbar_init(bar(30), 1);
        mbar_init(cleaned, kWorkers);                  // rows behind the last frame are zeroed
        mbar_init_done();
    }
    if (warp == 3) tmem_alloc(smem_u32(&tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    let_successor_start();
    const uint32_t tmem = tmem_slot;
    const int64_t f0 = it.span.first + it.t0;          // first frame
    const int tail = (int)(it.n - (int64_t)(chunks - 1) * kChunk);       // frames of the last chunk
    // Behind the last frame: zeros (the tensor's end), or frames of another packed sequence, which have to be.  (Chunks of a segment are full unless the
    // sequence ends there.)
    const bool clean = A.offsets && tail < kChunk;

    if (warp == 0) {
        if (elect_one()) {
            bool ok = true;
            uint32_t n = 0;                            // steps: chunks x heads
            auto frame = [&](int c) { return (int)(f0 + (int64_t)(OUT ? c : chunks - 1 - c) * kChunk); };
            auto load_q = [&](int c, int h) {
                const uint32_t s = n & 1, b = q_full + 8 * s;
                ok = ok && mbar_wait(q_empty + 8 * s, ((n >> 1) & 1) ^ 1, gave_up);
                if (!ok) return;
                mbar_expect_tx(b, KT);
#pragma unroll
                for (int p = 0; p < DK / 64; ++p) tma_load_4d(q_tiles + s * KT + p * 16384, &C.q_map, b, p * 64, it.g * A.share + h, (int)it.span.b, frame(c));
                ++n;
            };
            for (int c = 0; c < chunks && ok; ++c) {
                const uint32_t vs = c & 1, ks = c % NK;
                ok = mbar_wait(v_empty + 8 * vs, ((c >> 1) & 1) ^ 1, gave_up);
                if (!ok) break;
                mbar_expect_tx(v_full + 8 * vs, VT);
                tma_load_4d(v_tiles + vs * VT, &C.v_map, v_full + 8 * vs, it.c0, it.g, (int)it.span.b, frame(c));
                if (OUT) load_q(c, 0);
                ok = ok && mbar_wait(k_empty + 8 * ks, ((c / NK) & 1) ^ 1, gave_up);
                if (!ok) break;
                mbar_expect_tx(k_full + 8 * ks, KT);
#pragma unroll
                for (int p = 0; p < DK / 64; ++p) {
                    tma_load_4d(k_tiles + ks * KT + p * 16384, &C.k_map, k_full + 8 * ks, p * 64, it.g, (int)it.span.b, frame(c));
                    if (NK == 1 && c + 1 < chunks) tma_prefetch_4d(&C.k_map, p * 64, it.g, (int)it.span.b, frame(c + 1));
                }
                for (int h = 1; h < share && OUT; ++h) load_q(c, h);
            }
            if (!ok)                                   // what was asked for still has to land
                for (int s = 0; s < 2; ++s)
                    for (int p = 0; p < 2; ++p) {
                        mbar_drain(k_full + 8 * s, p);
                        mbar_drain(v_full + 8 * s, p);
                        mbar_drain(q_full + 8 * s, p);
                    }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            constexpr uint32_t i_scores = idesc_bf16(128, 0, 0), i_far = idesc_bf16(64, 0, 1), i_near = idesc_bf16(64, 0, 1), i_state = idesc_bf16(OUT ? 64 : 192, 1, 1);
            bool ok = true;
            uint32_t n = 0;
            // Scores of step m, the first of chunk c's if h is 0.
            auto scores = [&](uint32_t m, int c, int h) {
                const uint32_t q_at = q_tiles + (m & 1) * KT, k_at = k_tiles + (c % NK) * KT;
                if (h == 0) {
                    ok = ok && mbar_wait(k_full + 8 * (c % NK), (c / NK) & 1, gave_up);
                    if (clean && c + 1 == chunks) ok = ok && mbar_wait(cleaned, 0, gave_up);
                }
                if (OUT) {
                    ok = ok && mbar_wait(q_full + 8 * (m & 1), (m >> 1) & 1, gave_up);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < DK / 16; ++k)
                        mma_bf16(tmem + kScores, desc_k_major(q_at + (k / 4) * 16384) + 2 * (k % 4), desc_k_major(k_at + (k / 4) * 16384) + 2 * (k % 4), i_scores, k > 0);
                    tc_commit(scored);
                }
            };
            scores(0, 0, 0);
            for (int c = 0; c < chunks && ok; ++c) {
                const uint32_t k_at = k_tiles + (c % NK) * KT, v_at = v_tiles + (c & 1) * VT;
                const int steps = ((c + 1 == chunks ? tail : kChunk) + 15) / 16;        // of 16 frames
                // the state first: the next chunk waits for it
                ok = mbar_wait(parted(c), turn(c), gave_up);
                if (!ok) break;
                tc_fence_after();
                for (int k = 0; k < steps; ++k) {
                    const uint64_t keys = desc_mn_major(k_at + k * 2048, DK == 64 ? 0 : 16384);
                    const uint32_t parts = w_tiles + (c % NW) * 3 * VT + k * 2048;
                    if (OUT) {
#pragma unroll
                        for (int p = 0; p < 3; ++p) mma_bf16(tmem + kState + (p ? kCols : 0), keys, desc_mn_major(parts + p * VT, 0), i_state, 1);
                    } else {
                        mma_bf16(tmem + kState, keys, desc_mn_major(parts, VT), i_state, 1);
                    }
                }
                tc_commit(summed(c));
                if (share == 1) tc_commit(k_empty + 8 * (c % NK));
                for (int h = 0; h < share && ok; ++h, ++n) {
                    if (OUT) {
                        const uint32_t q_at = q_tiles + (n & 1) * KT;
                        ok = mbar_wait(taken, (n & 1) ^ 1, gave_up);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int k = 0; k < DK / 16; ++k)
                            for (int p = 0; p < 2; ++p)
                                mma_bf16(tmem + kFar, desc_k_major(q_at + (k / 4) * 16384) + 2 * (k % 4), desc_mn_major(s_tiles + p * ST + k * 2048, 0), i_far, k > 0 || p > 0);
                        tc_commit(q_empty + 8 * (n & 1));
                        ok = mbar_wait(weighed, n & 1, gave_up);
                        if (!ok) break;
                        tc_fence_after();
                        for (int k = 0; k < steps; ++k) {
                            mma_bf16_ta(tmem + kNear, tmem + kWeights + k * 8, desc_mn_major(v_at + k * 2048, 0), i_near, k > 0);
                            mma_bf16_ta(tmem + kNear, tmem + kRest + k * 8, desc_mn_major(v_at + k * 2048, 0), i_near, 1);
                        }
                        if (c + 1 == chunks && h + 1 == share) tc_commit(answered);
                    }
                    if (h + 1 == share) tc_commit(v_empty + 8 * (c & 1));
                    if (h + 1 < share) {
                        scores(n + 1, c, h + 1);
                        if (h + 2 == share) tc_commit(k_empty + 8 * (c % NK));
                    } else if (c + 1 < chunks) {
                        scores(n + 1, c + 1, 0);
                    }
                }
            }
        }
    } else if (warp == 2) {
        // decays of chunk after chunk, a few chunks ahead of the others
        double carry = 0.0;                            // what the decays of whole chunks have lost by rounding, relative
        const float* d = A.decay + it.span.b * A.sd.sequence + (int64_t)it.g * A.sd.head;
        double log_whole = 0.0;
        auto load = [&](int c, float (&x)[4]) {
            const int n = c + 1 == chunks ? tail : kChunk;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = lane * 4 + e;
                x[e] = c < chunks && j < n ? d[(f0 + (int64_t)(OUT ? c : chunks - 1 - c) * kChunk + j) * A.sd.frame] : 0.0f;
            }
        };
        float next[4];
        load(0, next);
        for (int c = 0; c < chunks; ++c) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = next[e] < -128.0f ? -128.0f : next[e];    // (exp(-128) is zero in 32 bits; sums of infinities would be NaN)
            load(c + 1, next);
            constexpr double l2e = 1.4426950408889634074;
            double g[4];
            g[0] = (double)x[0];
#pragma unroll
            for (int e = 1; e < 4; ++e) g[e] = g[e - 1] + (double)x[e];
            double before = g[3];
#pragma unroll
            for (int m = 1; m < 32; m *= 2) {
                const double up = __shfl_up_sync(0xFFFFFFFFu, before, m);
                if (lane >= m) before += up;
            }
            const double total = __shfl_sync(0xFFFFFFFFu, before, 31);
            before = __shfl_up_sync(0xFFFFFFFFu, before, 1);             // (not by subtraction: a NaN would reach the lane's frames ahead of it)
            if (lane == 0) before = 0.0;
            const double behind = OUT ? 0.0 : log_whole * l2e;           // (sums alone, from the last chunk to the first: the decays of the chunks behind this one)
            log_whole += total;
            const double last = total * l2e;
            double mine[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[e] = (before + g[e]) * l2e;
            const double block_end = __shfl_sync(0xFFFFFFFFu, mine[3], lane | 7);
            const double exact = exp2(last) * (1.0 + carry);
            const float rounded = (float)exact;
            carry = rounded > 1e-30f ? exact / (double)rounded - 1.0 : 0.0;
            const int slot = c % kDecays;
            if (!mbar_wait_warp(d_empty + 8 * slot, ((c / kDecays) & 1) ^ 1, gave_up)) break;
            Decays& D = decays[slot];
            float4 hi, lo, col, rest, row;
            auto fill = [&](double x, float& h, float& l, float& a, float& b, float& y) {
                b = exp2_two(last - x + behind);
                if (!OUT) return;
                h = (float)x;
                l = (float)(x - (double)h);
                a = exp2_two(block_end - x);
                y = exp2_two(x);
            };
            fill(mine[0], hi.x, lo.x, col.x, rest.x, row.x);
            fill(mine[1], hi.y, lo.y, col.y, rest.y, row.y);
            fill(mine[2], hi.z, lo.z, col.z, rest.z, row.z);
            fill(mine[3], hi.w, lo.w, col.w, rest.w, row.w);
            reinterpret_cast<float4*>(D.rest)[lane] = rest;
            if (OUT) {
                reinterpret_cast<float4*>(D.hi)[lane] = hi;
                reinterpret_cast<float4*>(D.lo)[lane] = lo;
                reinterpret_cast<float4*>(D.col)[lane] = col;
                reinterpret_cast<float4*>(D.row)[lane] = row;
            }
            if (OUT && lane == 0) {
                D.whole = rounded;
                D.odd = 0;
            }
            // (the workers wait for both at once)
            if (!mbar_wait_warp(v_full + 8 * (c & 1), (c >> 1) & 1, gave_up)) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(d_full + 8 * slot);
        }
        if (MODE == 1 && lane == 0 && it.c0 == 0) C.S.decays[(int64_t)it.slot * A.groups + it.g] = (float)exp(log_whole);
    } else if (warp >= 4) {
        // A worker has 32 rows (those of its quarter w of the TMEM lanes) and a quarter u of the columns of everything: frames' rows of V', of the scores and of the
        // outputs, rows of the state.  All of them do the same at the same time: warps with roles of their own, each with a loop of a few hundred
        // instructions, waited for instructions a third of their time (4096 frames, 148 CTAs of DK = 128: 128 us, and 92).  While the tensor pipe sums a chunk's
        // state they do the outputs of the step before, the weights of this one and the parts of the next chunk's values.
        const int w = warp & 3, u = (warp - 4) >> 2, i = w * 32 + lane, j0 = it.c0 + u * 16;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        const bool holds = w < SQ;                     // rows of the state
        const Pair minus = pair(-1.0f, -1.0f);
        const uint32_t place0 = (uint32_t)i * 128u + (((uint32_t)(2 * u) ^ (i & 7)) << 4), place1 = (uint32_t)i * 128u + (((uint32_t)(2 * u + 1) ^ (i & 7)) << 4);
        uint32_t n = 0;                                // steps: chunks x heads
        // Outputs of the step before, in two parts: out of the accumulators, which the MMAs wait for, and, behind this step's weights, on their way.
        uint32_t z[8];
        auto take = [&](int c) {
            uint32_t a[16], x[16];
            tc_ld(tmem + lanes + kFar + u * 16, tmem + lanes + kNear + u * 16, a, x);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(taken);
            const float r = decays[c % kDecays].row[i] * A.scale;
            const Pair row = pair(r, r), scale = pair(A.scale, A.scale);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = round_bf16(fma2(pair(x[2 * e], x[2 * e + 1]), scale, mul2(row, pair(a[2 * e], a[2 * e + 1]))));
        };
        auto store = [&](int c, int h) {
            const Decays& D = decays[c % kDecays];
            const bool odd = D.odd != 0;
            const int64_t f = f0 + (int64_t)c * kChunk;
            if (i >= (c + 1 == chunks ? tail : kChunk)) return;
            if (C.out_align && !odd && j0 + 16 <= A.dv) {
                // 32 bytes of a row, a whole sector of memory: in two stores packed sequences 336 us instead of 324
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(A.out) + it.span.b * A.so.sequence + (f + i) * A.so.frame + ((int64_t)it.g * A.share + h) * A.so.head + j0;
                if (C.out_align == 32) {
                    store_32_bytes(out, z);
                } else {
                    *reinterpret_cast<uint4*>(out) = make_uint4(z[0], z[1], z[2], z[3]);
                    *reinterpret_cast<uint4*>(out + 8) = make_uint4(z[4], z[5], z[6], z[7]);
                }
            } else {
                store_row(A, D, it, f, i, h, j0, odd, make_uint4(z[0], z[1], z[2], z[3]), make_uint4(z[4], z[5], z[6], z[7]));
            }
        };
        // Ahead of the first chunk: the state in the first of its two accumulators, zeros in the other and for the weights behind the diagonal.
        const uint32_t state = tmem + kState + lanes + u * 16;
        const uint32_t none[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        if (holds) {
            const float* from = MODE == 1 || i >= A.dk ? nullptr : MODE == 2 ? C.S.sums + (slot_at + i) * A.dv : A.state_in ? A.state_in + (state_at + i) * A.dv : nullptr;
            load_state(from, j0, A.dv, state);
            __syncwarp();
            tc_st(state + kCols, none);
            if (!OUT) tc_st(state + 2 * kCols, none);
        }
        if (OUT && u > w) {
            tc_st(tmem + kWeights + lanes + u * 16, none);
            tc_st(tmem + kRest + lanes + u * 16, none);
        }
        tc_wait_st();
        bool ok = true;
        for (int c = 0; c < chunks; ++c) {
            const int slot = c % kDecays, frames = c + 1 == chunks ? tail : kChunk;
            Decays& D = decays[slot];
            uint32_t a[8], b[8], d[8];                 // parts of V'
            uint8_t* const v = v_mem + (c & 1) * VT;
            ok = mbar_wait_warp(d_full + 8 * slot, (c / kDecays) & 1, gave_up);          // decays and values
            if (clean && c + 1 == chunks) {
                ok = ok && mbar_wait_warp(k_full + 8 * (c % NK), (c / NK) & 1, gave_up);
                if (!ok) break;
                if (i >= tail) {
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4*>(v + place0) = zero;
                    *reinterpret_cast<uint4*>(v + place1) = zero;
                    for (int p = 0; p < DK / 64; ++p) {
                        *reinterpret_cast<uint4*>(k_mem + (c % NK) * KT + p * 16384 + place0) = zero;
                        *reinterpret_cast<uint4*>(k_mem + (c % NK) * KT + p * 16384 + place1) = zero;
                    }
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) mbar_arrive(cleaned);
            }
            if (!ok) break;
            const Pair weight = pair(D.rest[i], D.rest[i]);
            __nv_bfloat162 odd = __floats2bfloat162_rn(0.0f, 0.0f);      // NaN as soon as a value is not finite
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint4 x = *reinterpret_cast<const uint4*>(v + (q ? place1 : place0));
                const uint32_t in[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (OUT) odd = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&in[e]), __floats2bfloat162_rn(0.0f, 0.0f), odd);
                    Pair y = mul2(widen_bf16(in[e]), weight);
                    a[4 * q + e] = round_bf16(y);
                    y = fma2(widen_bf16(a[4 * q + e]), minus, y);
                    b[4 * q + e] = round_bf16(y);
                    d[4 * q + e] = round_bf16(fma2(widen_bf16(b[4 * q + e]), minus, y));
                }
            }
            if (OUT && __any_sync(0xFFFFFFFFu, *reinterpret_cast<uint32_t*>(&odd) & 0x7FFF7FFFu)) {
                clear_odd(reinterpret_cast<uint4*>(v + place0), reinterpret_cast<uint4*>(v + place1));
#pragma unroll
                for (int e = 0; e < 8; ++e) {                            // the first part says what has to be said; what is left over is NaN
                    const uint32_t keep = finite_halves(b[e]);
                    b[e] &= keep;
                    d[e] &= keep;
                }
                D.odd = 1;
            }
            if (c >= NW) {
                ok = mbar_wait_warp(summed(c - NW), turn(c - NW), gave_up);
                if (!ok) break;
                tc_fence_after();
            }
            uint8_t* const w_mem = w_first + (c % NW) * 3 * VT;
            *reinterpret_cast<uint4*>(w_mem + place0) = make_uint4(a[0], a[1], a[2], a[3]);
            *reinterpret_cast<uint4*>(w_mem + place1) = make_uint4(a[4], a[5], a[6], a[7]);
            *reinterpret_cast<uint4*>(w_mem + VT + place0) = make_uint4(b[0], b[1], b[2], b[3]);
            *reinterpret_cast<uint4*>(w_mem + VT + place1) = make_uint4(b[4], b[5], b[6], b[7]);
            *reinterpret_cast<uint4*>(w_mem + 2 * VT + place0) = make_uint4(d[0], d[1], d[2], d[3]);
            *reinterpret_cast<uint4*>(w_mem + 2 * VT + place1) = make_uint4(d[4], d[5], d[6], d[7]);
            if (OUT && holds) {
                // the state that enters the chunk is the sum of its two accumulators
                uint32_t x0[16], x1[16];
                tc_ld(state, state + kCols, x0, x1);
                const Pair whole = pair(D.whole, D.whole);
                uint32_t part[8], rest[8];             // the state that enters the chunk in two parts
                __nv_bfloat162 far = __floats2bfloat162_rn(0.0f, 0.0f);  // NaN as soon as a value is not finite
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Pair y = add2(pair(x0[2 * e], x0[2 * e + 1]), pair(x1[2 * e], x1[2 * e + 1]));
                    part[e] = round_bf16(y);
                    rest[e] = left_bf16(y, part[e]);
                    far = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&part[e]), __floats2bfloat162_rn(0.0f, 0.0f), far);
                    const float2 z = split(mul2(y, whole));
                    x0[2 * e] = __float_as_uint(z.x);
                    x0[2 * e + 1] = __float_as_uint(z.y);
                }
                if (__any_sync(0xFFFFFFFFu, *reinterpret_cast<uint32_t*>(&far) & 0x7FFF7FFFu)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) rest[e] &= finite_halves(part[e]);       // (the first part says what has to be said)
                }
                tc_st(state, x0);
                tc_st(state + kCols, none);
                // (the far products that read the one before are long done)
                if (c > 0) ok = mbar_wait_warp(q_empty + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1, gave_up);
                if (!ok) break;
                *reinterpret_cast<uint4*>(s_mem + place0) = make_uint4(part[0], part[1], part[2], part[3]);
                *reinterpret_cast<uint4*>(s_mem + place1) = make_uint4(part[4], part[5], part[6], part[7]);
                *reinterpret_cast<uint4*>(s_mem + ST + place0) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
                *reinterpret_cast<uint4*>(s_mem + ST + place1) = make_uint4(rest[4], rest[5], rest[6], rest[7]);
                tc_wait_st();
            }
            fence_async_shared();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(parted(c));
            if (!OUT) {
                if (lane == 0) mbar_arrive(d_empty + 8 * slot);
                continue;
            }
            for (int h = 0; h < share && ok; ++h, ++n) {
                // (the scores come behind the products of the step before: with them that step's outputs are there)
                ok = mbar_wait_warp(scored, n & 1, gave_up);
                if (!ok) break;
                tc_fence_after();
                if (n > 0) take(h > 0 ? c : c - 1);
                // scores -> P: two workers of a quarter have 16 columns of the diagonal's 32 each, the other two 16 of all 32s to its left
                const float hi = D.hi[i], lo = D.lo[i];
                const int half = (u & 1) * 16;
                if (u < 2) {
                    if (w * 32 < frames) {
                        const int c0 = w * 32 + half, far = lane - half;         // columns up to the diagonal
                        const Pair hi2 = pair(hi, hi), lo2 = pair(lo, lo);
                        uint32_t s[16], p[8], rest[8];
                        tc_ld(tmem + kScores + lanes + c0, s);
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const ulonglong2 gh = *reinterpret_cast<const ulonglong2*>(&D.hi[c0 + 2 * e]), gl = *reinterpret_cast<const ulonglong2*>(&D.lo[c0 + 2 * e]);
                            const float2 g0 = split(add2(fma2(gh.x, minus, hi2), fma2(gl.x, minus, lo2))), g1 = split(add2(fma2(gh.y, minus, hi2), fma2(gl.y, minus, lo2)));
                            const float2 z0 = split(mul2(pair(s[2 * e], s[2 * e + 1]), pair(exp2_fast(g0.x), exp2_fast(g0.y))));
                            const float2 z1 = split(mul2(pair(s[2 * e + 2], s[2 * e + 3]), pair(exp2_fast(g1.x), exp2_fast(g1.y))));
                            const Pair y0 = pair(2 * e <= far ? z0.x : 0.0f, 2 * e + 1 <= far ? z0.y : 0.0f), y1 = pair(2 * e + 2 <= far ? z1.x : 0.0f, 2 * e + 3 <= far ? z1.y : 0.0f);
                            p[e] = round_bf16(y0);
                            p[e + 1] = round_bf16(y1);
                            rest[e] = left_bf16(y0, p[e]);
                            rest[e + 1] = left_bf16(y1, p[e + 1]);
                        }
                        tc_st(tmem + kWeights + lanes + c0 / 2, p);
                        tc_st(tmem + kRest + lanes + c0 / 2, rest);
                    }
                } else {
#pragma unroll 1
                    for (int m = 0; m < w && m * 32 < frames; ++m) {             // (to its right are the zeros of the start)
                        const int c0 = m * 32 + half;
                        uint32_t s[16], p[8], rest[8];
                        tc_ld(tmem + kScores + lanes + c0, s);
                        const float r = exp2_fast((hi - D.hi[m * 32 + 31]) + (lo - D.lo[m * 32 + 31]));
                        const Pair row = pair(r, r);
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const ulonglong2 g = *reinterpret_cast<const ulonglong2*>(&D.col[c0 + 2 * e]);
                            const Pair y0 = mul2(pair(s[2 * e], s[2 * e + 1]), mul2(row, g.x)), y1 = mul2(pair(s[2 * e + 2], s[2 * e + 3]), mul2(row, g.y));
                            p[e] = round_bf16(y0);
                            p[e + 1] = round_bf16(y1);
                            rest[e] = left_bf16(y0, p[e]);
                            rest[e + 1] = left_bf16(y1, p[e + 1]);
                        }
                        tc_st(tmem + kWeights + lanes + c0 / 2, p);
                        tc_st(tmem + kRest + lanes + c0 / 2, rest);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(weighed);
                if (n > 0) {
                    store(h > 0 ? c : c - 1, h > 0 ? h - 1 : share - 1);
                    if (h == 0) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(d_empty + 8 * ((c - 1) % kDecays));
                    }
                }
            }
            if (!ok) break;
        }
        ok = ok && mbar_wait_warp(summed(chunks - 1), turn(chunks - 1), gave_up);
        if (ok) {
            tc_fence_after();
            if (holds) {
                float* to = i >= A.dk ? nullptr : MODE == 1 ? C.S.sums + (slot_at + i) * A.dv : it.last && A.state_out ? A.state_out + (state_at + i) * A.dv : nullptr;
                store_state<OUT ? 2 : 3>(to, j0, A.dv, state);
                __syncwarp();
            }
            if (OUT && mbar_wait_warp(answered, 0, gave_up)) {
                tc_fence_after();
                take(chunks - 1);
                store(chunks - 1, share - 1);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && *gave_up) atomicExch(C.error, 1);
    if (warp == 3) tmem_free(tmem, 512);
}

// The states that enter the segments of a sequence, from their sums: one after the other, element by element.
__global__ void __launch_bounds__(256) sr_segments_kernel(const __grid_constant__ SegmentArgs C)
{
    __shared__ int64_t first_slot;
    const AttentionArgs& A = C.A;
    let_successor_start();
    wait_for_predecessor();
    const int b = blockIdx.y / A.groups, g = blockIdx.y % A.groups;
    const AttentionSpan sp = attention_span(A, b);
    const int64_t count = segments_of(sp.n, C.segment);
    if (!A.offsets) {
        if (threadIdx.x == 0) first_slot = (int64_t)b * count;
    } else if (threadIdx.x < 32) {
        int64_t before = 0;
        for (int x = threadIdx.x; x < b; x += 32) before += segments_of(attention_span(A, x).n, C.segment);
#pragma unroll
        for (int m = 16; m; m /= 2) before += __shfl_xor_sync(0xFFFFFFFFu, before, m);
        if (threadIdx.x == 0) first_slot = before;
    }
    __syncthreads();
    const int64_t size = (int64_t)A.dk * A.dv, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= size) return;
    float S = A.state_in ? A.state_in[((int64_t)b * A.groups + g) * size + i] : 0.0f;
    // (offsets that overlap may ask for more slots than there are)
    const int64_t n = min(count, (int64_t)C.slots - first_slot);
    constexpr int kAhead = 8;                          // segments whose sums are read at once: one after the other each would wait for memory
    for (int64_t s0 = 0; s0 < n; s0 += kAhead) {
        float sum[kAhead], decay[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int64_t slot = (first_slot + s0 + e) * A.groups + g;
            const bool wanted = s0 + e < n && s0 + e + 1 < count;        // (the last segment's sums are not made)
            sum[e] = wanted ? C.sums[slot * size + i] : 0.0f;
            decay[e] = wanted ? C.decays[slot] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (s0 + e < n) {
                C.sums[((first_slot + s0 + e) * A.groups + g) * size + i] = S;
                S = fmaf(decay[e], S, sum[e]);
            }
    }
}

// [frames][sequences][heads][size] in boxes of 128 frames x 64 elements.
bool encode(CUtensorMap* map, const void* data, const sr_attention_strides& st, int64_t size, int64_t heads, int64_t sequences, int64_t frames)
{
    const SrEncodeTiled fn = sr_encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)size, (cuuint64_t)heads, (cuuint64_t)sequences, (cuuint64_t)frames};
    auto stride = [](int64_t s, int64_t n) { return (cuuint64_t)(n > 1 ? 2 * s : 16); };
    const cuuint64_t strides[3] = {stride(st.head, heads), stride(st.sequence, sequences), stride(st.frame, frames)};
    const cuuint32_t box[4] = {64u, 1, 1, (cuuint32_t)kChunk}, steps[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(data), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Whether everything starts on `bytes` and TMA could copy it.
bool copies_fit(const void* p, const sr_attention_strides& st, int64_t heads, int64_t sequences, int64_t frames, int bytes = 16)
{
    auto fits = [bytes](int64_t s, int64_t n) { return n <= 1 || (s > 0 && s % (bytes / 2) == 0 && s < ((int64_t)1 << 38)); };
    return (uintptr_t)p % bytes == 0 && fits(st.head, heads) && fits(st.sequence, sequences) && fits(st.frame, frames);
}

template <int DK, int MODE>
cudaError_t launch(const ChunkArgs& C, int64_t blocks, cudaStream_t s)
{
    constexpr int tiles = kKeySlots<DK, MODE> * DK * 256 + 2 * kCols * 256;
    constexpr int smem = 1024 + tiles + (MODE == 1 ? 2 * 3 * kCols * 256 : 2 * DK * 256 + 3 * kCols * 256 + 2 * DK * 128);
    static SrSharedLimit limit;
    const cudaError_t e = limit.raise(sr_chunks_kernel<DK, MODE>, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sr_chunks_kernel<DK, MODE>, C);
}
template <int DK>
cudaError_t launch_all(ChunkArgs& C, cudaStream_t s)
{
    const AttentionArgs& A = C.S.A;
    const int64_t per_slot = (int64_t)A.groups * C.S.v_tiles;
    if (!C.S.segment) return launch<DK, 0>(C, A.batch * per_slot, s);
    cudaError_t e = launch<DK, 1>(C, C.S.slots * per_slot, s);
    if (e != cudaSuccess) return e;
    e = sr_segments_launch(C.S, s);
    return e != cudaSuccess ? e : launch<DK, 2>(C, C.S.slots * per_slot, s);
}

// Frames of a segment, 0: whole sequences.  Segments are read twice (k and v for their sums, then everything for the outputs) and cost two launches and the
// way of their states out and back, about as much as five chunks; they are for launches that would leave SMs without work, or wait for
// one long sequence.  A step (a chunk for one head) is the unit; a chunk's sums alone are 0.6 of one.  Of packed sequences only the mean is known: the longest
// is taken for three times that.  Us whole / cut, calls back to back on three sets of inputs: one sequence, 8 heads of 128, 32768 frames 760 / 157, 4096 frames 104 / 42; 4 of 8192, 4 heads of 128 200 / 99; 8 of 1024,
// 4 heads of 64 28 / 33; packed, 16 of 3000 on average, 16 heads on 4 of 128 538 / 317; 32 of 1000, 8 heads of 64 87 / 118.  More than one wave of segments lost:
// 32768 frames 210, 263 with two, three waves instead of 166, packed 355, 364, 396 instead of 353 (measured alike, on an earlier form of the kernel).
AttentionCut cut_of(const sr_attention_desc* d, bool packed, int64_t sms)
{
    AttentionCut cut{0, 0};
    const int64_t per_slot = (int64_t)d->groups * ((d->dv + kCols - 1) / kCols);
    if (d->batch < 1 || d->frames < 1 || (int64_t)d->batch * d->groups > 65535) return cut;
    const double share = (double)(d->heads / d->groups);
    const double total = packed ? (double)d->frames : (double)d->frames * d->batch, mean = total / d->batch;
    const double longest = packed ? std::min(total, 3.0 * mean) : mean;
    const double waves = (double)(((int64_t)d->batch * per_slot + sms - 1) / sms);
    const double whole = std::max(longest, waves * mean) / kChunk * share;
    const int64_t want = std::max<int64_t>(1, sms / per_slot);
    // whole segments of every sequence, no more than there are SMs for
    const int64_t each = packed ? (int64_t)(total / (double)want) : (d->frames + std::max<int64_t>(1, want / d->batch) - 1) / std::max<int64_t>(1, want / d->batch);
    const int64_t length = std::max<int64_t>(512, (each + kChunk - 1) / kChunk * kChunk);
    if (length >= d->frames) return cut;
    const int64_t slots = packed ? d->batch + d->frames / length : d->batch * ((d->frames + length - 1) / length);
    const double pieces = packed ? total / (double)length + 0.5 * d->batch : (double)slots;
    if (std::ceil(pieces * (double)per_slot / (double)sms) * (double)(length / kChunk) * (share + 0.6) + 5.0 > 0.9 * whole) return cut;
    cut.segment = length;
    cut.slots = slots;
    return cut;
}

}  // namespace

// Rows of q, k and v that TMA can copy, and sizes that the tiles hold.
bool sr_chunks_fit(const sr_attention_desc* d, bool packed, const void* q, const void* k, const void* v)
{
    const int64_t sequences = packed ? 1 : d->batch;
    return d->frames < 0x7FFFFF00 && copies_fit(q, d->q, d->heads, sequences, d->frames) && copies_fit(k, d->k, d->groups, sequences, d->frames) &&
           copies_fit(v, d->v, d->groups, sequences, d->frames);
}
bool sr_chunks_wanted(const sr_attention_desc* d)
{
    return d->dtype == SR_DTYPE_BF16 && d->dk <= 128 && d->frames >= 16 &&
           (int64_t)(d->batch + d->frames) * d->groups * ((d->dv + kCols - 1) / kCols) <= 0x7FFFFFFF;
}
AttentionCut sr_chunks_cut(const sr_attention_desc* d, bool packed, int sms) { return cut_of(d, packed, std::max(1, sms)); }

SegmentArgs sr_segment_args(const AttentionArgs& A, AttentionCut cut, int cols, void* workspace)
{
    SegmentArgs C{};
    C.A = A;
    C.segment = cut.segment;
    C.slots = (int32_t)cut.slots;
    C.v_tiles = (A.dv + cols - 1) / cols;
    C.sums = static_cast<float*>(workspace);
    C.decays = C.sums ? C.sums + (size_t)cut.slots * A.groups * A.dk * A.dv : nullptr;
    return C;
}

cudaError_t sr_segments_launch(const SegmentArgs& C, cudaStream_t s)
{
    const AttentionArgs& A = C.A;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(((int64_t)A.dk * A.dv + 255) / 256), (unsigned)(A.batch * A.groups));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sr_segments_kernel, C);
}

cudaError_t sr_chunks_launch(const AttentionArgs& A, const sr_attention_desc* d, AttentionCut cut, void* workspace, cudaStream_t s)
{
    ChunkArgs C{};
    C.S = sr_segment_args(A, cut, kCols, workspace);
    C.error = sr_operator_error_word();
    if (!C.error) return cudaErrorUnknown;
    const int64_t sequences = A.offsets ? 1 : d->batch;
    if (!encode(&C.q_map, A.q, A.sq, d->dk, d->heads, sequences, d->frames) || !encode(&C.k_map, A.k, A.sk, d->dk, d->groups, sequences, d->frames) ||
        !encode(&C.v_map, A.v, A.sv, d->dv, d->groups, sequences, d->frames))
        return cudaErrorInvalidValue;
    C.out_align = 0;
    for (const int bytes : {16, 32})
        if (copies_fit(A.out, A.so, d->heads, sequences, d->frames, bytes)) C.out_align = bytes;
    return d->dk <= 64 ? launch_all<64>(C, s) : launch_all<128>(C, s);
}
