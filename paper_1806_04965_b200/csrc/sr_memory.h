// Linear attention: what its two kernels for whole clips share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/sr_rollout.h"

struct AttentionArgs {
    const void *q, *k, *v;
    const float* decay;
    const int64_t* offsets;
    const float* state_in;
    float* state_out;
    void* out;
    int64_t frames;
    int32_t batch, groups, share, dk, dv;              // share: heads per group
    float scale;
    sr_attention_strides sq, sk, sv, so, sd;
};

// First frame and number of frames of a sequence; b: what its strides `sequence` are multiplied with.
struct AttentionSpan {
    int64_t first, n, b;
};

// Long sequences are cut into segments: their sums first (with no state entering), then the states that enter them, then their outputs.  Slots count the
// segments of all sequences one after the other.
struct SegmentArgs {
    AttentionArgs A;
    float* sums;                                       // [slot][group][dk][dv]: sums of a segment, then the states that enter it
    float* decays;                                     // [slot][group]: decay over a segment
    int64_t segment;                                   // frames of a segment (0: whole sequences)
    int32_t slots, v_tiles;                            // v_tiles: CTAs side by side over the columns of v
};
struct AttentionCut {
    int64_t segment, slots;                            // 0: whole sequences
};

#ifdef __CUDACC__
__device__ __forceinline__ AttentionSpan attention_span(const AttentionArgs& A, int b)
{
    AttentionSpan s{0, A.frames, b};
    if (A.offsets) {
        const int64_t lo = min(max(A.offsets[b], (int64_t)0), A.frames), hi = min(max(A.offsets[b + 1], (int64_t)0), A.frames);
        s.first = lo;
        s.n = max(hi - lo, (int64_t)0);
        s.b = 0;
    }
    return s;
}
__device__ __forceinline__ int64_t segments_of(int64_t n, int64_t length) { return n > length ? (n + length - 1) / length : 1; }

// A CTA's work: frames t0 .. t0 + n - 1 of sequence b, group g, columns of v from c0 on.
struct AttentionItem {
    int b, g, c0, slot;
    int64_t t0, n;
    AttentionSpan span;
    bool there, last;                                  // last: the sequence ends with it
};
// The sequence and segment of a slot.  (All lanes of a warp.)
__device__ __forceinline__ void find_slot(const SegmentArgs& C, int slot, int& b, int64_t& seg)
{
    const AttentionArgs& A = C.A;
    if (!A.offsets) {
        const int64_t per = segments_of(A.frames, C.segment);
        b = (int)(slot / per);
        seg = slot - b * per;
        if (b >= A.batch) b = -1;
        return;
    }
    const int lane = threadIdx.x & 31;
    int64_t before = 0;
    b = -1;
    seg = 0;
    for (int b0 = 0; b0 < A.batch; b0 += 32) {
        const int64_t mine = b0 + lane < A.batch ? segments_of(attention_span(A, b0 + lane).n, C.segment) : 0;
        int64_t sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
            if (lane >= d) sum += up;
        }
        const bool here = mine > 0 && before + sum - mine <= slot && slot < before + sum;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, here);
        if (who) {
            const int w = __ffs(who) - 1;
            b = b0 + w;
            seg = slot - (before + __shfl_sync(0xFFFFFFFFu, sum - mine, w));
            return;
        }
        before += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
}
// cut: the launch is one of segments.
__device__ __forceinline__ AttentionItem attention_item(const SegmentArgs& C, bool cut, int cols)
{
    const AttentionArgs& A = C.A;
    AttentionItem it;
    int x = blockIdx.x;
    it.c0 = (x % C.v_tiles) * cols;
    x /= C.v_tiles;
    it.g = x % A.groups;
    x /= A.groups;
    it.slot = x;
    it.b = x;
    int64_t seg = 0;
    if (cut) find_slot(C, x, it.b, seg);
    it.there = it.b >= 0;
    if (!it.there) return it;
    it.span = attention_span(A, it.b);
    it.t0 = cut ? seg * C.segment : 0;
    it.n = cut ? min(C.segment, it.span.n - it.t0) : it.span.n;
    it.last = it.t0 + it.n >= it.span.n;
    return it;
}
#endif

// sr_chunks.cu: bf16 on the tensor cores, chunks of 128 frames.
bool sr_chunks_fit(const sr_attention_desc* d, bool packed, const void* q, const void* k, const void* v);
bool sr_chunks_wanted(const sr_attention_desc* d);
AttentionCut sr_chunks_cut(const sr_attention_desc* d, bool packed, int sms);
cudaError_t sr_chunks_launch(const AttentionArgs& A, const sr_attention_desc* d, AttentionCut cut, void* workspace, cudaStream_t s);
cudaError_t sr_segments_launch(const SegmentArgs& C, cudaStream_t s);       // the states that enter the segments, from their sums
SegmentArgs sr_segment_args(const AttentionArgs& A, AttentionCut cut, int cols, void* workspace);
inline size_t sr_cut_bytes(const sr_attention_desc* d, AttentionCut cut)
{
    return cut.segment ? (size_t)cut.slots * d->groups * ((size_t)d->dk * d->dv * 4 + 4) + 256 : 0;
}
