// Linear attention: what its two kernels for whole clips share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/sr_rollout.h"
#include "sr_spans.cuh"

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

typedef FrameSpan AttentionSpan;

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
__device__ __forceinline__ AttentionSpan attention_span(const AttentionArgs& A, int b) { return frame_span(A.offsets, A.frames, b); }
__device__ __forceinline__ void find_slot(const SegmentArgs& C, int slot, int& b, int64_t& seg) { find_slot(C.A.offsets, C.A.frames, C.A.batch, C.segment, slot, b, seg); }
// A CTA's work: frames t0 .. t0 + n - 1 of sequence b, group g, columns of v from c0 on.
struct AttentionItem {
    int b, g, c0, slot;
    int64_t t0, n;
    AttentionSpan span;
    bool there, last;                                  // last: the sequence ends with it
};
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
