// Sequences of frames, side by side or packed one behind the other, and their segments: what kernels over the frames share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

// First frame and number of frames of a sequence; b: what its strides `sequence` are multiplied with.
struct FrameSpan {
    int64_t first, n, b;
};
// Searches and rounds over the sequences count up to 65535 places further in 32 bits.
constexpr int32_t kMostSequences = 0x7FFF0000;

// Whether neighbouring frames or sequences of `channels` elements would be written on top of each other.
inline bool frames_overlap(int64_t frame, int64_t sequence, int64_t frames, int64_t batch, int64_t channels)
{
    return (frames > 1 && frame < channels) || (batch > 1 && sequence < channels);
}

#ifdef __CUDACC__
// offsets NULL: sequences of `frames` frames side by side.  Offsets outside 0 .. frames are taken as the nearest of the two, a decreasing one as an empty sequence.
__device__ __forceinline__ FrameSpan frame_span(const int64_t* offsets, int64_t frames, int64_t b)
{
    FrameSpan s{0, frames, b};
    if (offsets) {
        const int64_t lo = min(max(offsets[b], (int64_t)0), frames), hi = min(max(offsets[b + 1], (int64_t)0), frames);
        s.first = lo;
        s.n = max(hi - lo, (int64_t)0);
        s.b = 0;
    }
    return s;
}
__host__ __device__ __forceinline__ int64_t segments_of(int64_t n, int64_t length) { return n > length ? (n + length - 1) / length : 1; }

// The sequence (-1: none) and segment of a slot; slots count the segments of all sequences one after the other.  (All lanes of a warp.)
__device__ __forceinline__ void find_slot(const int64_t* offsets, int64_t frames, int batch, int64_t segment, int64_t slot, int& b, int64_t& seg)
{
    if (!offsets) {
        const int64_t per = segments_of(frames, segment);
        const int64_t at = slot / per;
        b = at < batch ? (int)at : -1;
        seg = slot - at * per;
        return;
    }
    const int lane = threadIdx.x & 31;
    int64_t before = 0;
    b = -1;
    seg = 0;
    for (int b0 = 0; b0 < batch; b0 += 32) {
        const int64_t mine = b0 + lane < batch ? segments_of(frame_span(offsets, frames, b0 + lane).n, segment) : 0;
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
// The largest of a warp's values.
__device__ __forceinline__ int64_t most_of_warp(int64_t most)
{
#pragma unroll
    for (int d = 16; d; d /= 2) most = max(most, (int64_t)__shfl_xor_sync(0xFFFFFFFFu, most, d));
    return most;
}
// The frames of the longest of the packed sequences first, first + step and so on of a warp's lanes together.  (All of them.)
__device__ __forceinline__ int64_t longest_span(const int64_t* offsets, int64_t frames, int batch, int first, int step)
{
    int64_t most = 0;
#pragma unroll 8
    for (int i = first; i < batch; i += step) most = max(most, frame_span(offsets, frames, i).n);
    return most_of_warp(most);
}
// Packed sequences, slots that need no sum over the sequences before: sequence b has those from offsets[b] / segment + b on, as many as its segments at least, and all of them are
// frames / segment + batch.
__device__ __forceinline__ int64_t packed_first(const int64_t* offsets, int64_t frames, int64_t segment, int b)
{
    const int64_t o = min(max(offsets[b], (int64_t)0), frames);
    return (((uint64_t)o | (uint64_t)segment) >> 32 ? o / segment : (int64_t)((uint32_t)o / (uint32_t)segment)) + b;
}
// The sequence (-1: none) and segment of such a slot: a search in which every lane looks at one place.  (All lanes of a warp.)
__device__ __forceinline__ void packed_slot(const int64_t* offsets, int64_t frames, int batch, int64_t segment, int64_t slot, int& b, int64_t& seg)
{
    int lo = 0, n = batch;
    seg = 0;
    for (;;) {
        const int step = (n + 31) / 32, at = (threadIdx.x & 31) * step;
        const bool here = at < n;
        const int64_t first = here ? packed_first(offsets, frames, segment, lo + at) : 0;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, here && first <= slot);
        if (!who) {
            b = -1;
            return;
        }
        const int last = 31 - __clz(who);
        if (step == 1) {
            b = lo + last;
            seg = slot - __shfl_sync(0xFFFFFFFFu, first, last);
            if (seg && seg * segment >= frame_span(offsets, frames, b).n) b = -1;       // (the sequence has no more segments)
            return;
        }
        lo += last * step;
        n = min(step, n - last * step);
    }
}
#endif
