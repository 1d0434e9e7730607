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
#endif

// sr_chunks.cu: bf16 on the tensor cores, chunks of 128 frames.
bool sr_chunks_fit(const sr_attention_desc* d, bool packed, const void* q, const void* k, const void* v);
bool sr_chunks_wanted(const sr_attention_desc* d);
size_t sr_chunks_workspace(const sr_attention_desc* d, bool packed);
cudaError_t sr_chunks_launch(const AttentionArgs& A, const sr_attention_desc* d, void* workspace, cudaStream_t s);
