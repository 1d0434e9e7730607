// Linear attention with a decay for each head:  S_t = exp(g_t) S_{t-1} + k_t v_t^T,  out_t = scale * q_t S_t.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "sr_memory.h"

namespace {

// ------------------------------------------------------------------------------------------ frame by frame, any sizes
// A block holds 64 columns of a group's state: thread (column, rs) the rows of split rs, four neighbouring rows out of every 4 * RS.
// Frames come in through shared memory, kRunRows rows of queries at a time.
constexpr int kRunRows = 32, kRunCols = 64;

template <typename T, int RS>
__global__ void __launch_bounds__(kRunCols * RS) sr_attention_frames_kernel(const __grid_constant__ AttentionArgs A)
{
    constexpr int DK = RS * 32;
    extern __shared__ float smem[];
    const int ct = max(1, min(16, kRunRows / A.share));
    float* ks = smem;                                  // [ct][DK]
    float* vs = ks + ct * DK;                          // [ct][kRunCols]
    float* ds = vs + ct * kRunCols;                    // [16]
    float* qs = ds + 16;                               // [ct][share][DK]
    const int b = blockIdx.x / A.groups, g = blockIdx.x % A.groups, c0 = blockIdx.y * kRunCols;
    const int col = threadIdx.x / RS, rs = threadIdx.x % RS, j = c0 + col;
    const AttentionSpan sp = attention_span(A, b);
    const T* q = static_cast<const T*>(A.q) + sp.b * A.sq.sequence + (int64_t)g * A.share * A.sq.head;
    const T* k = static_cast<const T*>(A.k) + sp.b * A.sk.sequence + (int64_t)g * A.sk.head;
    const T* v = static_cast<const T*>(A.v) + sp.b * A.sv.sequence + (int64_t)g * A.sv.head;
    T* out = static_cast<T*>(A.out) + sp.b * A.so.sequence + (int64_t)g * A.share * A.so.head;
    const float* d = A.decay + sp.b * A.sd.sequence + (int64_t)g * A.sd.head;
    const int64_t at = ((int64_t)b * A.groups + g) * A.dk;
    auto row_of = [&](int r) { return (r >> 2) * (4 * RS) + rs * 4 + (r & 3); };
    float S[32];
#pragma unroll
    for (int r = 0; r < 32; ++r) S[r] = A.state_in && row_of(r) < A.dk && j < A.dv ? A.state_in[(at + row_of(r)) * A.dv + j] : 0.0f;
    for (int64_t t0 = 0; t0 < sp.n; t0 += ct) {
        const int n = (int)min((int64_t)ct, sp.n - t0);
        const int64_t f = sp.first + t0;
        for (int i = threadIdx.x; i < n * DK; i += blockDim.x) {
            const int t = i / DK, c = i % DK;
            ks[i] = c < A.dk ? (float)k[(f + t) * A.sk.frame + c] : 0.0f;
        }
        for (int i = threadIdx.x; i < n * A.share * DK; i += blockDim.x) {
            const int th = i / DK, c = i % DK, t = th / A.share, h = th % A.share;
            qs[i] = c < A.dk ? (float)q[(f + t) * A.sq.frame + h * A.sq.head + c] : 0.0f;
        }
        for (int i = threadIdx.x; i < n * kRunCols; i += blockDim.x) {
            const int t = i / kRunCols, c = i % kRunCols;
            vs[i] = c0 + c < A.dv ? (float)v[(f + t) * A.sv.frame + c0 + c] : 0.0f;
        }
        if (threadIdx.x < n) ds[threadIdx.x] = expf(d[(f + threadIdx.x) * A.sd.frame]);
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            const float decay = ds[t], x = vs[t * kRunCols + col];
#pragma unroll
            for (int r = 0; r < 32; r += 4) {
                const float4 y = *reinterpret_cast<const float4*>(&ks[t * DK + row_of(r)]);
                S[r] = fmaf(decay, S[r], y.x * x);
                S[r + 1] = fmaf(decay, S[r + 1], y.y * x);
                S[r + 2] = fmaf(decay, S[r + 2], y.z * x);
                S[r + 3] = fmaf(decay, S[r + 3], y.w * x);
            }
            for (int h = 0; h < A.share; ++h) {
                float o = 0.0f;
#pragma unroll
                for (int r = 0; r < 32; r += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(&qs[(t * A.share + h) * DK + row_of(r)]);
                    o = fmaf(y.x, S[r], o);
                    o = fmaf(y.y, S[r + 1], o);
                    o = fmaf(y.z, S[r + 2], o);
                    o = fmaf(y.w, S[r + 3], o);
                }
#pragma unroll
                for (int m = 1; m < RS; m *= 2) o += __shfl_xor_sync(0xFFFFFFFFu, o, m);
                if (rs == 0 && j < A.dv) out[(f + t) * A.so.frame + h * A.so.head + j] = (T)(A.scale * o);
            }
        }
        __syncthreads();
    }
    if (A.state_out)
#pragma unroll
        for (int r = 0; r < 32; ++r)
            if (row_of(r) < A.dk && j < A.dv) A.state_out[(at + row_of(r)) * A.dv + j] = S[r];
}

template <typename T, int RS>
cudaError_t launch_frames(const AttentionArgs& A, cudaStream_t s)
{
    const int ct = std::max(1, std::min(16, kRunRows / A.share));
    const size_t bytes = sizeof(float) * ((size_t)ct * RS * 32 * (1 + A.share) + (size_t)ct * kRunCols + 16);
    if (bytes > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(sr_attention_frames_kernel<T, RS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((unsigned)(A.batch * A.groups), (unsigned)((A.dv + kRunCols - 1) / kRunCols));
    sr_attention_frames_kernel<T, RS><<<grid, kRunCols * RS, bytes, s>>>(A);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch_frames_any(const AttentionArgs& A, cudaStream_t s)
{
    if (A.dk <= 32) return launch_frames<T, 1>(A, s);
    if (A.dk <= 64) return launch_frames<T, 2>(A, s);
    if (A.dk <= 128) return launch_frames<T, 4>(A, s);
    return launch_frames<T, 8>(A, s);
}

// ------------------------------------------------------------------------------------------ one frame
// Bound by the states: 8 bytes per element, read and written once.  A block of 256 threads has 32 columns of a group's state, so that a row of
// it is a whole line, and few sequences still make many blocks.  VEC columns per thread.
constexpr int kStepCols = 32, kStepHeads = 8;

template <typename T, int VEC, int ROWS>               // ROWS: rows of a thread
__global__ void __launch_bounds__(256) sr_attention_step_kernel(const __grid_constant__ AttentionArgs A)
{
    constexpr int CT = kStepCols / VEC, RL = 256 / CT; // threads per row; rows side by side
    __shared__ float part[kStepHeads][8][kStepCols];
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

template <typename T, int VEC>
cudaError_t launch_step(const AttentionArgs& A, cudaStream_t s)
{
    constexpr int RL = 256 / (kStepCols / VEC);
    const dim3 grid((unsigned)(A.batch * A.groups), (unsigned)((A.dv + kStepCols - 1) / kStepCols));
    const int rows = (A.dk + RL - 1) / RL;
    if (rows <= 2) sr_attention_step_kernel<T, VEC, 2><<<grid, 256, 0, s>>>(A);
    else if (rows <= 4) sr_attention_step_kernel<T, VEC, 4><<<grid, 256, 0, s>>>(A);
    else if (rows <= 8) sr_attention_step_kernel<T, VEC, 8><<<grid, 256, 0, s>>>(A);
    else sr_attention_step_kernel<T, VEC, 32><<<grid, 256, 0, s>>>(A);
    return cudaGetLastError();
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
    if ((int64_t)d->batch * d->groups > 0x7FFFFFFF || d->dv > 65535 * kStepCols) return SR_ERR_INVALID_ARG;
    if (d->dk > 256 || d->heads / d->groups > 128) return SR_ERR_UNSUPPORTED;
    return SR_OK;
}
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
    *bytes = sr_chunks_wanted(d) ? sr_chunks_workspace(d, packed != 0) : 0;
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
                      ((uintptr_t)decay & 3)))
        return SR_ERR_INVALID_ARG;
    const size_t needed = sr_chunks_wanted(d) ? sr_chunks_workspace(d, offsets != nullptr) : 0;
    if (needed && (!workspace || workspace_bytes < needed || ((uintptr_t)workspace & 255))) return SR_ERR_INVALID_ARG;
    AttentionArgs A = arguments(d, q, k, v, decay, out);
    A.offsets = offsets;
    A.state_in = state_in;
    A.state_out = state_out;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (sr_chunks_wanted(d) && sr_chunks_fit(d, offsets != nullptr, q, k, v)) e = sr_chunks_launch(A, d, workspace, s);
    else e = d->dtype == SR_DTYPE_F32 ? launch_frames_any<float>(A, s) : launch_frames_any<__nv_bfloat16>(A, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_linear_attention_step(const sr_attention_desc* d, const void* q, const void* k, const void* v, const float* decay, float* state, void* out,
                                   void* stream)
{
    const sr_status st = check(d);
    if (st != SR_OK) return st;
    if (!d->batch) return SR_OK;
    if (!q || !k || !v || !decay || !state || !out || !aligned(q, d->dtype) || !aligned(k, d->dtype) || !aligned(v, d->dtype) ||
        !aligned(out, d->dtype) || ((uintptr_t)decay & 3) || ((uintptr_t)state & 3))
        return SR_ERR_INVALID_ARG;
    AttentionArgs A = arguments(d, q, k, v, decay, out);
    A.state_out = state;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d->dtype == SR_DTYPE_F32 ? launch_step_any<float>(A, s) : launch_step_any<__nv_bfloat16>(A, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
