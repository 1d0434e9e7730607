// Product of microscaled matrices: out[r][o] = act(bias[o] + sum_c a[r][c] * w[o][c]).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "sr_microscale.cuh"

namespace {

struct ProductArgs {
    const uint8_t *a, *a_scales, *w, *w_scales;
    const float* bias;
    void* out;
    int64_t rows, cols, outs, out_stride, groups, tiles_g;
    int act, out_bf16;
};

template <int FMT>
__device__ __forceinline__ float element(const uint8_t* data, const uint8_t* scales, int64_t row, int64_t c, const ProductArgs& P)
{
    const float s = sr_scale(scales[sr_scale_place(row, c >> 5, P.tiles_g)]);
    if (FMT == SR_FORMAT_MX4) return s * sr_e2m1_value((data[row * P.groups * 16 + c / 2] >> (4 * (c & 1))) & 15u);
    return s * sr_e4m3_value(data[row * P.groups * 32 + c]);
}

// 32 x 32 outputs per block, 32 columns of both matrices at a time.
template <int FMT>
__global__ void __launch_bounds__(256) sr_product_kernel(const __grid_constant__ ProductArgs P)
{
    __shared__ float a[32][33], w[32][33];
    const int64_t o0 = (int64_t)blockIdx.x * 32, r0 = (int64_t)blockIdx.y * 32;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    float sum[4] = {0, 0, 0, 0};
    for (int64_t c0 = 0; c0 < P.groups * 32; c0 += 32) {
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + ty + 8 * i, o = o0 + ty + 8 * i, c = c0 + tx;
            a[ty + 8 * i][tx] = r < P.rows ? element<FMT>(P.a, P.a_scales, r, c, P) : 0.0f;
            w[ty + 8 * i][tx] = o < P.outs ? element<FMT>(P.w, P.w_scales, o, c, P) : 0.0f;
        }
        __syncthreads();
        for (int c = 0; c < 32; ++c)
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(a[ty + 8 * i][c], w[tx][c], sum[i]);
        __syncthreads();
    }
    const int64_t o = o0 + tx;
    for (int i = 0; i < 4; ++i) {
        const int64_t r = r0 + ty + 8 * i;
        if (r >= P.rows || o >= P.outs) continue;
        float v = sum[i] + (P.bias ? P.bias[o] : 0.0f);
        if (P.act && v < 0.0f) v = 0.0f;
        if (P.out_bf16) static_cast<__nv_bfloat16*>(P.out)[r * P.out_stride + o] = __float2bfloat16(v);
        else static_cast<float*>(P.out)[r * P.out_stride + o] = v;
    }
}

}  // namespace

extern "C" {

sr_status sr_microscale_product(const void* a_data, const void* a_scales, const void* w_data, const void* w_scales, int format, int64_t rows, int64_t cols,
                                int64_t outs, const float* bias, int act, void* out, int out_dtype, int64_t out_stride, void* stream)
{
    const int64_t most = 0x7FFFFFFF;
    if ((format != SR_FORMAT_MX8 && format != SR_FORMAT_MX4) || rows < 0 || outs < 0 || cols < 1 || rows > most || outs > most || cols > most ||
        (act != 0 && act != 1) || (out_dtype != SR_DTYPE_F32 && out_dtype != SR_DTYPE_BF16) || out_stride < outs)
        return SR_ERR_INVALID_ARG;
    if (!rows || !outs) return SR_OK;
    const int el = out_dtype == SR_DTYPE_F32 ? 4 : 2;
    if (!a_data || !a_scales || !w_data || !w_scales || !out || (uintptr_t)out % el || ((uintptr_t)bias & 3) || ((uintptr_t)a_data & 15) ||
        ((uintptr_t)a_scales & 15) || ((uintptr_t)w_data & 15) || ((uintptr_t)w_scales & 15))
        return SR_ERR_INVALID_ARG;
    const SrScaled z = sr_scaled(rows, cols, format);
    ProductArgs P{};
    P.a = static_cast<const uint8_t*>(a_data);
    P.a_scales = static_cast<const uint8_t*>(a_scales);
    P.w = static_cast<const uint8_t*>(w_data);
    P.w_scales = static_cast<const uint8_t*>(w_scales);
    P.bias = bias;
    P.out = out;
    P.rows = rows;
    P.cols = cols;
    P.outs = outs;
    P.out_stride = out_stride;
    P.groups = z.groups;
    P.tiles_g = z.tiles_g;
    P.act = act;
    P.out_bf16 = out_dtype == SR_DTYPE_BF16;
    const dim3 grid((unsigned)((outs + 31) / 32), (unsigned)((rows + 31) / 32));
    if (grid.y > 65535) return SR_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (format == SR_FORMAT_MX4) sr_product_kernel<SR_FORMAT_MX4><<<grid, 256, 0, s>>>(P);
    else sr_product_kernel<SR_FORMAT_MX8><<<grid, 256, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_operator_status(void* stream)
{
    return cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"
