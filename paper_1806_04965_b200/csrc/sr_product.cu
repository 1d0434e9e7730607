// Product of microscaled matrices: out[r][o] = act(bias[o] + sum_c a[r][c] * w[o][c]), on the tensor cores' block-scaled MMAs (tcgen05.mma
// kind::mxf8f6f4 and kind::mxf4: products of the elements times the two scales of their groups of 32, summed in 32 bits).
//
// Roles.  The weights are the M operand (128 outputs per tile: TMEM lane = output), the rows of a the N operand (NT of them: TMEM column = row), as in
// the frame update's kernel: few rows then cost few columns, and a warp's stores are 32 neighbouring outputs of one row.
// Stages.  One ring slot holds 128 bytes of every row of both operands (128 elements of 8 bits, 256 of 4), K-major with the 128-byte swizzle, by two
// TMA copies (zero fill behind the last column and row), and their scales: the formats' scale tiles of 128 rows x 4 groups are what tcgen05.cp takes,
// 512 bytes onto four TMEM columns (byte g of lane r % 32, column r / 32), so a stage's scales are one or two bulk copies per operand and one or two
// tcgen05.cp.  An MMA takes 32 bytes of a row: one group of 8-bit elements, two of 4-bit ones.
// Warps: 0 copies, 1 MMAs, 2 TMEM, 4..11 epilogue (bias, ReLU, rounding), which works on one accumulator while the MMAs fill the other.
// Many tiles: two CTAs as a pair (cta_group::2) share a tile of 256 outputs.  Each brings its 128 outputs' weights and half of the rows and has its outputs' sums; the first
// one issues the MMAs, which read both CTAs' memory.  8192 x 4096 x 8192 in 4 bits 117 -> 106 us (5.2 PFLOP/s), in 8 bits 229 -> 205 (2.7).  MMAs want to follow
// one another: with the next stage's scales or only the wait for it between them 117 and 223, with two stages at a time 112 and 217.
// Few tiles: the CTAs of a cluster share a tile's reduction; their sums meet in distributed shared memory, each CTA finishing its share of the
// columns in a fixed order.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "sr_microscale.cuh"
#include "sr_operators.h"
#include "sr_ptx.cuh"

static __device__ int sr_operator_error;              // 1: a bounded wait expired since the last sr_operator_reset

namespace {
using namespace srx;

constexpr int kThreads = 384, kEpilogueWarps = 8, kOuts = 128, kMaxStages = 8;
constexpr int kSmem = 200 * 1024;
constexpr int64_t kMost = 0x7FFFFFFF - 256;           // rows, outputs, columns

struct ProductArgs {
    CUtensorMap w_map, a_map;
    CUtensorMap ws_map, as_map;                        // (pairs) scale tiles
    const uint8_t *w_scales, *a_scales;
    const float* bias;
    void* out;
    int64_t out_stride;
    int32_t rows, outs, row_bytes, tiles_g, tiles_r;
    int32_t out_tiles, row_tiles, stages, ring;       // stages of the whole reduction; ring slots
    int32_t act, out_bf16, split;
    int* error;
};

// PAIR: two CTAs share a tile of twice the outputs, each with half of them and half of the rows of a.
template <int FMT, int NT, bool PAIR>
struct Shape {
    static constexpr int TG = FMT == SR_FORMAT_MX4 ? 2 : 1;          // scale tiles of a stage along the groups
    static constexpr int RT = NT > 128 ? 2 : 1;                      // ... along the rows of a
    static constexpr int W = kOuts * 128, A = (PAIR ? NT / 2 : NT) * 128, SW = TG * 512, SA = RT * TG * 512;
    static constexpr int kStage = (W + A + SW + SA + 1023) / 1024 * 1024;
    static constexpr int kAccs = 2;
    static constexpr int kScaleCols = TG * 4 + TG * RT * 4;          // TMEM columns of a stage's scales
    static constexpr int kScaleBase = kAccs * NT;
    static constexpr int kCols = kScaleBase + 2 * kScaleCols;
    static constexpr int kAlloc = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static_assert(kCols <= 512, "TMEM has 512 columns");
};

#define SR_MMA_SCALED(group, kind)                                                                                             \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                                            \
                 "tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"                        \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
template <int FMT, bool PAIR>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate)
{
    if constexpr (FMT == SR_FORMAT_MX4) {
        if constexpr (PAIR) SR_MMA_SCALED("2", "mxf4.block_scale.scale_vec::2X");
        else SR_MMA_SCALED("1", "mxf4.block_scale.scale_vec::2X");
    } else {
        if constexpr (PAIR) SR_MMA_SCALED("2", "mxf8f6f4.block_scale.scale_vec::1X");
        else SR_MMA_SCALED("1", "mxf8f6f4.block_scale.scale_vec::1X");
    }
}
#undef SR_MMA_SCALED
// 512 bytes (32 lanes x 16 bytes, lane after lane) onto four TMEM columns, the same in all four quarters of the lanes; in a pair, from each CTA's own memory
// onto its own columns.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t smem)
{
    const uint64_t desc = (uint64_t)((smem & 0x3FFFFu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }
// max that hands a NaN on
__device__ __forceinline__ float at_least(float v, float low)
{
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(v) : "f"(low));
    return v;
}

// Epilogue of a warp: outputs of its lanes, every second chunk of CW columns, tile after tile.  A store of the warp is 32 neighbouring outputs of a row.
template <int NT, int CW, bool PAIR, typename T>
__device__ __forceinline__ void drain(const ProductArgs& P, T* out, uint32_t taddr, int lane_out, int half, uint32_t tfull, uint32_t tempty, int first, int step,
                                      int tiles, volatile int* gave_up)
{
    const float low = P.act ? 0.0f : -__int_as_float(0x7F800000);
    uint32_t it = 0;
    for (int t = first; t < tiles; t += step, ++it) {
        const int o = t % P.out_tiles * (PAIR ? 2 * kOuts : kOuts) + lane_out, r0 = t / P.out_tiles * NT;
        const uint32_t acc = it & 1u;
        const float b = P.bias && o < P.outs ? P.bias[o] : 0.0f;
        if (!mbar_wait_warp(tfull + 8 * acc, (it >> 1) & 1u, gave_up)) break;
        tc_fence_after();
        const int n = min(NT, P.rows - r0);
        T* p = out + (int64_t)(r0 + half * CW) * P.out_stride + o;
        for (int c = half * CW; c < n; c += 2 * CW, p += 2 * CW * P.out_stride) {
            uint32_t v[CW];
            tc_ld(taddr + acc * NT + c, v);
            if (o < P.outs) {
                T* q = p;
                if (c + CW <= n) {
#pragma unroll
                    for (int i = 0; i < CW; ++i, q += P.out_stride) put(q, at_least(__uint_as_float(v[i]) + b, low));
                } else {
#pragma unroll
                    for (int i = 0; i < CW; ++i, q += P.out_stride)
                        if (c + i < n) put(q, at_least(__uint_as_float(v[i]) + b, low));
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            if constexpr (PAIR) mbar_arrive_at(tempty + 8 * acc, 0);
            else mbar_arrive(tempty + 8 * acc);
        }
    }
}

template <int FMT, int NT, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) sr_product_kernel(const __grid_constant__ ProductArgs P)
{
    using S = Shape<FMT, NT, PAIR>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 4];
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_flag;
    volatile int* gave_up = &gave_up_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t full = smem_u32(&bars[0]), empty = smem_u32(&bars[kMaxStages]), tfull = smem_u32(&bars[2 * kMaxStages]), tempty = tfull + 16;
    if (threadIdx.x == 0) {
        gave_up_flag = 0;
        for (int s = 0; s < P.ring; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull + 8 * a, 1);
            mbar_init(tempty + 8 * a, PAIR ? 2 * kEpilogueWarps : kEpilogueWarps);
        }
        mbar_init_done();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&P.w_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&P.a_map) : "memory");
    }
    wait_for_predecessor();
    if (warp == 2) {
        if constexpr (PAIR) tmem_alloc_pair(smem_u32(&tmem_slot), S::kAlloc);
        else tmem_alloc(smem_u32(&tmem_slot), S::kAlloc);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();                // (barriers and tensor memory of both)
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    let_successor_start();

    constexpr int kTile = PAIR ? 2 * kOuts : kOuts;    // outputs of a tile
    const int half_of = PAIR ? (int)cluster_rank() : 0;
    const int rank = !PAIR && P.split > 1 ? (int)cluster_rank() : 0, together = PAIR ? 2 : P.split;
    const int first = (int)blockIdx.x / together, step = (int)gridDim.x / together;
    const int tiles = P.out_tiles * P.row_tiles;
    const int k0 = (int)((int64_t)P.stages * rank / P.split), k1 = (int)((int64_t)P.stages * (rank + 1) / P.split);

    if (warp == 0) {
        if (elect_one()) {
            uint32_t n = 0, s = 0, ph = 1;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                const int o0 = t % P.out_tiles * kTile + half_of * kOuts, r0 = t / P.out_tiles * NT;
                const int rt0 = r0 >> 7, rts = min(S::RT, min(P.tiles_r - rt0, ((r0 & 127) + NT + 127) >> 7));
                for (int k = k0; k < k1; ++k) {
                    ok = mbar_wait(empty + 8 * s, ph, gave_up);
                    if (!ok) break;
                    const uint32_t at = ring + s * S::kStage, bar = full + 8 * s, to = at + S::W + S::A;
                    if constexpr (PAIR) {
                        // both CTAs' copies count on the first one's barrier (boxes that reach over an end bring zeros, or scales that no MMA takes)
                        if (half_of == 0) mbar_expect_tx(bar, 2 * (S::W + S::A + S::SW + S::SA));
                        tma_load_2d_pair(at, &P.w_map, bar, k * 128, o0);
                        tma_load_2d_pair(at + S::W, &P.a_map, bar, k * 128, r0 + half_of * (NT / 2));
                        tma_load_2d_pair(to, &P.ws_map, bar, 0, (o0 >> 7) * P.tiles_g + k * S::TG);
#pragma unroll
                        for (int q = 0; q < S::RT; ++q) tma_load_2d_pair(to + S::SW + q * S::TG * 512, &P.as_map, bar, 0, (rt0 + q) * P.tiles_g + k * S::TG);
                    } else {
                        const uint32_t sb = (uint32_t)min(S::TG, P.tiles_g - k * S::TG) * 512u;
                        mbar_expect_tx(bar, S::W + S::A + sb * (1 + rts));
                        tma_load_2d(at, &P.w_map, bar, k * 128, o0);
                        tma_load_2d(at + S::W, &P.a_map, bar, k * 128, r0);
                        bulk_load(to, P.w_scales + ((int64_t)(o0 >> 7) * P.tiles_g + k * S::TG) * 512, sb, bar);
                        for (int q = 0; q < rts; ++q) bulk_load(to + S::SW + q * S::TG * 512, P.a_scales + ((int64_t)(rt0 + q) * P.tiles_g + k * S::TG) * 512, sb, bar);
                    }
                    ++n;
                    if (++s == (uint32_t)P.ring) { s = 0; ph ^= 1; }
                }
            }
            // (a pair's first CTA waits for both; the second one does not leave before it)
            for (uint32_t v = 0; v < (uint32_t)P.ring && v < n && half_of == 0; ++v) mbar_drain(full + 8 * v, ((n - 1 - v) / P.ring) & 1);
        }
    } else if (warp == 1) {
        if (half_of == 0 && elect_one()) {                                                   // (a pair's first CTA issues its MMAs)
            // D = f32; A, B = e4m3 (code 0) or e2m1 (1); scales ue8m0; both operands K-major
            const uint32_t type = FMT == SR_FORMAT_MX4 ? 1u : 0u;
            const uint32_t idesc = (type << 7) | (type << 10) | ((uint32_t)(NT >> 3) << 17) | (1u << 23) | ((uint32_t)(kTile >> 4) << 24);
            uint32_t s = 0, ph = 0, it = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, ++it) {
                const int r0 = t / P.out_tiles * NT;
                const uint32_t acc = it & 1u, d = tmem + acc * NT;
                ok = mbar_wait<PAIR>(tempty + 8 * acc, ((it >> 1) & 1u) ^ 1u, gave_up);
                if (!ok) break;
                tc_fence_after();
                for (int k = k0; k < k1; ++k) {
                    ok = mbar_wait<PAIR>(full + 8 * s, ph, gave_up);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t at = ring + s * S::kStage;
                    const uint32_t sw = tmem + S::kScaleBase + (uint32_t)(k & 1) * S::kScaleCols, sa = sw + S::TG * 4;
#pragma unroll
                    for (int g = 0; g < S::TG; ++g) {
                        copy_scales<PAIR>(sw + 4 * g, at + S::W + S::A + 512 * g);
#pragma unroll
                        for (int q = 0; q < S::RT; ++q) copy_scales<PAIR>(sa + (g * S::RT + q) * 4, at + S::W + S::A + S::SW + (q * S::TG + g) * 512);
                    }
                    const uint64_t da = desc_k_major(at), db = desc_k_major(at + S::W);
                    const int n = min(4, (P.row_bytes - k * 128 + 31) / 32);
                    const uint32_t shift = (uint32_t)(r0 & 127) >> 5;                        // columns of 32 rows that the tile starts into its first scale tile
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i >= n) break;
                        const int g = FMT == SR_FORMAT_MX4 ? i / 2 : 0;
                        const uint32_t id = FMT == SR_FORMAT_MX4 ? (uint32_t)(i & 1) * 2 : (uint32_t)i;
                        mma_scaled<FMT, PAIR>(d, da + 2 * i, db + 2 * i, idesc | (id << 4) | (id << 29), sw + 4 * g, sa + g * S::RT * 4 + shift, (k > k0 || i > 0) ? 1u : 0u);
                    }
                    if constexpr (PAIR) tc_commit_pair(empty + 8 * s);
                    else tc_commit(empty + 8 * s);
                    if (++s == (uint32_t)P.ring) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                if constexpr (PAIR) tc_commit_pair(tfull + 8 * acc);
                else tc_commit(tfull + 8 * acc);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // two warps per quarter of the lanes, which take its chunks of columns in turn
        constexpr int CW = NT < 32 ? NT : 32;
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const int at = half_of * kOuts + quarter * 32 + lane;
        if (!PAIR && P.split > 1) {
            // (one tile per cluster) the partial sums lie in the ring, which is idle by now: [column][output]
            const bool ok = mbar_wait_warp(tfull, 0, gave_up);
            tc_fence_after();
            float* mine = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)));
            for (int c = half * CW; c < NT && ok; c += 2 * CW) {
                uint32_t v[CW];
                tc_ld(tmem + lanes + c, v);
#pragma unroll
                for (int i = 0; i < CW; ++i) mine[(c + i) * kOuts + quarter * 32 + lane] = __uint_as_float(v[i]);
            }
        } else if (P.out_bf16) {
            drain<NT, CW, PAIR>(P, static_cast<__nv_bfloat16*>(P.out), tmem + lanes, at, half, tfull, tempty, first, step, tiles, gave_up);
        } else {
            drain<NT, CW, PAIR>(P, static_cast<float*>(P.out), tmem + lanes, at, half, tfull, tempty, first, step, tiles, gave_up);
        }
    }
    if (!PAIR && P.split > 1) {
        __syncwarp();
        cluster_sync();
        const int o0 = first % P.out_tiles * kOuts, r0 = first / P.out_tiles * NT;
        const int share = NT / P.split;
        for (int i = threadIdx.x; i < share * (kOuts / 4); i += kThreads) {
            const int c = rank * share + i / (kOuts / 4), o = i % (kOuts / 4) * 4;
            const uint32_t at = ring + (uint32_t)(c * kOuts + o) * 4u;
            float4 v = ld_cluster(at, 0);
#pragma unroll
            for (int q = 1; q < 8; ++q) {
                if (q >= P.split) break;
                const float4 x = ld_cluster(at, (uint32_t)q);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            if (r0 + c >= P.rows) continue;
            const float y[4] = {v.x, v.y, v.z, v.w};
            const int64_t to = (int64_t)(r0 + c) * P.out_stride + o0 + o;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (o0 + o + e >= P.outs) break;
                const float z = at_least(y[e] + (P.bias ? P.bias[o0 + o + e] : 0.0f), P.act ? 0.0f : -__int_as_float(0x7F800000));
                if (P.out_bf16) put(static_cast<__nv_bfloat16*>(P.out) + to + e, z);
                else put(static_cast<float*>(P.out) + to + e, z);
            }
        }
        cluster_sync();                                // (nobody leaves while others read its memory)
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();                // (neither leaves while the other's MMAs read its memory or its warps arrive here)
    tc_fence_after();
    if (threadIdx.x == 0 && *gave_up) atomicExch(P.error, 1);
    if (warp == 2) {
        if constexpr (PAIR) tmem_free_pair(tmem, S::kAlloc);
        else tmem_free(tmem, S::kAlloc);
    }
}

// Rows of bytes, box_rows rows x 128 bytes at a time.
bool encode_rows(CUtensorMap* map, const void* data, int64_t row_bytes, int64_t rows, int box_rows)
{
    const SrEncodeTiled fn = sr_encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(data), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of scales, 512 bytes each, a stage's at a time.
bool encode_scales(CUtensorMap* map, const void* scales, int64_t tiles, int box_tiles)
{
    const SrEncodeTiled fn = sr_encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {128, (cuuint64_t)tiles}, strides[1] = {512};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_tiles}, steps[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(scales), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows of a tile, and CTAs that share a tile's reduction: the pair with the least estimated time in cycles.  A stage costs its four MMAs (NT / 2 cycles each,
// or (128 + NT) / 4 where the operands' way out of shared memory is longer) or its copies (60 bytes per cycle and SM).  Draining a tile costs 16 cycles per
// column, beside the next tile's MMAs, the exchange of a shared reduction 36.  Us, one CTA per tile / shared by four: 1 x 4096 x 4096 in 4 bits 6.8 / 5.9 (tiles of 16),
// 64 x 4096 x 4096 7.0 / 7.0 (64); shared by two with tiles of 128 200 x 4096 x 4096 7.9 / 9.4.  Tiles of 64 / 128 / 192 rows: 777 x 1000 x 1111 in 8 bits 5.5 / 5.9 / 6.7,
// 4096 x 1024 x 4608 40 / 24 / 22.
struct Plan {
    int nt, split;
    bool pair;
};
Plan plan_product(int64_t rows, int64_t outs, int stages, int sms)
{
    Plan best{16, 1, false};
    double least = 1e300;
    for (int nt : {16, 32, 64, 128, 192}) {
        if (nt == 16 && rows > 16) continue;
        if (nt == 32 && rows > 32) continue;          // (a tile starts at a multiple of 64 rows: two TMEM columns of scales)
        const int64_t tiles = ((outs + kOuts - 1) / kOuts) * ((rows + nt - 1) / nt);
        const double per_stage = std::max(4.0 * std::max(nt / 2.0, (128 + nt) / 4.0), (16384.0 + nt * 128.0) / 60.0);
        const double drain = 16.0 * nt;
        for (int split : {1, 2, 4, 8}) {
            if (split > stages || (split > 1 && tiles * split > sms)) continue;
            const double waves = (double)((tiles * split + sms - 1) / sms);
            const double work = ((stages + split - 1) / split) * per_stage;
            const double t = split > 1 ? work + drain / split + 36.0 * nt : waves * (std::max(work, drain) + 300.0) + std::min(work, drain);
            if (t < least) {
                least = t;
                best = {nt, split, false};
            }
        }
    }
    // Pairs of CTAs with tiles of 256 x 192.  A stage takes them 640 cycles, whatever its format, the ring's depth or the threads that ask for its copies: reads
    // and copies of shared memory, scales and outputs on their way each add to its 384 cycles of MMAs (8192 x 4096 x 8192 in 4 bits 106 us; without its copies 101, without its
    // outputs 92, without its scales 97, without all three 79).
    const int64_t tiles = ((outs + 2 * kOuts - 1) / (2 * kOuts)) * ((rows + 191) / 192), pairs = sms / 2;
    const double work = stages * 640.0, drain = 16.0 * 192;
    if (pairs > 0 && (double)((tiles + pairs - 1) / pairs) * (std::max(work, drain) + 600.0) + std::min(work, drain) < least) best = {192, 1, true};
    return best;
}

template <int FMT, int NT, bool PAIR>
cudaError_t launch(ProductArgs& P, int sms, cudaStream_t stream)
{
    using S = Shape<FMT, NT, PAIR>;
    P.ring = std::min(kMaxStages, (kSmem - 1024) / S::kStage);
    const size_t smem = 1024 + (size_t)P.ring * S::kStage;
    static SrSharedLimit limit;
    const cudaError_t e = limit.raise(sr_product_kernel<FMT, NT, PAIR>, (int)smem);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)P.out_tiles * P.row_tiles;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = PAIR ? 2u : (unsigned)P.split;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(PAIR ? 2 * std::min<int64_t>(tiles, sms / 2) : P.split > 1 ? tiles * P.split : std::min<int64_t>(tiles, sms)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = PAIR || P.split > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, sr_product_kernel<FMT, NT, PAIR>, P);
}
template <int FMT>
cudaError_t launch_any(ProductArgs& P, const Plan& plan, int sms, cudaStream_t s)
{
    if (plan.pair) return launch<FMT, 192, true>(P, sms, s);
    switch (plan.nt) {
        case 16: return launch<FMT, 16, false>(P, sms, s);
        case 32: return launch<FMT, 32, false>(P, sms, s);
        case 64: return launch<FMT, 64, false>(P, sms, s);
        case 128: return launch<FMT, 128, false>(P, sms, s);
        default: return launch<FMT, 192, false>(P, sms, s);
    }
}

}  // namespace

extern "C" {

sr_status sr_microscale_product_plan(int format, int64_t rows, int64_t cols, int64_t outs, int sms, sr_product_plan* plan)
{
    if (!plan || (format != SR_FORMAT_MX8 && format != SR_FORMAT_MX4) || rows < 1 || outs < 1 || cols < 1 || rows > kMost || outs > kMost || cols > kMost || sms < 0)
        return SR_ERR_INVALID_ARG;
    if (!sms) sms = sr_device_sms();
    if (sms < 1) return SR_ERR_CUDA;
    const Plan p = plan_product(rows, outs, (int)((sr_scaled(rows, cols, format).row_bytes + 127) / 128), sms);
    *plan = sr_product_plan{p.nt, p.pair ? 2 * kOuts : kOuts, p.split, p.pair ? 1 : 0};
    return SR_OK;
}

sr_status sr_microscale_product(const void* a_data, const void* a_scales, const void* w_data, const void* w_scales, int format, int64_t rows, int64_t cols,
                                int64_t outs, const float* bias, int act, void* out, int out_dtype, int64_t out_stride, void* stream)
{
    if ((format != SR_FORMAT_MX8 && format != SR_FORMAT_MX4) || rows < 0 || outs < 0 || cols < 1 || rows > kMost || outs > kMost || cols > kMost ||
        (act != 0 && act != 1) || (out_dtype != SR_DTYPE_F32 && out_dtype != SR_DTYPE_BF16) || out_stride < outs)
        return SR_ERR_INVALID_ARG;
    if (!rows || !outs) return SR_OK;
    const int el = out_dtype == SR_DTYPE_F32 ? 4 : 2;
    if (!a_data || !a_scales || !w_data || !w_scales || !out || (uintptr_t)out % el || ((uintptr_t)bias & 3) || ((uintptr_t)a_data & 15) ||
        ((uintptr_t)a_scales & 15) || ((uintptr_t)w_data & 15) || ((uintptr_t)w_scales & 15))
        return SR_ERR_INVALID_ARG;
    const int sms = sr_device_sms();
    if (sms < 1) return SR_ERR_CUDA;
    const SrScaled z = sr_scaled(rows, cols, format);
    ProductArgs P{};
    P.w_scales = static_cast<const uint8_t*>(w_scales);
    P.a_scales = static_cast<const uint8_t*>(a_scales);
    P.bias = bias;
    P.out = out;
    P.out_stride = out_stride;
    P.rows = (int32_t)rows;
    P.outs = (int32_t)outs;
    P.row_bytes = (int32_t)z.row_bytes;
    P.tiles_g = (int32_t)z.tiles_g;
    P.tiles_r = (int32_t)z.tiles_r;
    P.stages = (int32_t)((z.row_bytes + 127) / 128);
    const Plan plan = plan_product(rows, outs, P.stages, sms);
    P.out_tiles = (int32_t)(plan.pair ? (outs + 2 * kOuts - 1) / (2 * kOuts) : (outs + kOuts - 1) / kOuts);
    P.row_tiles = (int32_t)((rows + plan.nt - 1) / plan.nt);
    if ((int64_t)P.out_tiles * P.row_tiles > kMost) return SR_ERR_INVALID_ARG;
    P.split = plan.split;
    P.act = act;
    P.out_bf16 = out_dtype == SR_DTYPE_BF16;
    P.error = sr_operator_error_word();
    if (!P.error) return SR_ERR_CUDA;
    if (!encode_rows(&P.w_map, w_data, z.row_bytes, outs, kOuts) || !encode_rows(&P.a_map, a_data, z.row_bytes, rows, plan.pair ? plan.nt / 2 : plan.nt)) return SR_ERR_CUDA;
    const int tg = format == SR_FORMAT_MX4 ? 2 : 1;
    if (plan.pair && (!encode_scales(&P.ws_map, w_scales, (outs + 127) / 128 * z.tiles_g, tg) || !encode_scales(&P.as_map, a_scales, z.tiles_r * z.tiles_g, tg)))
        return SR_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = format == SR_FORMAT_MX4 ? launch_any<SR_FORMAT_MX4>(P, plan, sms, s) : launch_any<SR_FORMAT_MX8>(P, plan, sms, s);
    return e == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

sr_status sr_operator_status(void* stream)
{
    // read in the stream's own order and left as it is: another stream's owner has to see it, too
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(s, &capturing) != cudaSuccess) return SR_ERR_CUDA;
    if (capturing != cudaStreamCaptureStatusNone) return SR_ERR_STATE;
    int expired = 0;
    const int* word = sr_operator_error_word();
    if (!word || cudaMemcpyAsync(&expired, word, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) return SR_ERR_CUDA;
    return expired ? SR_ERR_TIMEOUT : SR_OK;
}

sr_status sr_operator_reset(void* stream)
{
    int* word = sr_operator_error_word();
    return word && cudaMemsetAsync(word, 0, sizeof(int), static_cast<cudaStream_t>(stream)) == cudaSuccess ? SR_OK : SR_ERR_CUDA;
}

}  // extern "C"

int* sr_operator_error_word()
{
    static std::atomic<int*> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
    if (dev < 64)
        if (int* had = known[dev].load(std::memory_order_relaxed)) return had;
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, sr_operator_error) != cudaSuccess) return nullptr;
    if (dev < 64) known[dev].store(static_cast<int*>(p), std::memory_order_relaxed);
    return static_cast<int*>(p);
}

SrEncodeTiled sr_encode_tiled()
{
    static const SrEncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<SrEncodeTiled>(p);
    }();
    return fn;
}

int sr_device_sms()
{
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < 64)
        if (const int had = known[dev].load(std::memory_order_relaxed)) return had;
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    return n;
}
