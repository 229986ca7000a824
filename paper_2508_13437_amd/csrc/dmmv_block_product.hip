// Product of two block matrices, y = x w^T + bias (include/dmmv_layer.h).
//
// The 8-bit matrix instructions of gfx950 line the products of a step up against the largest and drop what
// lies some 13 bits below it: against 64 bits their sums are off by 1e-5 to 5e-5 of the result's norm
// (random codes; up to 2^-11 of sum |x w| for single results).  That is far below the rounding of a bf16 result
// (2e-3), so bf16 results are summed by them; 32-bit results are summed by the 16-bit instructions, which keep the
// 32-bit sum (8e-8) at half the rate: a code is exact in f16.
#include "dmmv_layer_common.h"

namespace dmmv {

// 32 codes of a row from column `col` on, zero past `cols`
__device__ __forceinline__ void codes32(const uint8_t* __restrict__ row, int64_t col, int64_t cols, bool ok, piece16 (&v)[2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t c = col + 16 * h;
        piece16 a = {0u, 0u, 0u, 0u};
        if (ok && c + 16 <= cols) {
            a = *reinterpret_cast<const piece16_any*>(row + c);
        } else if (ok) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < cols) a[i >> 2] |= (uint32_t)row[c + i] << (8 * (i & 3));
        }
        v[h] = a;
    }
}

typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

// eight codes (two words) as f16
__device__ __forceinline__ halfx8 half8(int lo, int hi) {
    const halfx2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const halfx2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return halfx8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// sum over a block of 128 of a 16 x 16 tile, from 32 codes a lane (the order of k inside the block is free as
// long as both operands have the same)
template <bool WIDE>
__device__ __forceinline__ floatx4 block_sum(const intx8& a, const intx8& b) {
    floatx4 p = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (WIDE) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
            p = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(a[2 * s], a[2 * s + 1]), half8(b[2 * s], b[2 * s + 1]), p, 0, 0, 0);
    } else {
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, p, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
    }
    return p;
}

__device__ __forceinline__ void put_y(float* y, float v) { *y = v; }
__device__ __forceinline__ void put_y(bf16_t* y, float v) { y->u = (uint16_t)bf16_bits(v); }

// Any sizes, strides and scales.  64 x 64 tile, 4 wavefronts of 32 x 32; the codes of one block of 128
// go through the LDS, and the block's two scales are applied to its sum in 32 bits.
template <class T>
__global__ __launch_bounds__(256) void k_block_product(int64_t T_, int64_t O, int64_t K, BlockView x, BlockView w,
                                                       const float* __restrict__ bias, T* __restrict__ y, int64_t ldy, int64_t tiles_o) {
    constexpr int LS = 144;                                   // bytes of an LDS row: 128 and a skew of 16
    __shared__ __align__(16) uint8_t As[64 * LS], Bs[64 * LS];
    __shared__ float sa[64], sb[64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t t0 = (blockIdx.x / tiles_o) * 64, o0 = (blockIdx.x % tiles_o) * 64;
    const int m0 = (wv >> 1) * 32, n0 = (wv & 1) * 32;
    floatx4 acc[2][2] = {};
    const int r = tid >> 2, c = (tid & 3) * 32;
    for (int64_t k0 = 0, kb = 0; k0 < K; k0 += 128, ++kb) {
        piece16 a[2], b[2];
        codes32(x.codes + (t0 + r) * x.ld, k0 + c, K, t0 + r < T_, a);
        codes32(w.codes + (o0 + r) * w.ld, k0 + c, K, o0 + r < O, b);
        float s = 0.0f;
        if (tid < 64) s = t0 + tid < T_ ? scale_at(x, t0 + tid, kb) : 0.0f;
        else if (tid < 128) s = o0 + tid - 64 < O ? scale_at(w, o0 + tid - 64, kb) : 0.0f;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            *reinterpret_cast<piece16*>(As + r * LS + c + 16 * h) = a[h];
            *reinterpret_cast<piece16*>(Bs + r * LS + c + 16 * h) = b[h];
        }
        if (tid < 64) sa[tid] = s;
        else if (tid < 128) sb[tid - 64] = s;
        __syncthreads();
        intx8 fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* pa = As + (m0 + 16 * i + (lane & 15)) * LS + (lane >> 4) * 32;
            const uint8_t* pb = Bs + (n0 + 16 * i + (lane & 15)) * LS + (lane >> 4) * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const piece16 qa = *reinterpret_cast<const piece16*>(pa + 16 * h), qb = *reinterpret_cast<const piece16*>(pb + 16 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) { fa[i][4 * h + e] = (int)qa[e]; fb[i][4 * h + e] = (int)qb[e]; }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const floatx4 p = block_sum<sizeof(T) == 4>(fa[i], fb[j]);
                const float s_o = sb[n0 + 16 * j + (lane & 15)];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][j][e] = dmmv_fma(p[e], sa[m0 + 16 * i + (lane >> 4) * 4 + e] * s_o, acc[i][j][e]);
            }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t o = o0 + n0 + 16 * j + (lane & 15);
        if (o >= O) continue;
        const float bo = bias ? bias[o] : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t t = t0 + m0 + 16 * i + (lane >> 4) * 4 + e;
                if (t < T_) put_y(y + t * ldy + o, acc[i][j][e] + bo);
            }
    }
}

template <class T>
static dmmv_status product(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, T* y, int64_t ldy, hipStream_t s) {
    const int64_t tiles_t = ceil_div(x->rows, 64), tiles_o = ceil_div(w->rows, 64);
    if (tiles_t > INT32_MAX / tiles_o) return fail(DMMV_ERR_SHAPE, "y: more tiles than a launch takes");
    hipLaunchKernelGGL((k_block_product<T>), dim3((unsigned)(tiles_t * tiles_o)), dim3(256), 0, s, x->rows, w->rows, x->cols,
                       layer_view(x), layer_view(w), bias, y, ldy, tiles_o);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

static size_t product_workspace(int64_t, int64_t, int64_t) { return 0; }

}  // namespace dmmv

using namespace dmmv;

extern "C" size_t dmmv_block_product_workspace_bytes(int64_t T, int64_t O, int64_t K) {
    if (layer_check_sizes(T, K, "x") != DMMV_OK || layer_check_sizes(O, K, "w") != DMMV_OK) return 0;
    return product_workspace(T, O, K);
}

extern "C" dmmv_status dmmv_block_product(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, int32_t dtype,
                                          void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_block(x, false, "x"));
    DMMV_TRY(layer_check_block(w, false, "w"));
    if (x->cols != w->cols) return fail(DMMV_ERR_SHAPE, "x has %lld columns, w has %lld", (long long)x->cols, (long long)w->cols);
    DMMV_TRY(layer_check_array(y, x->rows, w->rows, ldy, layer_width(dtype), "y"));
    if ((uintptr_t)bias % 4) return fail(DMMV_ERR_SHAPE, "bias is not aligned to its elements");
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, product_workspace(x->rows, w->rows, x->cols)));
    if (x->rows == 0 || w->rows == 0) return DMMV_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return dtype == DMMV_F32 ? product(x, w, bias, static_cast<float*>(y), ldy, s) : product(x, w, bias, static_cast<bf16_t*>(y), ldy, s);
}
