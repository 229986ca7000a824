// Gradients of the product of block matrices (include/dmmv_layer.h).
//
// Both large products contract over the ROWS of a block matrix: dx = dy w over the outputs, dw = dy^T x
// over the tokens.  code * scale is exact in bf16 where scales are powers of two, so they run on
// the bf16 matrix cores without rounding the 8-bit operand; what needs 24 bits (32-bit gradients, other
// scales) is cut into three bf16 that sum to it, and the products of parts below the last bit are left out.
#include "dmmv_layer_common.h"

namespace dmmv {

__device__ __forceinline__ void put_c(float* y, float v) { *y = v; }
__device__ __forceinline__ void put_c(bf16_t* y, float v) { y->u = (uint16_t)bf16_bits(v); }

// C[m][n] = sum_k A(m, k) B(k, n), A(m, k) = a[m][k] or (TRANS) a[k][m], B a block matrix [k][n].
// PA, PB: parts that an operand is cut into.  64 x 64 tile, 4 wavefronts of 32 x 32, 32 of k a step.
template <class TA, bool TRANS, int PA, int PB, class TC>
__global__ __launch_bounds__(256) void k_block_grad(int64_t M, int64_t N, int64_t Kc, const TA* __restrict__ a, int64_t lda, BlockView b,
                                                    TC* __restrict__ c, int64_t ldc, int64_t tiles_n) {
    constexpr int LS = 40;                                    // 32 and a skew of 8
    __shared__ __align__(16) uint16_t As[PA][64 * LS], Bs[PB][64 * LS];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t m0 = (blockIdx.x / tiles_n) * 64, n0 = (blockIdx.x % tiles_n) * 64;
    const int wm = (wv >> 1) * 32, wn = (wv & 1) * 32;
    floatx4 acc[2][2] = {};
    for (int64_t k0 = 0; k0 < Kc; k0 += 32) {
        float va[8] = {}, vb[8] = {};
        const int am = TRANS ? (tid & 7) * 8 : tid >> 2, ak = TRANS ? tid >> 3 : (tid & 3) * 8;
        if (TRANS) {
            if (k0 + ak < Kc) load8(a + (k0 + ak) * lda, m0 + am, M, va);
        } else {
            if (m0 + am < M) load8(a + (m0 + am) * lda, k0 + ak, Kc, va);
        }
        const int bk = tid >> 3, bn = (tid & 7) * 8;
        if (k0 + bk < Kc && n0 + bn < N)
            decode8(load8_codes(b.codes + (k0 + bk) * b.ld, n0 + bn, N), scale_at(b, k0 + bk, (n0 + bn) >> 7), vb);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t p[3];
            if (PA == 3) split3(va[e], p);
            else p[0] = bf16_bits(va[e]);
            const int at = TRANS ? (am + e) * LS + ak : am * LS + ak + e;
#pragma unroll
            for (int i = 0; i < PA; ++i) As[i][at] = (uint16_t)p[i];
            if (PB == 3) split3(vb[e], p);
            else p[0] = bf16_bits(vb[e]);
#pragma unroll
            for (int i = 0; i < PB; ++i) Bs[i][(bn + e) * LS + bk] = (uint16_t)p[i];
        }
        __syncthreads();
        bf16x8_t fa[PA][2], fb[PB][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int p = 0; p < PA; ++p)
                fa[p][i] = *reinterpret_cast<const bf16x8_t*>(&As[p][(wm + 16 * i + (lane & 15)) * LS + (lane >> 4) * 8]);
#pragma unroll
            for (int p = 0; p < PB; ++p)
                fb[p][i] = *reinterpret_cast<const bf16x8_t*>(&Bs[p][(wn + 16 * i + (lane & 15)) * LS + (lane >> 4) * 8]);
        }
        constexpr int PM = PA > PB ? PA : PB;                 // parts i, j with i + j >= PM are below 24 bits
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int p = PA - 1; p >= 0; --p)
#pragma unroll
                    for (int r = PB - 1; r >= 0; --r)
                        if (p + r < PM) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[p][i], fb[r][j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t m = m0 + wm + 16 * i + (lane >> 4) * 4 + e, n = n0 + wn + 16 * j + (lane & 15);
                if (m < M && n < N) put_c(c + m * ldc + n, acc[i][j][e]);
            }
}

// a strip of 512 columns and every gridDim.y-th group of 4 rows
template <class T>
__global__ __launch_bounds__(256) void k_block_column_sums(int64_t rows, int64_t cols, const T* __restrict__ dy, int64_t lddy,
                                                           float* __restrict__ part) {
    __shared__ float sh[4][512];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = blockIdx.x * 512ll + lane * 8;
    float s[8] = {};
    if (col < cols)
        for (int64_t r = blockIdx.y * 4ll + w; r < rows; r += gridDim.y * 4ll) {
            float v[8];
            load8(dy + r * lddy, col, cols, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[e];
        }
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[w][lane * 8 + e] = s[e];
    __syncthreads();
    for (int j = threadIdx.x; j < 512; j += 256) {
        const int64_t cc = blockIdx.x * 512ll + j;
        if (cc < cols) part[blockIdx.y * cols + cc] = ((sh[0][j] + sh[1][j]) + sh[2][j]) + sh[3][j];
    }
}

static int64_t bias_strips(int64_t T, int64_t O) {
    int64_t s = 1024 / ceil_div(O, 512);
    if (s < 1) s = 1;
    const int64_t most = ceil_div(T, 4);
    return most < s ? most : s;
}
static size_t backward_workspace(int64_t T, int64_t O, int64_t) {
    if (T <= 0 || O <= 0) return 0;
    return ((size_t)bias_strips(T, O) * O * 4 + 255) / 256 * 256;
}

template <class TA, bool TRANS, class TC>
static dmmv_status grad(int64_t M, int64_t N, int64_t Kc, const TA* a, int64_t lda, const dmmv_block_matrix* b, TC* c, int64_t ldc,
                        hipStream_t s) {
    if (M == 0 || N == 0) return DMMV_OK;
    const int64_t tiles_m = ceil_div(M, 64), tiles_n = ceil_div(N, 64);
    if (tiles_m > INT32_MAX / tiles_n) return fail(DMMV_ERR_SHAPE, "gradient: more tiles than a launch takes");
    constexpr int PA = sizeof(TA) == 4 ? 3 : 1;
    const dim3 grid((unsigned)(tiles_m * tiles_n));
    const bool exact = !b->scales || b->scale_type == DMMV_E8M0;
    if (exact)
        hipLaunchKernelGGL((k_block_grad<TA, TRANS, PA, 1, TC>), grid, dim3(256), 0, s, M, N, Kc, a, lda, layer_view(b), c, ldc, tiles_n);
    else
        hipLaunchKernelGGL((k_block_grad<TA, TRANS, PA, 3, TC>), grid, dim3(256), 0, s, M, N, Kc, a, lda, layer_view(b), c, ldc, tiles_n);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T>
static dmmv_status backward(int64_t Tn, int64_t O, int64_t K, const T* dy, int64_t lddy, const dmmv_block_matrix* x,
                            const dmmv_block_matrix* w, T* dx, int64_t lddx, float* dw, int64_t lddw, float* dbias, void* ws, hipStream_t s) {
    if (dx) DMMV_TRY((grad<T, false, T>(Tn, K, O, dy, lddy, w, dx, lddx, s)));
    if (dw) DMMV_TRY((grad<T, true, float>(O, K, Tn, dy, lddy, x, dw, lddw, s)));
    if (dbias && O > 0) {
        float* part = static_cast<float*>(ws);
        const int64_t strips = Tn > 0 ? bias_strips(Tn, O) : 0;
        if (strips) {
            hipLaunchKernelGGL((k_block_column_sums<T>), dim3((unsigned)ceil_div(O, 512), (unsigned)strips), dim3(256), 0, s, Tn, O, dy,
                               lddy, part);
            DMMV_LAUNCH_CHECK();
        }
        DMMV_TRY(layer_sum_parts(part, strips, O, dbias, O, nullptr, s));
    }
    return DMMV_OK;
}

}  // namespace dmmv

using namespace dmmv;

extern "C" size_t dmmv_block_backward_workspace_bytes(int64_t T, int64_t O, int64_t K) {
    if (layer_check_sizes(T, O, "dy") != DMMV_OK || layer_check_sizes(O, K, "w") != DMMV_OK) return 0;
    return backward_workspace(T, O, K);
}

extern "C" dmmv_status dmmv_block_backward(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy,
                                           const dmmv_block_matrix* x, const dmmv_block_matrix* w, void* dx, int64_t lddx, float* dw,
                                           int64_t lddw, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(T, O, "dy"));
    DMMV_TRY(layer_check_sizes(O, K, "w"));
    const int width = layer_width(dtype);
    DMMV_TRY(layer_check_array(dy, T, O, lddy, width, "dy"));
    if (dx) {
        DMMV_TRY(layer_check_block(w, false, "w"));
        if (w->rows != O || w->cols != K) return fail(DMMV_ERR_SHAPE, "w is not %lld x %lld", (long long)O, (long long)K);
        DMMV_TRY(layer_check_array(dx, T, K, lddx, width, "dx"));
    }
    if (dw) {
        DMMV_TRY(layer_check_block(x, false, "x"));
        if (x->rows != T || x->cols != K) return fail(DMMV_ERR_SHAPE, "x is not %lld x %lld", (long long)T, (long long)K);
        DMMV_TRY(layer_check_array(dw, O, K, lddw, 4, "dw"));
    }
    if ((uintptr_t)dbias % 4) return fail(DMMV_ERR_SHAPE, "dbias is not aligned to its elements");
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, backward_workspace(T, O, K)));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dtype == DMMV_F32)
        return backward(T, O, K, static_cast<const float*>(dy), lddy, x, w, static_cast<float*>(dx), lddx, dw, lddw, dbias, workspace, s);
    return backward(T, O, K, static_cast<const bf16_t*>(dy), lddy, x, w, static_cast<bf16_t*>(dx), lddx, dw, lddw, dbias, workspace, s);
}
