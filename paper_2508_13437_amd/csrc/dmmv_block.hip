// Block matrices: host checks, quantising (checkpoints of activations, trained weights) and back.
#include "dmmv_layer_common.h"

namespace dmmv {

// ---- host checks ------------------------------------------------------------------------------
dmmv_status layer_check_dtype(int32_t dtype) {
    if (dtype != DMMV_F32 && dtype != DMMV_BF16) return fail(DMMV_ERR_DTYPE, "dtype %d is not DMMV_F32 / DMMV_BF16", dtype);
    return DMMV_OK;
}

dmmv_status layer_check_sizes(int64_t rows, int64_t cols, const char* what) {
    if (rows < 0 || cols < 0) return fail(DMMV_ERR_SHAPE, "%s: negative size (%lld x %lld)", what, (long long)rows, (long long)cols);
    if (rows > INT32_MAX - 256 || cols > INT32_MAX - 256) return fail(DMMV_ERR_SHAPE, "%s: sizes must fit in 31 bits", what);
    return DMMV_OK;
}

dmmv_status layer_check_array(const void* p, int64_t rows, int64_t cols, int64_t ld, int width, const char* what) {
    if (rows == 0 || cols == 0) return DMMV_OK;
    if (!p) return fail(DMMV_ERR_NULL, "%s is NULL", what);
    if (ld < cols && rows > 1) return fail(DMMV_ERR_SHAPE, "%s: row stride %lld < %lld columns", what, (long long)ld, (long long)cols);
    if (ld < 0 || ld > INT64_MAX / 16 / (rows > 0 ? rows : 1)) return fail(DMMV_ERR_SHAPE, "%s: row stride out of range", what);
    if ((uintptr_t)p % width) return fail(DMMV_ERR_SHAPE, "%s is not aligned to its elements", what);
    return DMMV_OK;
}

dmmv_status layer_check_block(const dmmv_block_matrix* q, bool output, const char* what) {
    if (!q) return fail(DMMV_ERR_NULL, "%s is NULL", what);
    DMMV_TRY(layer_check_sizes(q->rows, q->cols, what));
    if (q->scale_type != DMMV_E8M0 && q->scale_type != DMMV_F32)
        return fail(DMMV_ERR_DTYPE, "%s: scale_type %d is not DMMV_E8M0 / DMMV_F32", what, q->scale_type);
    if (q->scale_rows != 1 && q->scale_rows != 128) return fail(DMMV_ERR_SHAPE, "%s: scale_rows is not 1 or 128", what);
    if (q->rows == 0 || q->cols == 0) return DMMV_OK;
    DMMV_TRY(layer_check_array(q->codes, q->rows, q->cols, q->ld, 1, what));
    const int64_t nr = ceil_div(q->rows, q->scale_rows), nb = ceil_div(q->cols, 128);
    const int64_t sr = q->scale_row_stride, sb = q->scale_block_stride;
    if (q->scales) {
        if (sr < 0 || sb < 0 || sr > INT64_MAX / 16 / nr || sb > INT64_MAX / 16 / nb)
            return fail(DMMV_ERR_SHAPE, "%s: scale strides out of range", what);
        if (q->scale_type == DMMV_F32 && (uintptr_t)q->scales % 4) return fail(DMMV_ERR_SHAPE, "%s: scales are not aligned to 4 bytes", what);
    } else if (output) {
        return fail(DMMV_ERR_NULL, "%s: scales is NULL", what);
    }
    if (output) {
        const bool by_rows = sb >= 1 && (nr == 1 || sr >= (nb - 1) * sb + 1);
        const bool by_blocks = sr >= 1 && (nb == 1 || sb >= (nr - 1) * sr + 1);
        if (!by_rows && !by_blocks) return fail(DMMV_ERR_SHAPE, "%s: scales overlap", what);
    }
    return DMMV_OK;
}

dmmv_status layer_check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return DMMV_OK;
    if (!ws) return fail(DMMV_ERR_WORKSPACE, "workspace is NULL, %zu bytes needed", need);
    if ((uintptr_t)ws % 256) return fail(DMMV_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (have < need) return fail(DMMV_ERR_WORKSPACE, "workspace too small: %zu bytes, %zu needed", have, need);
    return DMMV_OK;
}

BlockView layer_view(const dmmv_block_matrix* q) {
    BlockView v = {};
    if (!q) return v;
    v.codes = static_cast<uint8_t*>(q->codes);
    v.ld = q->ld;
    v.scales = q->rows == 0 || q->cols == 0 ? nullptr : q->scales;      // (an empty matrix need not have any)
    v.srow = q->scale_row_stride;
    v.sblk = q->scale_block_stride;
    v.e8m0 = q->scale_type == DMMV_E8M0;
    v.shift = q->scale_rows == 128 ? 7 : 0;
    return v;
}

// ---- quantise ---------------------------------------------------------------------------------
// A lane takes 8 columns, so 16 lanes (one DPP row) take a block of 128 and find its largest value
// without the LDS.  One pass, bound by memory: 11008 x 4096 from 32 bits 31.4 us (7.2 TB/s), 4096 x 11008 from bf16 24.4 (5.5).
template <class T>
__global__ __launch_bounds__(256) void k_block_quantize_rows(int64_t rows, int64_t cols, int64_t nb, const T* __restrict__ x,
                                                             int64_t ldx, BlockView q) {
    const int64_t g = (blockIdx.x * 256ll + threadIdx.x) >> 4;
    const int64_t row = g / nb, blk = g - row * nb;
    const int64_t col = blk * 128 + (threadIdx.x & 15) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < rows) load8(x + row * ldx, col, cols, v);
    const uint32_t b = scale_byte(row16_max(max8_bits(v)));
    if (row >= rows) return;
    store8_codes(q.codes + row * q.ld, col, cols, encode8(v, b));
    if ((threadIdx.x & 15) == 0) scale_put(q, row, blk, b);
}

// 128 x 128 blocks: one workgroup holds its block in registers (8 rows of 8 columns a thread).  11008 x 4096 from 32 bits: 34 us,
// 6.6 TB/s.
template <class T>
__global__ __launch_bounds__(256) void k_block_quantize_tiles(int64_t rows, int64_t cols, int64_t nb, const T* __restrict__ x,
                                                              int64_t ldx, BlockView q) {
    __shared__ uint32_t top[4];
    const int64_t br = blockIdx.x / nb, blk = blockIdx.x - br * nb;
    const int64_t col = blk * 128 + (threadIdx.x & 15) * 8, row0 = br * 128 + (threadIdx.x >> 4);
    float v[8][8];
    uint32_t a = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
        if (row0 + 16 * i < rows) load8(x + (row0 + 16 * i) * ldx, col, cols, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, max8_bits(v[i]));
    a = row16_max(a);
    a = max(max((uint32_t)__builtin_amdgcn_readlane((int)a, 0), (uint32_t)__builtin_amdgcn_readlane((int)a, 16)),
            max((uint32_t)__builtin_amdgcn_readlane((int)a, 32), (uint32_t)__builtin_amdgcn_readlane((int)a, 48)));
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = a;
    __syncthreads();
    const uint32_t b = scale_byte(max(max(top[0], top[1]), max(top[2], top[3])));
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (row0 + 16 * i < rows) store8_codes(q.codes + (row0 + 16 * i) * q.ld, col, cols, encode8(v[i], b));
    if (threadIdx.x == 0) scale_put(q, br, blk, b);
}

// A code times a scale of 24 bits, for a result that is rounded to fewer: 28 bits, cut to 32-bit form with the last bit set where something was
// cut off, so that the second rounding is the only one.  What the product's rounding took away is exact in 32 bits while the scale is moderate,
// else in 64 (4096 x 11008 to bf16: 24.7 us, 27.2 with 64 bits throughout).
__device__ __forceinline__ float cut(float f, bool inexact, bool too_large) {
    const uint32_t u = __float_as_uint(f);           // (NaN stays NaN)
    return inexact ? __uint_as_float((too_large ? u - 1u : u) | 1u) : f;
}
__device__ __forceinline__ float cut_product(float code, float scale) {
    const float f = code * scale, rest = dmmv_fma(code, scale, -f);
    return cut(f, rest != 0.0f, (__float_as_uint(rest) ^ __float_as_uint(f)) >> 31);
}
__device__ __forceinline__ float cut_product64(float code, float scale) {
    const double d = (double)code * (double)scale;
    const float f = (float)d;
    return cut(f, (double)f != d, fabs((double)f) > fabs(d));
}

// 8 columns a lane, rounded once: values are exact in 32 bits with power-of-two scales, and with others cut_product makes bf16 of them.
// 11008 x 4096: to bf16 22.9 us (5.9 TB/s), to 32 bits 34 (6.6).
template <class T>
__global__ __launch_bounds__(256) void k_block_dequantize(int64_t rows, int64_t cols, int64_t chunks, BlockView q,
                                                          T* __restrict__ x, int64_t ldx) {
    const int64_t g = blockIdx.x * 256ll + threadIdx.x;
    const int64_t row = g / chunks, col = (g - row * chunks) * 8;
    if (row >= rows) return;
    float v[8];
    const float s = scale_at(q, row, col >> 7);
    const piece8 c = load8_codes(q.codes + row * q.ld, col, cols);
    if (sizeof(T) == 4 || q.e8m0) {
        decode8(c, s, v);
    } else {
        decode8(c, 1.0f, v);
        ScaleRange r;
        r.take(s);
        if (r.moderate() && fabsf(s) < __builtin_huge_valf()) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = cut_product(v[e], s);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = cut_product64(v[e], s);
        }
    }
    store8(x + row * ldx, col, cols, v);
}

// ---- sums of parts (the second stage of every reduction over rows) -------------------------------
// A workgroup takes 64 columns; its 16 wavefronts read every 16th part each, in 8 chains, and are joined in order: the same
// sum for every run.  Bound by the latency of the chains: 256 parts of 2 x 4096 numbers 3.9 us.
__global__ __launch_bounds__(1024) void k_layer_sum_parts(const float* __restrict__ part, int64_t parts, int64_t n,
                                                          float* __restrict__ out0, int64_t n0, float* __restrict__ out1) {
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t j = blockIdx.x * 64ll + lane;
    // eight parts' numbers are requested together, a chain of sums for each
    float c[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (j < n) {
        int64_t p = w;
        for (; p + 112 < parts; p += 128)
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] += part[(p + 16 * u) * n + j];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (p + 16 * u < parts) c[u] += part[(p + 16 * u) * n + j];
    }
    float s = ((c[0] + c[1]) + (c[2] + c[3])) + ((c[4] + c[5]) + (c[6] + c[7]));
    sh[w][lane] = s;
    __syncthreads();
    if (w != 0 || j >= n) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sh[i][lane];
    float* out = j < n0 ? out0 : out1;
    if (out) out[j < n0 ? j : j - n0] = s;
}

dmmv_status layer_sum_parts(const float* part, int64_t parts, int64_t n, float* out0, int64_t n0, float* out1,
                            hipStream_t stream) {
    if (n <= 0) return DMMV_OK;
    hipLaunchKernelGGL(k_layer_sum_parts, dim3((unsigned)ceil_div(n, 64)), dim3(1024), 0, stream, part, parts, n, out0, n0, out1);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

// Codes with rows of whole aligned chunks of 16 bytes, for the large tiles.
__global__ __launch_bounds__(256) void k_block_lay_codes(int64_t rows, int64_t cols, const uint8_t* __restrict__ codes, int64_t ld,
                                                         uint8_t* __restrict__ out, int64_t Kp) {
    const int64_t i = blockIdx.x * 256ll + threadIdx.x, chunks = Kp >> 4, row = i / chunks, col = (i - row * chunks) * 16;
    if (row >= rows) return;
    const piece8 a = load8_codes(codes + row * ld, col, cols), b = load8_codes(codes + row * ld, col + 8, cols);
    *reinterpret_cast<piece16*>(out + row * Kp + col) = piece16{a[0], a[1], b[0], b[1]};
}

dmmv_status layer_lay_codes(const dmmv_block_matrix* q, uint8_t* out, int64_t ld, hipStream_t stream) {
    const int64_t grid = ceil_div(q->rows * (ld / 16), 256);
    if (grid > INT32_MAX) return fail(DMMV_ERR_SHAPE, "more codes than a launch takes");
    hipLaunchKernelGGL(k_block_lay_codes, dim3((unsigned)grid), dim3(256), 0, stream, q->rows, q->cols, static_cast<const uint8_t*>(q->codes), q->ld, out, ld);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T>
static dmmv_status quantize(const T* x, int64_t ldx, const dmmv_block_matrix* q, hipStream_t stream) {
    const int64_t nb = ceil_div(q->cols, 128);
    const int64_t grid = q->scale_rows == 1 ? ceil_div(q->rows * nb, 16) : ceil_div(q->rows, 128) * nb;
    if (grid > INT32_MAX) return fail(DMMV_ERR_SHAPE, "q: more blocks than a launch takes");
    if (q->scale_rows == 1)
        hipLaunchKernelGGL((k_block_quantize_rows<T>), dim3((unsigned)grid), dim3(256), 0, stream, q->rows, q->cols, nb, x, ldx, layer_view(q));
    else
        hipLaunchKernelGGL((k_block_quantize_tiles<T>), dim3((unsigned)grid), dim3(256), 0, stream, q->rows, q->cols, nb, x, ldx, layer_view(q));
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T>
static dmmv_status dequantize(const dmmv_block_matrix* q, T* x, int64_t ldx, hipStream_t stream) {
    const int64_t chunks = ceil_div(q->cols, 8), grid = ceil_div(q->rows * chunks, 256);
    if (grid > INT32_MAX) return fail(DMMV_ERR_SHAPE, "q: more elements than a launch takes");
    hipLaunchKernelGGL((k_block_dequantize<T>), dim3((unsigned)grid), dim3(256), 0, stream, q->rows, q->cols, chunks, layer_view(q), x, ldx);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

}  // namespace dmmv

using namespace dmmv;

extern "C" dmmv_status dmmv_block_quantize(int32_t dtype, const void* x, int64_t ldx, const dmmv_block_matrix* q, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_block(q, true, "q"));
    DMMV_TRY(layer_check_array(x, q->rows, q->cols, ldx, layer_width(dtype), "x"));
    if (q->rows == 0 || q->cols == 0) return DMMV_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return dtype == DMMV_F32 ? quantize(static_cast<const float*>(x), ldx, q, s) : quantize(static_cast<const bf16_t*>(x), ldx, q, s);
}

extern "C" dmmv_status dmmv_block_dequantize(const dmmv_block_matrix* q, int32_t dtype, void* x, int64_t ldx, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_block(q, false, "q"));
    DMMV_TRY(layer_check_array(x, q->rows, q->cols, ldx, layer_width(dtype), "x"));
    if (q->rows == 0 || q->cols == 0) return DMMV_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return dtype == DMMV_F32 ? dequantize(q, static_cast<float*>(x), ldx, s) : dequantize(q, static_cast<bf16_t*>(x), ldx, s);
}
