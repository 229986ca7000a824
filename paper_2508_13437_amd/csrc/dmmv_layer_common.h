// Shared by the operators of a quantised linear layer (include/dmmv_layer.h): checks of block
// matrices, the e4m3 block format on the device, loads and stores of eight columns a lane.
#pragma once

#include "dmmv_common.h"
#include "../../include/dmmv_layer.h"

namespace dmmv {

// A block matrix as kernels take it.
struct BlockView {
    uint8_t* codes;
    int64_t ld;
    void* scales;         // NULL: all 1
    int64_t srow, sblk;
    int32_t e8m0;         // scales are exponent bytes, else float
    int32_t shift;        // log2(rows per scale): 0 or 7
};

// host checks; `what` names the argument in the message
dmmv_status layer_check_dtype(int32_t dtype);
dmmv_status layer_check_sizes(int64_t rows, int64_t cols, const char* what);
// a row-major array of elements of `width` bytes (empty ones may be NULL)
dmmv_status layer_check_array(const void* p, int64_t rows, int64_t cols, int64_t ld, int width, const char* what);
dmmv_status layer_check_block(const dmmv_block_matrix* q, bool output, const char* what);
dmmv_status layer_check_workspace(const void* ws, size_t have, size_t need);
BlockView layer_view(const dmmv_block_matrix* q);      // all zero for NULL

static inline int layer_width(int32_t dtype) { return dtype == DMMV_BF16 ? 2 : 4; }

// out[j] = sum over the parts of part[p][j], in an order that the number of parts fixes;
// the first n0 columns go to out0, the others to out1 (either may be NULL)
dmmv_status layer_sum_parts(const float* part, int64_t parts, int64_t n, float* out0, int64_t n0, float* out1,
                            hipStream_t stream);

// a copy of the codes with rows of ld bytes (a multiple of 16), zeros after the columns
dmmv_status layer_lay_codes(const dmmv_block_matrix* q, uint8_t* out, int64_t ld, hipStream_t stream);

#ifdef __HIPCC__

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
// 16 and 8 bytes at any address of the element's own alignment: global loads need no more
typedef uint32_t piece16 __attribute__((ext_vector_type(4)));
typedef uint32_t piece8 __attribute__((ext_vector_type(2)));
typedef piece16 piece16_any __attribute__((aligned(1)));
typedef piece8 piece8_any __attribute__((aligned(1)));

struct bf16_t { uint16_t u; };

__device__ __forceinline__ float bf16_value(uint32_t low16) { return __uint_as_float(low16 << 16); }
// nearest, ties to even; NaN stays NaN
__device__ __forceinline__ uint32_t bf16_bits(float v) {
    const __bf16 b = (__bf16)v;
    return (uint32_t)__builtin_bit_cast(uint16_t, b);
}

// eight columns of a row from `col` on, zero past `cols`
__device__ __forceinline__ void load8(const float* __restrict__ row, int64_t col, int64_t cols, float (&v)[8]) {
    if (col + 8 <= cols) {
        const piece16 a = *reinterpret_cast<const piece16_any*>(row + col), b = *reinterpret_cast<const piece16_any*>(row + col + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[i + 4] = __uint_as_float(b[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? row[col + i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const bf16_t* __restrict__ row, int64_t col, int64_t cols, float (&v)[8]) {
    if (col + 8 <= cols) {
        const piece16 a = *reinterpret_cast<const piece16_any*>(row + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_value(a[i] & 0xFFFFu); v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? bf16_value(row[col + i].u) : 0.0f;
    }
}
__device__ __forceinline__ void store8(float* __restrict__ row, int64_t col, int64_t cols, const float (&v)[8]) {
    if (col + 8 <= cols) {
        piece16 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[i] = __float_as_uint(v[i]); b[i] = __float_as_uint(v[i + 4]); }
        *reinterpret_cast<piece16_any*>(row + col) = a;
        *reinterpret_cast<piece16_any*>(row + col + 4) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = v[i];
    }
}
__device__ __forceinline__ void store8(bf16_t* __restrict__ row, int64_t col, int64_t cols, const float (&v)[8]) {
    if (col + 8 <= cols) {
        piece16 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = bf16_bits(v[2 * i]) | (bf16_bits(v[2 * i + 1]) << 16);
        *reinterpret_cast<piece16_any*>(row + col) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i].u = (uint16_t)bf16_bits(v[i]);
    }
}
__device__ __forceinline__ piece8 load8_codes(const uint8_t* __restrict__ row, int64_t col, int64_t cols) {
    if (col + 8 <= cols) return *reinterpret_cast<const piece8_any*>(row + col);
    piece8 a = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) a[i >> 2] |= (uint32_t)row[col + i] << (8 * (i & 3));
    return a;
}
__device__ __forceinline__ void store8_codes(uint8_t* __restrict__ row, int64_t col, int64_t cols, piece8 a) {
    if (col + 8 <= cols) {
        *reinterpret_cast<piece8_any*>(row + col) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = (uint8_t)(a[i >> 2] >> (8 * (i & 3)));
    }
}

// ---- scales ---------------------------------------------------------------------------------
__device__ __forceinline__ float e8m0_value(uint32_t b) {
    return __uint_as_float(b == 255u ? 0x7FC00000u : b == 0u ? 0x00400000u : b << 23);
}
// a scale as it is stored, and its value; apart, because a conversion waits for the load
__device__ __forceinline__ uint32_t scale_bits(const BlockView& q, int64_t row, int64_t block) {
    if (!q.scales) return q.e8m0 ? 127u : 0x3F800000u;
    const int64_t at = (row >> q.shift) * q.srow + block * q.sblk;
    return q.e8m0 ? static_cast<const uint8_t*>(q.scales)[at] : static_cast<const uint32_t*>(q.scales)[at];
}
__device__ __forceinline__ float scale_of(const BlockView& q, uint32_t bits) { return q.e8m0 ? e8m0_value(bits) : __uint_as_float(bits); }
__device__ __forceinline__ float scale_at(const BlockView& q, int64_t row, int64_t block) { return scale_of(q, scale_bits(q, row, block)); }
// The same for loops that may not wait between a request and its use: the aligned word that holds the scale, always loaded (without
// scales some word of the codes), and what it means.  A branch around a load makes the compiler wait for all loads.
__device__ __forceinline__ const __attribute__((address_space(1))) uint32_t* scale_word(const BlockView& q, int64_t at) {
    const uintptr_t p = q.scales ? reinterpret_cast<uintptr_t>(q.scales) + (q.e8m0 ? at : 4 * at) : reinterpret_cast<uintptr_t>(q.codes);
    // (a pointer made of a number is not known to be one to global memory: its load would be counted with those of the LDS)
    return (const __attribute__((address_space(1))) uint32_t*)(p & ~(uintptr_t)3);
}
__device__ __forceinline__ uint32_t word_bits(const BlockView& q, int64_t at, uint32_t word) {
    const uint32_t byte = (word >> (8 * ((reinterpret_cast<uintptr_t>(q.scales) + at) & 3))) & 0xFFu;      // (no branch)
    const uint32_t there = q.e8m0 ? byte : word, one = q.e8m0 ? 127u : 0x3F800000u;
    return q.scales ? there : one;
}
// acc + p a b for a sum p of products of codes and the scales a, b of its operands.  The scales are multiplied first where their product is
// a normal number, as p (2^-18 to 2^49, or 0) then leaves the range only where the result does.  Otherwise p meets the larger one first: beyond
// the range both are over 1, below it p times the larger keeps its bits.
__device__ __forceinline__ float add_scaled(float p, float a, float b, float acc) {
    const float c = a * b;
    if (__builtin_amdgcn_classf(c, 0x108) || a == 0.0f || b == 0.0f) return dmmv_fma(p, c, acc);
    return fabsf(a) > fabsf(b) ? dmmv_fma(p * a, b, acc) : dmmv_fma(p * b, a, acc);
}
// the same with scales that are exponent bytes
__device__ __forceinline__ float times_exponents(float p, uint32_t a, uint32_t b) {
    return max(a, b) == 255u ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(p, (int)(a + b) - 254);
}
// The scales met so far need no such care: all are 2^-62 to 2^63, so that products of two are normal numbers, or 0, or not finite
struct ScaleRange {
    uint32_t lo = ~0u, hi = 0u;                      // magnitudes as bits, doubled; lo less 1, so that 0 does not count
    __device__ __forceinline__ void take(float s) {
        const uint32_t u = __float_as_uint(s) << 1;
        hi = max(hi, u < 0xFF000000u ? u : 0u);
        lo = min(lo, u - 1u);
    }
    __device__ __forceinline__ bool small() const { return lo < (65u << 24) - 1u; }
    __device__ __forceinline__ bool large() const { return hi >= (190u << 24); }
    __device__ __forceinline__ bool moderate() const { return !small() && !large(); }
};
// A scale that is the same along a row leaves the sum, but its exponent (as a scale's byte) goes in where those of blocks go, so that the sum
// has the result's size; what is left of it, `rest`, is 1 to 2 (for exponents outside what scaled8 takes a little more or less; 0, infinite or NaN as the scale).
struct RowScale {
    uint32_t byte;
    float rest;
};
__device__ __forceinline__ RowScale row_scale(float s) {
    const uint32_t e = (__float_as_uint(s) >> 23) & 255u, byte = e == 255u ? 127u : min(max(e, 3u), 246u);
    return RowScale{byte, s * __uint_as_float((254u - byte) << 23)};         // exact
}
__device__ __forceinline__ void scale_put(const BlockView& q, int64_t scale_row, int64_t block, uint32_t b) {
    const int64_t at = scale_row * q.srow + block * q.sblk;
    if (q.e8m0) static_cast<uint8_t*>(q.scales)[at] = (uint8_t)b;
    else static_cast<float*>(q.scales)[at] = e8m0_value(b);
}

// |x| as bits if finite, else 0 (the order of non-negative floats is that of their bits)
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}
// exponent byte of the smallest power of two >= a / 448: 448 = 1.75 * 2^8, so it is a's own exponent
// less 8, or less 7 where a's fraction is over 0.75
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
    if (a == 0u) return 127u;
    const int e = (int)(a >> 23) - 8 + ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1u : (uint32_t)e;
}
// eight values to codes, scale 2^(b - 127) with 1 <= b <= 247; the conversion rounds to nearest even
__device__ __forceinline__ piece8 encode8(const float (&v)[8], uint32_t b) {
    const float inv = __uint_as_float((254u - b) << 23);
    piece8 r;
    uint32_t most = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inv, v[4 * h + 1] * inv, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inv, v[4 * h + 3] * inv, w, true);
        r[h] = (uint32_t)w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    if (most >= 0x7F800000u) {               // infinities and NaN: one code for all
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((__float_as_uint(v[i]) & 0x7FFFFFFFu) >= 0x7F800000u)
                r[i >> 2] = (r[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | (0x7Fu << (8 * (i & 3)));
    }
    return r;
}
__device__ __forceinline__ void decode8(piece8 c, float scale, float (&v)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
        v[4 * h] = lo[0] * scale; v[4 * h + 1] = lo[1] * scale;
        v[4 * h + 2] = hi[0] * scale; v[4 * h + 3] = hi[1] * scale;
    }
}

// maximum over each row of 16 lanes (one block of 128 columns), in all its lanes; all 64 lanes active
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    v = max(v, dpp_u32<DPP_QUAD_XOR1>(v));
    v = max(v, dpp_u32<DPP_QUAD_XOR2>(v));
    v = max(v, dpp_u32<DPP_ROW_HALF_MIRROR>(v));
    return max(v, dpp_u32<DPP_ROW_MIRROR>(v));
}
__device__ __forceinline__ uint32_t max8_bits(const float (&v)[8]) {
    uint32_t a = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, finite_bits(v[i]));
    return a;
}
// sum over the wavefront in a fixed order, the same value in every lane; all 64 lanes active
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp_mov<DPP_QUAD_XOR1>(v);
    v += dpp_mov<DPP_QUAD_XOR2>(v);
    v += dpp_mov<DPP_ROW_HALF_MIRROR>(v);
    v += dpp_mov<DPP_ROW_MIRROR>(v);
    return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}

// A 32-bit number as the sum of three bf16 (8 + 8 + 8 significant bits, by truncation).  An infinity or NaN
// stays whole in the first.
__device__ __forceinline__ void split3(float x, uint32_t (&p)[3]) {
    const uint32_t u = __float_as_uint(x);
    const float r1 = x - __uint_as_float(u & 0xFFFF0000u);
    const uint32_t u1 = __float_as_uint(r1) & 0xFFFF0000u;
    const float r2 = r1 - __uint_as_float(u1);
    p[0] = u >> 16; p[1] = u1 >> 16; p[2] = __float_as_uint(r2) >> 16;
    if ((u & 0x7F800000u) == 0x7F800000u) {
        p[0] |= (u & 0x7FFFFFu) ? 0x40u : 0u;
        p[1] = p[2] = 0u;
    }
}
// eight of them, as the words of three rows of eight bf16
template <int PARTS>
__device__ __forceinline__ void split8(const float (&v)[8], piece16 (&w)[3]) {
    uint32_t most = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    if (most < 0x7F800000u) {                        // all finite: no selection between the parts
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
#pragma unroll
            for (int e = 0; e < 8; e += 2)           // the upper halves of two words
                w[k][e >> 1] = __builtin_amdgcn_perm(__float_as_uint(r[e + 1]), __float_as_uint(r[e]), 0x07060302u);
            if (k + 1 < PARTS)
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] -= __uint_as_float(__float_as_uint(r[e]) & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            uint32_t p[3], q[3];
            split3(v[e], p);
            split3(v[e + 1], q);
#pragma unroll
            for (int k = 0; k < PARTS; ++k) w[k][e >> 1] = p[k] | (q[k] << 16);
        }
    }
}

// ---- eight numbers of a row as they are stored, and what a row's end cuts off -----------------------
// A piece is loaded whole, from `moved` places further left where the row ends inside it, and put right when it is used:
// the request does not wait.  Rows shorter than 8 are read one by one.
template <class T> struct Raw8;
template <> struct Raw8<float> {
    piece16 v[2];
    __device__ __forceinline__ void load(const float* p) {
        v[0] = *reinterpret_cast<const piece16_any*>(p);
        v[1] = *reinterpret_cast<const piece16_any*>(p + 4);
    }
    __device__ __forceinline__ void set(int i, float x) { v[i >> 2][i & 3] = __float_as_uint(x); }
    __device__ __forceinline__ void right(int n) {   // by n < 8 numbers, zeros after them
#pragma unroll
        for (int s = 4; s >= 1; s >>= 1)
            if (n & s) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = i + s < 8 ? v[(i + s) >> 2][(i + s) & 3] : 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = w[i];
            }
    }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(v[i >> 2][i & 3]); }
};
template <> struct Raw8<bf16_t> {
    piece16 v;
    __device__ __forceinline__ void load(const bf16_t* p) { v = *reinterpret_cast<const piece16_any*>(p); }
    __device__ __forceinline__ void set(int i, bf16_t x) { v[i >> 1] |= (uint32_t)x.u << (16 * (i & 1)); }
    __device__ __forceinline__ void right(int n) {
        const uint64_t lo = v[0] | ((uint64_t)v[1] << 32), hi = v[2] | ((uint64_t)v[3] << 32);
        const int s = 16 * n;
        const uint64_t l = s >= 64 ? hi >> (s - 64) : s == 0 ? lo : (lo >> s) | (hi << (64 - s)), h = s >= 64 ? 0 : hi >> s;
        v = piece16{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? __uint_as_float(v[i >> 1] & 0xFFFF0000u) : bf16_value(v[i >> 1] & 0xFFFFu); }
};
template <> struct Raw8<uint8_t> {
    piece8 v;
    __device__ __forceinline__ void load(const uint8_t* p) { v = *reinterpret_cast<const piece8_any*>(p); }
    __device__ __forceinline__ void set(int i, uint8_t x) { v[i >> 2] |= (uint32_t)x << (8 * (i & 3)); }
    __device__ __forceinline__ void right(int n) {
        const uint64_t w = (v[0] | ((uint64_t)v[1] << 32)) >> (8 * n);
        v = piece8{(uint32_t)w, (uint32_t)(w >> 32)};
    }
};
template <class T>
__device__ __forceinline__ void raw_request(Raw8<T>& r, const T* __restrict__ row, int64_t col, int64_t cols) {
    if (cols >= 8) {
        r.load(row + min(col, cols - 8));
    } else {
        r = Raw8<T>{};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) r.set(i, row[col + i]);
    }
}
// the piece as it belongs: zeros past the row's end, all zero unless `ok`
template <class T>
__device__ __forceinline__ void raw_settle(Raw8<T>& r, int64_t col, int64_t cols, bool ok) {
    const int64_t moved = cols >= 8 ? col - min(col, cols - 8) : 0;
    if (!ok || moved >= 8) r = Raw8<T>{};
    else if (moved > 0) r.right((int)moved);
}

// ---- shared by the tiled products ------------------------------------------------------------
// The workgroup's tile.  Workgroups go to the 8 XCDs in turn, each with an L2 of its own: an XCD gets an eighth of the tiles in
// a row, 4 tiles high and side by side, so that those of one moment share their operands' lines (4096 x 4096 x 11008: 171 us
// against 188 with the tiles in rows; bands of 8: 185).
__device__ __forceinline__ void tile_of_workgroup(int tiles_t, int tiles_o, int& tile_t, int& tile_o) {
    const int n = tiles_t * tiles_o, per = n >> 3, b = (int)blockIdx.x;
    const int id = b < per * 8 ? (b & 7) * per + (b >> 3) : b;
    const int band = id / (4 * tiles_o), high = min(4, tiles_t - 4 * band), in = id - band * 4 * tiles_o;
    // (a division runs on the vector unit: back to scalar registers)
    tile_o = __builtin_amdgcn_readfirstlane(in / high);
    tile_t = __builtin_amdgcn_readfirstlane(4 * band + in % high);
}

// eight codes as bf16, times 2^(b - 127): exact for b from 3 (the smallest code is 2^-133 then, as bf16 is) to 246; NaN for 255
__device__ __forceinline__ bf16x8_t scaled8(int lo, int hi, uint32_t b) {
    const float s = __uint_as_float(b << 23);
    const auto p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true);
    const auto r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true);
    return bf16x8_t{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
}

__device__ __forceinline__ void put_y(float* y, float v) { *y = v; }
__device__ __forceinline__ void put_y(bf16_t* y, float v) { y->u = (uint16_t)bf16_bits(v); }

// four results of a row to the LDS
template <class T>
__device__ __forceinline__ void put4(T* __restrict__ row, const float (&v)[4]);
template <>
__device__ __forceinline__ void put4(float* __restrict__ row, const float (&v)[4]) {
    *reinterpret_cast<floatx4*>(row) = floatx4{v[0], v[1], v[2], v[3]};
}
template <>
__device__ __forceinline__ void put4(bf16_t* __restrict__ row, const float (&v)[4]) {
    *reinterpret_cast<piece8*>(row) = piece8{bf16_bits(v[0]) | (bf16_bits(v[1]) << 16), bf16_bits(v[2]) | (bf16_bits(v[3]) << 16)};
}

typedef int intx4 __attribute__((ext_vector_type(4)));

// `bytes` bytes from p on as a buffer (p the same in every lane): reads past them give zero
__device__ __forceinline__ intx4 buffer_of(const uint8_t* p, uint32_t bytes) {
    const uint64_t u = (uint64_t)p;
    return intx4{__builtin_amdgcn_readfirstlane((int)(uint32_t)u), __builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32) & 0xFFFF),
                 __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}
// 16 bytes a lane from a buffer (offsets: `off` a lane's, `soff` the wavefront's) to 1 KB of the LDS at the uniform address `at`,
// in the order of the lanes; in flight until lds_requests_left().  The instruction writes no register.
__device__ __forceinline__ void lds_request(intx4 buf, uint32_t off, uint32_t soff, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at), "v"(off), "s"(buf), "s"(soff));
}
// until at most N of the wavefront's requests are in flight
template <int N>
__device__ __forceinline__ void lds_requests_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

#endif  // __HIPCC__

}  // namespace dmmv
