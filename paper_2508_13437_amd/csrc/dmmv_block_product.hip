// Product of two block matrices, y = x w^T + bias (include/dmmv_layer.h).
//
// The 8-bit matrix instructions of gfx950 line the products of a step up against the largest and drop what
// lies some 13 bits below it: against 64 bits their sums are off by 1e-5 to 5e-5 of the result's norm
// (random codes; up to 2^-11 of sum |x w| for single results).  That is far below the rounding of a bf16 result
// (2e-3), so bf16 results are summed by them; 32-bit results are summed by the 16-bit instructions, which keep the
// 32-bit sum (8e-8) at half the rate: a code is exact in f16.
#include <type_traits>

#include "dmmv_activation.h"

namespace dmmv {

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

// 16 codes of a row of which `left` (any number) belong to the row, the others zero; `have` codes of the row lie before
// them.  A piece that the row's end cuts is loaded so that it ends there, and shifted.
__device__ __forceinline__ piece16 chunk_tail(const uint8_t* __restrict__ p, int left, int64_t have) {
    if (left >= 16) return *reinterpret_cast<const piece16_any*>(p);
    piece16 a = {0u, 0u, 0u, 0u};
    if (left <= 0) return a;
    if (have + left >= 16) {
        const piece16 v = *reinterpret_cast<const piece16_any*>(p - (16 - left));
        const uint64_t lo = v[0] | ((uint64_t)v[1] << 32), hi = v[2] | ((uint64_t)v[3] << 32);
        const int s = 8 * (16 - left);               // 8 .. 120
        const uint64_t l = s >= 64 ? hi >> (s - 64) : (lo >> s) | (hi << (64 - s)), h = s >= 64 ? 0 : hi >> s;
        return piece16{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
    }
#pragma unroll
    for (int i = 0; i < 15; ++i)                     // rows shorter than 16
        if (i < left) a[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return a;
}

__device__ __forceinline__ intx8 words8(piece16 a, piece16 b) {
    return intx8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// ---- what becomes of a product ---------------------------------------------------------------------
// The result alone, or with EPI what follows it: v = act(u) + residual of the product u, as y, in 8 bits, or in 32 bits for a
// pass that makes 8 bits of it; and u itself.
template <class T, bool EPI>
struct ProductOut {
    T* y;
    int64_t ldy;
};
template <class T>
struct ProductOut<T, true> {
    T* y;                                // each may be NULL
    int64_t ldy;
    const T* residual;
    int64_t ldr;
    T* u;
    int64_t ldu;
    float* v;                            // [T][O]
    BlockView q;
    int32_t act, has_q;
};

// eight columns of u from `col` on; r the residual's; the 16 lanes of a block of 128 come together
template <class T>
__device__ __forceinline__ void finish8(const ProductOut<T, true>& o, int64_t row, int64_t col, int64_t cols, float (&v)[8], const float (&r)[8]) {
    if (o.u) store8(o.u + row * o.ldu, col, cols, v);
    act_values<sizeof(T) == 2>(o.act, v);
    if (o.residual)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r[e];
    if (o.y) store8(o.y + row * o.ldy, col, cols, v);
    if (!o.has_q) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < cols ? v[e] : 0.0f;
    put_q<T>(o.q, row, col, cols, v);
}
// one number of u
template <class T>
__device__ __forceinline__ void finish1(const ProductOut<T, true>& o, int64_t row, int64_t col, int64_t cols, float u) {
    if (o.u) put_y(o.u + row * o.ldu + col, u);
    float v[1] = {u};
    act_values<false>(o.act, v);
    if (o.residual) v[0] += value_of(o.residual[row * o.ldr + col]);
    if (o.y) put_y(o.y + row * o.ldy + col, v[0]);
    if (o.v) o.v[row * cols + col] = v[0];
}
// What makes u of the sums in a tile, for its columns and rows: u = fma(sum * so, st, bias).  In the LDS.
struct TileScales {
    float *bias, *so, *st;
};
// ROWS x COLS numbers in the LDS (rows of LD floats): u, or with SUMS sums that become it.  256 threads, eight columns of a row a turn, always the
// same ones, and the rows (256 * 8 / COLS a turn) are those of the thread at turn 0 and rows_on(turn) further.  What two turns read of the LDS
// is requested in the two before.  Code that runs once is bound by its fetching, so there is little of it: one piece for whole wavefronts, one for the
// matrix's ends.  Turns in pairs hide one another's waits: there is one wavefront a SIMD.  4096 x 11008 x 4096, us: product 161 (170 by the
// other epilogue), RELU 162, SiLU 172, GELU 180, u beside it 3 to 4 more, in 8 bits instead 10 more (20 with one turn after the other), a residual 4 more
// (12; its requests wait for the stores before them).  With everything unrolled by the compiler the up-projection with GELU and u took 240, now 184.
template <int ROWS, int COLS, int LD, bool Q, bool SUMS, class T, class F>
__device__ __forceinline__ void finish_tile(const ProductOut<T, true>& o, float* tile, const TileScales& k, int64_t row0, int64_t rows, int64_t cols, int64_t col0,
                                            F rows_on) {
    constexpr int PER_ROW = COLS / 8, STEP = 256 / PER_ROW, TURNS = ROWS / STEP;
    static_assert(TURNS % 2 == 0, "turns in pairs");
    const int r0 = (int)threadIdx.x / PER_ROW, h = (int)threadIdx.x % PER_ROW;
    const int64_t col = col0 + h * 8, at0 = row0 + r0;
    const int left = (int)min(cols - col, (int64_t)8), below = (int)min(rows - at0, (int64_t)1 << 20);      // of the columns, of the rows
    T* const y = o.y + at0 * o.ldy + col;
    T* const u = o.u + at0 * o.ldu + col;
    const T* const residual = o.residual + at0 * o.ldr + col;
    uint8_t* const codes = Q ? o.q.codes + at0 * o.q.ld + col : nullptr;
    const int64_t scale0 = Q ? at0 * o.q.srow + (col >> 7) * o.q.sblk : 0;
    auto get8 = [&](const float* p, float (&w)[8]) __attribute__((always_inline)) {
        const floatx4 f0 = *reinterpret_cast<const floatx4*>(p), f1 = *reinterpret_cast<const floatx4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { w[i] = f0[i]; w[4 + i] = f1[i]; }
    };
    float so[8], bias[8];
    if constexpr (SUMS) {
        if (k.so) get8(k.so + h * 8, so);
        get8(k.bias + h * 8, bias);
    }
    float* const mine = tile + r0 * LD + h * 8;
    // u of a turn
    struct Sums {
        float v[8], st;
    };
    auto read = [&](int turn, Sums& x) __attribute__((always_inline)) {
        get8(mine + turn * (STEP * LD), x.v);
        if constexpr (SUMS) x.st = k.st[r0 + rows_on(turn)];
    };
    auto u_of = [&](const Sums& x, float* v) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = x.v[e];
            if constexpr (SUMS) v[e] = dmmv_fma(k.so ? v[e] * so[e] : v[e], x.st, bias[e]);
        }
    };
    auto scale_to = [&](int on, uint32_t scale) __attribute__((always_inline)) {
        if ((threadIdx.x & 15) != 0) return;
        if (o.q.e8m0) static_cast<uint8_t*>(o.q.scales)[scale0 + on * o.q.srow] = (uint8_t)scale;
        else static_cast<float*>(o.q.scales)[scale0 + on * o.q.srow] = e8m0_value(scale);
    };
    Sums next[2];
    read(0, next[0]);
    read(1, next[1]);
#pragma unroll 1
    for (int turn = 0; turn < TURNS; turn += 2) {
        const int on[2] = {rows_on(turn), rows_on(turn + 1)};        // (the same for all)
        // (rows come in order; a wavefront's lanes go together, for the largest of 128)
        if (__all(on[1] < below && left >= 8)) {
            float v[2][8];
            Raw8<T> res[2];                          // (a turn ahead they would wait for the stores before them: 28 us more at 4096 x 11008 x 4096)
            if (o.residual) {
                res[0].load(residual + on[0] * o.ldr);
                res[1].load(residual + on[1] * o.ldr);
            }
            u_of(next[0], v[0]);
            u_of(next[1], v[1]);
            if (turn + 2 < TURNS) {
                read(turn + 2, next[0]);
                read(turn + 3, next[1]);
            }
            if (o.u)
#pragma unroll
                for (int i = 0; i < 2; ++i) store8(u + on[i] * o.ldu, 0, 8, v[i]);
            act_values<sizeof(T) == 2>(o.act, v);
            if (o.residual)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] += res[i].get(e);
            if (o.y)
#pragma unroll
                for (int i = 0; i < 2; ++i) store8(y + on[i] * o.ldy, 0, 8, v[i]);
            if (!Q && o.v)
#pragma unroll
                for (int i = 0; i < 2; ++i) store8(o.v + (at0 + on[i]) * cols + col, 0, 8, v[i]);
            if constexpr (Q) {
                if (!o.has_q) continue;
                uint32_t most[2], scale[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) most[i] = row16_max(most8(v[i]));
                piece8 code[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    scale[i] = scale_byte(most[i]);
                    code[i] = encode8_finite(v[i], scale[i]);
                }
                if (__any(max(most[0], most[1]) >= 0x7F800000u))
#pragma unroll
                    for (int i = 0; i < 2; ++i) code[i] = quantize8(v[i], scale[i]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    *reinterpret_cast<piece8_any*>(codes + on[i] * o.q.ld) = code[i];
                    scale_to(on[i], scale[i]);
                }
            }
            continue;
        }
        // the matrix ends in this wavefront's rows or columns
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            const int at = rows_on(turn + i);
            const bool ok = at < below && left > 0;
            float v[8];
            Sums x;
            read(turn + i, x);
            u_of(x, v);
            const int there = ok ? left : 0;         // of the columns
            if (o.u) store8(u + at * o.ldu, 0, there, v);
            act_values<sizeof(T) == 2>(o.act, v);
            if (o.residual) {
                float r[8];
                load8(residual + at * o.ldr, 0, there, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += r[e];
            }
            if (o.y) store8(y + at * o.ldy, 0, there, v);
            if (!Q && o.v) store8(o.v + (at0 + at) * cols + col, 0, there, v);
            if constexpr (Q) {
                if (!o.has_q) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = e < there ? v[e] : 0.0f;
                uint32_t scale;
                const piece8 code = quantize8(v, scale);
                store8_codes(codes + at * o.q.ld, 0, there, code);
                if (ok) scale_to(at, scale);
            }
        }
        if (turn + 2 < TURNS) {
            read(turn + 2, next[0]);
            read(turn + 3, next[1]);
        }
    }
}

// ---- any sizes, strides, scales ------------------------------------------------------------------
// Tile of 64 tokens x 64 outputs, 4 wavefronts (2 x 2), one block of 128 a step.  A step's codes and scales go from
// memory through registers, requested two steps ahead, into one of two LDS stages while the other is multiplied.  The
// rows of w are the A operand, so that a lane's four results are consecutive outputs of one token.
//   LDS row: 128 codes, the 16-byte chunk c of row r at c ^ (r & 7): neither the 8 lanes that write a row
//   nor the 8 rows that are read together meet in a bank.
// SCALED: power-of-two scales go into the instruction (8 bits) or the conversion to bf16 (32-bit results), and so does the exponent of a scale
// that is the same along a row; the rest of that is multiplied at the end.  Otherwise a block's sum is multiplied by the product of its two
// scales in 32 bits.  That is right while all scales are moderate, and a conversion to bf16 is while exponents are (scaled8); where a tile has
// met others, its results are made once more by tile_any, unless those scales are of zeros (a branch in the loop would cost every product a
// fifth).
// Bound by the vector unit (conversions to 16 bits, sums of blocks) and by the waits of four wavefronts in step: 4096 x 11008 x 4096 in
// 32 bits 490 to 514 us, 0.72 PFLOP/s, with 32-bit scales per block 560, in bf16 with those 450; 500 x 1777 x 2731 in 32 bits 20 us.  Tiles of
// 64 x 64 keep the chip full at such sizes (224 tiles); larger ones would leave most of it idle.
struct ProductScales {
    int32_t x_blocks, w_blocks;         // SCALED: exponents per block, else constant along the row
};

// Whether exponents are beyond what the conversion to bf16 holds exactly (scaled8)
__device__ __forceinline__ bool beyond_bf16(uint32_t b) { return b - 3u > 243u && b != 255u; }

// Whether a row has a block whose scale the loop does not take.  Such scales are often those of blocks of zeros, where only
// a large one does harm (a product of scales that is infinite): the codes are looked at, by a wavefront.
template <bool SCALED>
__device__ __forceinline__ bool row_beyond(const BlockView& q, int64_t row, int64_t K) {
    bool bad = false;
#pragma unroll 1
    for (int64_t at = (threadIdx.x & 63) * 16; at < K; at += 1024) {
        const uint32_t bits = scale_bits(q, row, at >> 7);
        bool small;
        if constexpr (SCALED) {
            small = beyond_bf16(bits);
        } else {
            ScaleRange r;
            r.take(scale_of(q, bits));
            bad |= r.large();
            small = r.small();
        }
        if (small) {
            const piece16 v = chunk_tail(q.codes + row * q.ld + at, (int)min(K - at, (int64_t)16), at);
            bad |= ((v[0] | v[1] | v[2] | v[3]) & 0x7F7F7F7Fu) != 0u;
        }
    }
    return __any(bad);
}

// 32 x 32 results with any scales, straight from memory: lane (lr, lg) has 32 codes of two rows of each operand and block, and the results
// of four outputs and two tokens twice.  500 x 1777 x 2731 in 32 bits with all scales of x 2^-126: 133 us, the loop and then this; with those of
// zeros 39.
template <class T, bool SCALED, class P>
__device__ __forceinline__ void tile_any(int64_t t0, int64_t T_, int64_t o0, int64_t O, int64_t K, const BlockView& x, const BlockView& w, ProductScales how,
                                         const float* __restrict__ bias, P put) {
    int lane = threadIdx.x & 63;
    floatx4 acc[2][2];
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q >> 1][q & 1] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int64_t at = 0; at < K; at += 128) {
        asm volatile("" : "+v"(lane));               // (addresses are made again for every block: few registers)
        const int lr = lane & 15, lg = lane >> 4;
        const int64_t b = at >> 7;
        const int left = (int)min(K - at, (int64_t)128) - lg * 32;
        intx8 fx[2], fw[2];
        uint32_t sx[2], sw[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t t = min(t0 + 16 * j + lr, T_ - 1), o = min(o0 + 16 * j + lr, O - 1);
            const uint8_t* px = x.codes + t * x.ld + at + lg * 32;
            const uint8_t* pw = w.codes + o * w.ld + at + lg * 32;
            fx[j] = words8(chunk_tail(px, left, at + lg * 32), chunk_tail(px + 16, left - 16, at + lg * 32 + 16));
            fw[j] = words8(chunk_tail(pw, left, at + lg * 32), chunk_tail(pw + 16, left - 16, at + lg * 32 + 16));
            sx[j] = SCALED && !how.x_blocks ? row_scale(scale_at(x, t, 0)).byte : scale_bits(x, t, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t oe = min(o0 + 16 * j + lg * 4 + e, O - 1);
                sw[j][e] = SCALED && !how.w_blocks ? row_scale(scale_at(w, oe, 0)).byte : scale_bits(w, oe, b);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const floatx4 p = block_sum<sizeof(T) == 4>(fw[i], fx[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[i][j][e] = SCALED ? acc[i][j][e] + times_exponents(p[e], sw[i][e], sx[j]) : add_scaled(p[e], scale_of(w, sw[i][e]), scale_of(x, sx[j]), acc[i][j][e]);
                __builtin_amdgcn_sched_barrier(0);
            }
    }
    const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t t = t0 + 16 * j + lr;
        if (t >= T_) break;
        const float st = SCALED && !how.x_blocks ? row_scale(scale_at(x, t, 0)).rest : 1.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t oe = o0 + 16 * i + lg * 4 + e;
                if (oe >= O) continue;
                const float so = SCALED && !how.w_blocks ? row_scale(scale_at(w, oe, 0)).rest : 1.0f;
                put(t, oe, dmmv_fma(acc[i][j][e] * so, st, bias ? bias[oe] : 0.0f));
            }
    }
}

// WAVES: wavefronts a SIMD that the registers leave room for at least.  32-bit results use more than three (32-bit scales) and four (exponents) allow:
// where a compute unit gets one tile they stay (500 x 1777 x 2731 20.6 and 19.8 us, 21.5 and 20.4 with three and four), else not (4096 x 11008 x 4096
// 570 and 500 us, 650 and 530 without).
template <class T, bool SCALED, int WAVES, bool EPI>
__global__ __launch_bounds__(256, WAVES) void k_block_product(int64_t T_, int64_t O, int64_t K, BlockView x, BlockView w, ProductScales how,
                                                       const float* __restrict__ bias, ProductOut<T, EPI> out, int32_t tiles_t, int32_t tiles_o) {
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr int MI = 2, NI = 2, BM = 32 * MI, BN = 32 * NI;
    __shared__ __align__(16) uint8_t codes[2][128 * (BM + BN)];
    __shared__ __align__(16) uint32_t scl[2][BM + BN];
    constexpr bool RANGED = !SCALED || WIDE;         // (the 8-bit instruction takes every exponent)
    __shared__ uint64_t far[2];                      // RANGED: rows whose scales are not all moderate
    __shared__ int again;                            // and some of them count
    if (RANGED && threadIdx.x == 0) again = 0;       // (a barrier follows before it is set)
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = (wv & 1) * (16 * MI), wo = (wv >> 1) * (16 * NI);
    int tile_t, tile_o;
    tile_of_workgroup(tiles_t, tiles_o, tile_t, tile_o);
    const int64_t t0 = (int64_t)tile_t * BM, o0 = (int64_t)tile_o * BN;
    const int nb = (int)((K + 127) >> 7);
    // this thread's chunks of a step: rows tid / 8 + 32 u of x, then of w; its scale: of row tid of both together
    const int crow = tid >> 3, cchunk = tid & 7;
    const uint8_t* xr[MI];
    const uint8_t* wr[NI];
#pragma unroll
    for (int u = 0; u < MI; ++u) xr[u] = x.codes + min(t0 + crow + 32 * u, T_ - 1) * x.ld + cchunk * 16;
#pragma unroll
    for (int u = 0; u < NI; ++u) wr[u] = w.codes + min(o0 + crow + 32 * u, O - 1) * w.ld + cchunk * 16;
    const int put = crow * 128 + ((cchunk ^ (crow & 7)) << 4);
    const bool mine_x = tid < BM, mine = tid < BM + BN;
    BlockView sq;                                    // (by value: a reference to one of two arguments is read from memory)
    sq.codes = mine_x ? x.codes : w.codes;
    sq.scales = mine_x ? x.scales : w.scales;
    sq.e8m0 = mine_x ? x.e8m0 : w.e8m0;
    const int64_t sblk = mine_x ? x.sblk : w.sblk;
    const int64_t sat = mine_x ? (min(t0 + tid, T_ - 1) >> x.shift) * x.srow : (min(o0 + max(tid - BM, 0), O - 1) >> w.shift) * w.srow;
    uint32_t along = 127u;                           // SCALED: the exponent of a scale that is the same along the row
    if (SCALED && !(mine_x ? how.x_blocks : how.w_blocks)) {
        if (sq.scales) along = row_scale(sq.e8m0 ? e8m0_value(static_cast<const uint8_t*>(sq.scales)[sat]) : static_cast<const float*>(sq.scales)[sat]).byte;
        sq.scales = nullptr;
        sq.e8m0 = 1;
    }

    struct Step {
        piece16 c[MI + NI];
        uint32_t s;
    };
    auto request = [&](Step& r, int kb) __attribute__((always_inline)) {      // a whole block
#pragma unroll
        for (int u = 0; u < MI; ++u) r.c[u] = *reinterpret_cast<const piece16_any*>(xr[u] + kb * 128ll);
#pragma unroll
        for (int u = 0; u < NI; ++u) r.c[MI + u] = *reinterpret_cast<const piece16_any*>(wr[u] + kb * 128ll);
        r.s = *scale_word(sq, sat + kb * sblk);
    };
    ScaleRange met;                                  // this thread's scales
    bool exact = true;                               // and exponents: those that scaled8 takes
    auto deposit = [&](const Step& r, int kb, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < MI + NI; ++u) *reinterpret_cast<piece16*>(&codes[stage][put + u * 4096]) = r.c[u];
        const uint32_t bits = word_bits(sq, sat + kb * sblk, r.s);
        const uint32_t s = SCALED ? (sq.scales ? bits : along) : sq.e8m0 ? __float_as_uint(e8m0_value(bits)) : bits;
        if (mine) scl[stage][tid] = s;
        if (!SCALED) met.take(__uint_as_float(s));
        else if (WIDE) exact &= !beyond_bf16(s);
    };
    floatx4 acc[NI][MI];
    const int c0 = (lg ^ (lr & 7)) << 4;
    auto multiply = [&](int stage) __attribute__((always_inline)) {
        const uint8_t* px = &codes[stage][(wt + lr) * 128];
        const uint8_t* pw = &codes[stage][(BM + wo + lr) * 128];
        intx8 fx[MI], fw[NI];
#pragma unroll
        for (int j = 0; j < MI; ++j)
            fx[j] = words8(*reinterpret_cast<const piece16*>(px + j * 2048 + c0), *reinterpret_cast<const piece16*>(px + j * 2048 + (c0 ^ 64)));
#pragma unroll
        for (int i = 0; i < NI; ++i)
            fw[i] = words8(*reinterpret_cast<const piece16*>(pw + i * 2048 + c0), *reinterpret_cast<const piece16*>(pw + i * 2048 + (c0 ^ 64)));
        if constexpr (SCALED) {
            uint32_t sx[MI], sw[NI];
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] = scl[stage][wt + 16 * j + lr];
#pragma unroll
            for (int i = 0; i < NI; ++i) sw[i] = scl[stage][BM + wo + 16 * i + lr];
            if constexpr (!WIDE) {
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < MI; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx[j], acc[i][j], 0, 0, 0, (int)sw[i], 0, (int)sx[j]);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    bf16x8_t bx[MI], bw[NI];
#pragma unroll
                    for (int j = 0; j < MI; ++j) bx[j] = scaled8(fx[j][2 * s], fx[j][2 * s + 1], sx[j]);
#pragma unroll
                    for (int i = 0; i < NI; ++i) bw[i] = scaled8(fw[i][2 * s], fw[i][2 * s + 1], sw[i]);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int j = 0; j < MI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[i], bx[j], acc[i][j], 0, 0, 0);
                }
            }
        } else {
            float sx[MI];
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] = __uint_as_float(scl[stage][wt + 16 * j + lr]);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const floatx4 sw = *reinterpret_cast<const floatx4*>(&scl[stage][BM + wo + 16 * i + lg * 4]);
#pragma unroll
                for (int j = 0; j < MI; ++j) {
                    const floatx4 p = block_sum<WIDE>(fw[i], fx[j]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = dmmv_fma(p[e], sw[e] * sx[j], acc[i][j][e]);
                }
            }
        }
    };
    // The whole blocks.  Requests are made without a condition, or a use would wait for all of them; those past the end ask for
    // the last block again.
    const int full = (int)(K >> 7), most = full - 1;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    Step r0, r1;
    if (full > 0) {
        request(r0, 0);
        request(r1, min(1, most));
        deposit(r0, 0, 0);
        request(r0, min(2, most));
        __syncthreads();
        for (int kb = 0; kb < full; kb += 2) {
            deposit(r1, min(kb + 1, most), 1);
            request(r1, min(kb + 3, most));
            multiply(0);
            __syncthreads();
            deposit(r0, min(kb + 2, most), 0);
            request(r0, min(kb + 4, most));
            if (kb + 1 < full) multiply(1);
            __syncthreads();
        }
    }
    if (full < nb) {                                 // the last block, zeros past the row's end
        const int64_t at = full * 128ll;
        const int left = (int)(K - at) - cchunk * 16;
#pragma unroll
        for (int u = 0; u < MI; ++u) r0.c[u] = chunk_tail(xr[u] + at, left, at + cchunk * 16);
#pragma unroll
        for (int u = 0; u < NI; ++u) r0.c[MI + u] = chunk_tail(wr[u] + at, left, at + cchunk * 16);
        r0.s = *scale_word(sq, sat + full * sblk);
        deposit(r0, full, 0);
        __syncthreads();
        multiply(0);
    }
    if constexpr (RANGED) {
        // rows of x (wavefront 0) and of w (wavefront 1) with scales that the loop does not take; do they count?
        static_assert(BM == 64 && BN == 64, "a wavefront has an operand's scales");
        const uint64_t rows = __ballot(!(SCALED ? exact : met.moderate()));
        if (wv < 2 && lane == 0) far[wv] = rows;
        __syncthreads();
        if (far[0] | far[1]) {
            bool bad = false;
#pragma unroll 1
            for (int r = wv; r < BM + BN; r += 4)
                if ((far[r >> 6] >> (r & 63)) & 1)
                    bad |= r < BM ? (!SCALED || how.x_blocks) && row_beyond<SCALED>(x, min(t0 + r, T_ - 1), K)
                                  : (!SCALED || how.w_blocks) && row_beyond<SCALED>(w, min(o0 + r - BM, O - 1), K);
            if (bad) again = 1;
            __syncthreads();
            if (again) {
                tile_any<T, SCALED>(t0 + wt, T_, o0 + wo, O, K, x, w, how, bias, [&](int64_t t, int64_t o, float v) __attribute__((always_inline)) {
                    if constexpr (EPI) finish1(out, t, o, O, v);
                    else put_y(out.y + t * out.ldy + o, v);
                });
                return;
            }
        }
    }
    constexpr int LDO = BN + 4;
    static_assert(BM * LDO * 4 <= (int)sizeof(codes), "the results take the stages' place");
    float* tile = reinterpret_cast<float*>(codes[0]);
    if constexpr (EPI) __syncthreads();              // the last block has been read
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        float bo[4], so[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t o = min(o0 + wo + 16 * i + lg * 4 + e, O - 1);
            bo[e] = bias ? bias[o] : 0.0f;
            so[e] = SCALED && !how.w_blocks ? row_scale(scale_at(w, o, 0)).rest : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < MI; ++j) {
            const int64_t t = t0 + wt + 16 * j + lr, o = o0 + wo + 16 * i + lg * 4;
            if (t >= T_) continue;
            const float st = SCALED && !how.x_blocks ? row_scale(scale_at(x, t, 0)).rest : 1.0f;
            if constexpr (EPI) {
                *reinterpret_cast<floatx4*>(tile + (wt + 16 * j + lr) * LDO + wo + 16 * i + lg * 4) =
                    floatx4{dmmv_fma(acc[i][j][0] * so[0], st, bo[0]), dmmv_fma(acc[i][j][1] * so[1], st, bo[1]), dmmv_fma(acc[i][j][2] * so[2], st, bo[2]),
                            dmmv_fma(acc[i][j][3] * so[3], st, bo[3])};
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (o + e < O) put_y(out.y + t * out.ldy + o + e, dmmv_fma(acc[i][j][e] * so[e], st, bo[e]));
            }
        }
    }
    if constexpr (EPI) {
        __syncthreads();
        finish_tile<BM, BN, LDO, false, false>(out, tile, TileScales{}, t0, T_, O, o0, [](int turn) { return 32 * turn; });
    }
}

// ---- large products ------------------------------------------------------------------------------
// The same tiles, LDS rows and operands for bf16 results with SCALED scales, where rows are aligned to 16 bytes: the
// codes go straight from memory into the LDS (NST stages of one block of 128), and the loop is written so that the matrix
// unit has a product at all times: what else there is to do is placed in the products' shadows by hand.
// Where the scales of w come from, WS: 0 a table of exponents of every row (those that are the same along a row repeated), 1 of every 128 rows,
// 2 registers, as they are the same along a row.
// T float: workgroup row y of the grid takes its share of the contraction, and y [share][T_][O] is joined by k_block_product_join.
// 256 x 256 tiles, 128 x 128 a wavefront: 64 products a step from 16 + 16 fragments, which the LDS can deliver beside the requests;
// smaller tiles are bound by it.  4096 x 11008 x 4096: 158 to 167 us (2.2 to 2.35 PFLOP/s), the matrix unit busy for 53 % of the
// cycles; 688 tiles are 2.7 rounds of the chip (256 tiles of K = 11008: 131 us, 2.8 PFLOP/s), the clock falls under this load.
// exponents of `blocks` blocks from kb on for `rows` rows (or groups of `per` rows) of a tile, to bytes of the LDS
__device__ __forceinline__ void stage_exponents(const BlockView& q, int64_t row0, int64_t last, int per, int rows, int kb, int blocks,
                                                uint8_t* to, int stride) {
    for (int r = threadIdx.x; r < rows; r += 256) {
        const int64_t row = min(row0 + (int64_t)r * per, last - 1);
        const uint8_t* p = static_cast<const uint8_t*>(q.scales) + (row >> q.shift) * q.srow + kb * q.sblk;
        int b = 0;
        if (q.sblk == 1)
#pragma unroll 1
            for (; b + 16 <= blocks; b += 16) {
                const piece16 v = *reinterpret_cast<const piece16_any*>(p + b);
#pragma unroll
                for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(to + r * stride + b + 4 * e) = v[e];
            }
#pragma unroll 4
        for (; b < blocks; ++b) to[r * stride + b] = p[b * q.sblk];
    }
}

constexpr int product_lds(int MI, int NI, int width, int ws, int nst, bool epi) {
    const int stages = nst * 128 * 32 * (MI + NI) + 68 * (32 * MI + (ws == 2 ? 0 : ws == 1 ? (32 * NI + 127) / 128 : 32 * NI));
    const int out = epi ? 2 * 64 * (32 * NI * 4 + 16) + 4 * (64 * NI + 32 * MI) : 32 * MI * (32 * NI * width + 16);
    return stages > out ? stages : out;
}

template <class T, int MI, int NI, int WS, int NST, bool EPI>
__global__ __launch_bounds__(256) void k_block_product_tiled(int64_t T_, int64_t O, int64_t K, BlockView x, BlockView w, ProductScales how,
                                                             const float* __restrict__ bias, ProductOut<T, EPI> out,
                                                             int32_t tiles_t, int32_t tiles_o) {
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int BM = 32 * MI, BN = 32 * NI, STAGE = 128 * (BM + BN);
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = (wv & 1) * (16 * MI), wo = (wv >> 1) * (16 * NI);
    int tile_t, tile_o;
    tile_of_workgroup(tiles_t, tiles_o, tile_t, tile_o);
    const int64_t t0 = (int64_t)tile_t * BM, o0 = (int64_t)tile_o * BN;
    if constexpr (sizeof(T) == 4) {                  // everything of this share but the place of its results begins at block `from`
        const int64_t share = ((K + 127) / 128 + gridDim.y - 1) / gridDim.y, from = share * blockIdx.y;
        x.codes += from * 128;
        w.codes += from * 128;
        if (how.x_blocks) x.scales = static_cast<uint8_t*>(x.scales) + from * x.sblk;
        if (how.w_blocks) w.scales = static_cast<uint8_t*>(w.scales) + from * w.sblk;
        K = min(K - from * 128, share * 128);
        out.y += (int64_t)blockIdx.y * T_ * O;
    }
    const int nb = (int)((K + 127) >> 7);

    // One request brings 8 rows of a step (1 KB) from memory to the LDS, 16 bytes a lane in the order of the lanes:
    // lane l has row l / 8 and the chunk that belongs at place l % 8 of it.  A wavefront brings 8 MI rows of x and
    // 8 NI of w.
    const uint8_t* xb = x.codes + t0 * x.ld;
    const uint8_t* wb = w.codes + o0 * w.ld;
    const uint32_t ldx = (uint32_t)x.ld, ldw = (uint32_t)w.ld;                    // below 2^23
    const uint32_t lastx = (uint32_t)min((int64_t)BM - 1, T_ - 1 - t0), lastw = (uint32_t)min((int64_t)BN - 1, O - 1 - o0);
    const intx4 bufx = buffer_of(xb, lastx * ldx + (uint32_t)K), bufw = buffer_of(wb, lastw * ldw + (uint32_t)K);
    const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;
    const uint32_t offx = crow * ldx + cchunk * 16, offw = crow * ldw + cchunk * 16;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

    floatx4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    // Exponents of SB blocks of every row of the tile, one byte each (WS 1: of every 128 rows of w), past the stages; a
    // lane has those of two steps in a register.
    constexpr int SB = 64, SROW = SB + 4, WROWS = WS == 2 ? 0 : WS == 1 ? (BN + 127) / 128 : BN, NS = WS == 1 ? 1 : NI;
    uint8_t* scl = lds + NST * STAGE;
    uint32_t sx[MI], sw[NS];
    // Exponents of scales that are the same along a row, for all blocks: a row of the table a thread; requested ahead of the codes
    static_assert(WS == 0 ? BM + BN <= 256 : BM <= 256, "a thread has one row");
    const bool mine_x = tid < BM, fills = mine_x ? !how.x_blocks : WS == 0 && !how.w_blocks;
    float along = 1.0f, along_w[WS == 2 ? NS : 1];
    if (fills) along = mine_x ? scale_at(x, min(t0 + tid, T_ - 1), 0) : scale_at(w, min(o0 + tid - BM, O - 1), 0);
    if constexpr (WS == 2)
#pragma unroll
        for (int i = 0; i < NS; ++i) along_w[i] = scale_at(w, min(o0 + wo + 16 * i + lr, O - 1), 0);
    auto scales_along = [&]() __attribute__((always_inline)) {
        if (fills) {
            const uint32_t b = row_scale(along).byte * 0x01010101u;
#pragma unroll
            for (int i = 0; i < SROW / 4; ++i) reinterpret_cast<uint32_t*>(scl + tid * SROW)[i] = b;
        }
        if constexpr (WS == 2)
#pragma unroll
            for (int i = 0; i < NS; ++i) sw[i] = row_scale(along_w[i]).byte * 0x0101u;
    };
#define BP_SCALES_STAGE(kb)                                                                                     \
    {                                                                                                           \
        if (how.x_blocks) stage_exponents(x, t0, T_, 1, BM, kb, min(nb - (kb), SB), scl, SROW);                 \
        if (WS < 2 && how.w_blocks) stage_exponents(w, o0, O, WS == 1 ? 128 : 1, WROWS, kb, min(nb - (kb), SB), scl + BM * SROW, SROW); \
    }
#define BP_SCALES_TAKE(kb)                                                                                      \
    {                                                                                                           \
        const uint8_t* p_ = scl + ((kb) & (SB - 1));                                                            \
        _Pragma("unroll") for (int j = 0; j < MI; ++j)                                                          \
            sx[j] = *reinterpret_cast<const uint16_t*>(p_ + (wt + 16 * j + lr) * SROW);                         \
        if (WS < 2)                                                                                             \
            _Pragma("unroll") for (int i = 0; i < NS; ++i)                                                      \
                sw[i] = *reinterpret_cast<const uint16_t*>(p_ + (BM + (WS == 1 ? wo >> 7 : wo + 16 * i + lr)) * SROW); \
    }

    // Request i (of MI / 2) of this wavefront for half `h` of the wavefronts' rows of x (W 0) or w (W 1): 8 rows
    static_assert(MI == NI && MI % 4 == 0, "quadrants of the wavefront's tile");
    auto bring = [&](int kb, int stage, auto W, auto h, int i) __attribute__((always_inline)) {
        const int row = (wv >> 1) * (16 * MI) + h.value * (8 * MI) + ((wv & 1) * (MI / 2) + i) * 8;
        lds_request(W.value ? bufw : bufx, W.value ? offw : offx, (uint32_t)kb * 128u + (uint32_t)row * (W.value ? ldw : ldx),
                    lds0 + stage + (W.value ? BM * 128 : 0) + row * 128);
    };

    piece16 fx[MI][2], fw[NI][2];                    // a fragment's 32 codes, in two halves
    const int c0 = (lg ^ (lr & 7)) << 4;
    const uint8_t* px[2] = {lds + (wt + lr) * 128 + c0, lds + (wt + lr) * 128 + (c0 ^ 64)};
    const uint8_t* pw[2] = {lds + BM * 128 + (wo + lr) * 128 + c0, lds + BM * 128 + (wo + lr) * 128 + (c0 ^ 64)};
    auto mul = [&](auto byte, int i, int j) __attribute__((always_inline)) {
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(words8(fw[i][0], fw[i][1]), words8(fx[j][0], fx[j][1]), acc[i][j], 0, 0,
                                                                     byte.value, (int)sw[WS == 1 ? 0 : i], byte.value, (int)sx[j]);
    };
    auto frag_x = [&](int stage, int j, int h) __attribute__((always_inline)) {
        fx[j][h] = *reinterpret_cast<const piece16*>(px[h] + stage + j * 2048);
    };
    auto frag_w = [&](int stage, int i, int h) __attribute__((always_inline)) {
        fw[i][h] = *reinterpret_cast<const piece16*>(pw[h] + stage + i * 2048);
    };
    // blocks in pairs (the loop's body is one piece of straight code, or the compiler takes the products out of it)
    const int paired = (int)(K >> 8) * 2, last = paired - 1;
    // One quadrant of the wavefront's tile (halves ih of w, jh of x) with step parity P.  Between the products, a few
    // instructions in the shadow of each and in this order: the fragments of half `fh` of x (FX) or w for the next
    // quadrant, from the stage at fs, and the requests for half rh of w (RW) or x of block kb into the stage at rs.
    auto quad = [&](auto P, auto ih, auto jh, auto FX, int fs, auto fh, auto RW, auto rh, int kb, int rs) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < MI / 2; ++g) {
#pragma unroll
            for (int i = 0; i < NI / 2; ++i) {
                mul(P, ih.value * (NI / 2) + i, jh.value * (MI / 2) + g);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k * (NI / 2) / 4 != i) continue;
                    if (k < 2) {
                        if (FX.value) frag_x(fs, fh.value * (MI / 2) + g, k);
                        else frag_w(fs, fh.value * (NI / 2) + g, k);
                    } else if (k == 2) {
                        bring(kb, rs, RW, rh, g);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // A step: four quadrants, each with one new half of fragments and a quarter of a block's requests (all of them at once
    // would keep the address unit, and with it the wavefront, for half of the step).  X0: the half of x that is there at the
    // start; the other half comes first, and at the end next step's w half 0 and x half 1 - X0 are there.
    // Block j's first requests are for what is read first, w half 0 and x half j & 1: made in the second half of step j - NST, when its
    // stage has been read, and whole at the middle of step j - 1; the others a half step later.  So there is a barrier
    // in the middle and at the end of a step, and at either the wavefront's last LEFT requests may still be on their way.
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    constexpr int LEFT = (2 * NST - 3) * MI;
    auto step = [&](auto P, auto N, int cur, int nxt, int prv, int to) __attribute__((always_inline)) {        // P: parity of the step and X0, N = 1 - P
        quad(P, C0, P, C1, cur, N, C0, P, min(to - 1, last), prv);
        quad(P, C0, N, C0, cur, C1, C1, C1, min(to - 1, last), prv);
        lds_requests_left<LEFT>();
        __syncthreads();
        quad(P, C1, N, C0, nxt, C0, C1, C0, min(to, last), cur);
        quad(P, C1, P, C1, nxt, N, C0, P, min(to, last), cur);
        lds_requests_left<LEFT>();
        __syncthreads();
    };

    if (paired > 0) {
#pragma unroll
        for (int st = 0; st < NST; ++st) {           // all of NST - 1 blocks, the first half of one
            const int kb = min(st, last);
            auto half = [&](auto wh, auto xh) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < MI / 2; ++i) bring(kb, st * STAGE, C1, wh, i);
#pragma unroll
                for (int i = 0; i < MI / 2; ++i) bring(kb, st * STAGE, C0, xh, i);
            };
            if (st & 1) half(C0, C1);
            else half(C0, C0);
            if (st < NST - 1) {
                if (st & 1) half(C1, C0);
                else half(C1, C1);
            }
        }
        scales_along();
        BP_SCALES_STAGE(0);
        lds_requests_left<LEFT>();
        __syncthreads();
#pragma unroll
        for (int g = 0; g < MI / 2; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                frag_w(0, g, h);
                frag_x(0, g, h);
            }
        for (int kb = 0;;) {
            const int end = min(kb + SB, paired);
            for (; kb < end; kb += 2) {
                BP_SCALES_TAKE(kb);
                const int at = NST == 2 ? 0 : (kb & (NST - 1)) * STAGE, after = NST == 2 ? 0 : ((kb + 2) & (NST - 1)) * STAGE;
                const int before = NST == 2 ? STAGE : ((kb - 1) & (NST - 1)) * STAGE;
                step(C0, C1, at, at + STAGE, before, kb + NST);
                step(C1, C0, at + STAGE, after, at, kb + NST + 1);
            }
            if (kb >= paired) break;
            __syncthreads();
            BP_SCALES_STAGE(kb);
            __syncthreads();
        }
        lds_requests_left<0>();
    }
    // one whole block at most, and a last shorter one: zeros past the row's end
#pragma unroll 1
    for (int kb = paired; kb < nb; ++kb) {
        const int left = (int)(K - kb * 128ll) - cchunk * 16;
        __syncthreads();
        if (paired == 0 && kb == 0) scales_along();
        if (kb == paired && (kb & (SB - 1)) == 0) BP_SCALES_STAGE(kb);
#pragma unroll 1
        for (int q = 0; q < MI; ++q) {
            const uint32_t row = 8 * (wv * MI + q) + crow;
            uint8_t* to = lds + (wv * MI + q) * 1024 + lane * 16;
            *reinterpret_cast<piece16*>(to) = chunk_tail(xb + kb * 128ll + min(row, lastx) * ldx + cchunk * 16, left, kb * 128ll + cchunk * 16);
            *reinterpret_cast<piece16*>(to + BM * 128) = chunk_tail(wb + kb * 128ll + min(row, lastw) * ldw + cchunk * 16, left, kb * 128ll + cchunk * 16);
        }
        __syncthreads();
        BP_SCALES_TAKE(kb & ~1);
        if (kb & 1) {
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] >>= 8;
#pragma unroll
            for (int i = 0; WS < 2 && i < NS; ++i) sw[i] >>= 8;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                frag_w(0, i, h);
                frag_x(0, i, h);
            }
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < MI; ++j) mul(C0, i, j);
    }
    __syncthreads();
    if constexpr (EPI) {
        // 64 rows at a time through the LDS in 32 bits, two places in turn: 32 of each half of the tile's rows
        constexpr int LDF = BN + 4;
        float* const first = reinterpret_cast<float*>(lds);
        const TileScales k = {first + 2 * 64 * LDF, WS == 1 ? nullptr : first + 2 * 64 * LDF + BN, first + 2 * 64 * LDF + 2 * BN};
        if (tid < BN) {
            const int64_t o = min(o0 + tid, O - 1);
            k.bias[tid] = bias ? bias[o] : 0.0f;
            if constexpr (WS != 1) k.so[tid] = !how.w_blocks ? row_scale(scale_at(w, o, 0)).rest : 1.0f;
        }
        if (tid < BM) k.st[tid] = !how.x_blocks ? row_scale(scale_at(x, min(t0 + tid, T_ - 1), 0)).rest : 1.0f;
        auto pass = [&](auto P) __attribute__((always_inline)) {
            constexpr int p = P.value;
            float* tile = first + (p & 1) * 64 * LDF;
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    *reinterpret_cast<floatx4*>(tile + ((wv & 1) * 32 + 16 * j + lr) * LDF + wo + 16 * i + lg * 4) = acc[i][2 * p + j];
            __syncthreads();
            finish_tile<64, BN, LDF, true, true>(out, tile, k, t0, T_, O, o0, [](int turn) {
                constexpr int STEP = 2048 / BN;              // rows a turn
                return turn * STEP / 32 * (BM / 2 - 32) + turn * STEP + 32 * p;
            });
        };
        pass(C0);
        pass(C1);
        if constexpr (MI == 8) {
            pass(std::integral_constant<int, 2>{});
            pass(std::integral_constant<int, 3>{});
        }
        return;
    }
    // results through the LDS: rows of the tile, stored 16 bytes a lane
    constexpr int LDO = BN * (int)sizeof(T) + 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        float bo[4], so[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t o = min(o0 + wo + 16 * i + lg * 4 + e, O - 1);
            bo[e] = bias ? bias[o] : 0.0f;
            so[e] = !how.w_blocks ? row_scale(scale_at(w, o, 0)).rest : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < MI; ++j) {
            const float st = !how.x_blocks ? row_scale(scale_at(x, min(t0 + wt + 16 * j + lr, T_ - 1), 0)).rest : 1.0f;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = dmmv_fma(acc[i][j][e] * so[e], st, bo[e]);
            put4(reinterpret_cast<T*>(lds + (wt + 16 * j + lr) * LDO) + wo + 16 * i + lg * 4, v);
        }
    }
    __syncthreads();
    constexpr int PER = 16 / (int)sizeof(T), CPR = BN / PER;
    for (int c = tid; c < BM * CPR; c += 256) {
        const int r = c / CPR, h = c % CPR;
        const int64_t t = t0 + r, o = o0 + h * PER;
        if (t >= T_ || o >= O) continue;
        const piece16 v = *reinterpret_cast<const piece16*>(lds + r * LDO + h * 16);
        T* dst = out.y + t * out.ldy + o;
        if (o + PER <= O) {
            *reinterpret_cast<piece16_any*>(dst) = v;
        } else {
            const T* one = reinterpret_cast<const T*>(lds + r * LDO + h * 16);
            for (int e = 0; e < PER && o + e < O; ++e) dst[e] = one[e];
        }
    }
}


// ---- few tokens ------------------------------------------------------------------------------------
// Up to 64 tokens: the weights are read once, straight into registers in the order of the operands (a lane 32 codes of
// a row and block, 128 bytes of a row side by side), and nothing else counts.  A workgroup has 16 outputs and
// 16 MT tokens, its four wavefronts a share of the blocks each, joined in order through the LDS.  RING: U blocks are on their way at any time; else
// U of them are requested together and waited for together (few_in_ring).  One token of 4096 by 11008
// outputs: 10.6 us, 4.3 TB/s, 14.0 in 8 bits with a pass for those; 24 tokens of 4096 by 4096: 9.6 us, two thirds of it start,
// join and end (eight wavefronts a workgroup were no faster); 24 of 11008 by 4096 17.6: the tokens, read for every 16 outputs, from the L2.
constexpr int few_ring(int MT) { return MT == 1 ? 6 : MT == 2 ? 5 : 2; }
template <class T, int MT, bool SCALED, bool WIDE, bool RING, bool EPI>
__global__ __launch_bounds__(256) void k_block_product_few(int32_t T_, int64_t O, int64_t K, BlockView x, BlockView w, ProductScales how,
                                                                  const float* __restrict__ bias, ProductOut<T, EPI> out) {
    // (BRIEF: a bf16 result that is summed in 32 bits, exponents)
    constexpr bool BRIEF = SCALED && WIDE && sizeof(T) == 2;
    static_assert(!RING || SCALED, "exponents");
    constexpr int U = RING ? few_ring(MT) : MT >= 4 ? 2 : 4, WAVES = 4;
    __shared__ floatx4 part[WAVES][MT][64];
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t o0 = blockIdx.x * 16ll, t0 = blockIdx.y * (16ll * MT);
    const int nb = (int)((K + 127) >> 7), full = (int)(K >> 7);
    const int b0 = (int)((int64_t)nb * wv / WAVES), b1 = (int)((int64_t)nb * (wv + 1) / WAVES);
    const int64_t orow = min(o0 + lr, O - 1);
    const uint8_t* wr = w.codes + orow * w.ld + lg * 32;
    const uint8_t* xr[MT];
    int64_t trow[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        trow[m] = min(t0 + 16 * m + lr, (int64_t)T_ - 1);
        xr[m] = x.codes + trow[m] * x.ld + lg * 32;
    }
    floatx4 acc[MT];

    // one block's codes and scales in registers
    struct Block {
        piece16 w[2], x[MT][2];
        uint32_t ew, ex[MT];           // SCALED: exponents
        uint32_t fw[4], fx[MT];        // else: scales of this lane's four outputs, of its tokens, as they are stored
    };
    auto exponent = [&](const BlockView& q, int64_t row, int b) __attribute__((always_inline)) {
        return (uint32_t)static_cast<const uint8_t*>(q.scales)[(row >> q.shift) * q.srow + b * q.sblk];
    };
    // SCALED: scales that are the same along a row, and their exponents, taken when the first codes have been requested.  RING: a byte is loaded for every
    // block all the same (of the codes, the same one): a branch around a load makes the compiler wait for all of them.
    float row_w = 1.0f, row_x[MT];
    uint32_t along_w = 127u, along_x[MT];
    if (SCALED && !how.w_blocks) row_w = scale_at(w, orow, 0);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        row_x[m] = SCALED && !how.x_blocks ? scale_at(x, trow[m], 0) : 1.0f;
        along_x[m] = 127u;
    }
    auto exponents_along = [&]() __attribute__((always_inline)) {
        along_w = row_scale(row_w).byte;
#pragma unroll
        for (int m = 0; m < MT; ++m) along_x[m] = row_scale(row_x[m]).byte;
    };
    const uint8_t* pw = how.w_blocks ? static_cast<const uint8_t*>(w.scales) + (orow >> w.shift) * w.srow : w.codes;
    const uint8_t* px[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) px[m] = how.x_blocks ? static_cast<const uint8_t*>(x.scales) + (trow[m] >> x.shift) * x.srow : x.codes;
    const int64_t step_w = how.w_blocks ? w.sblk : 0, step_x = how.x_blocks ? x.sblk : 0;
    auto scales = [&](Block& k, int b) __attribute__((always_inline)) {
        if constexpr (RING) {
            k.ew = pw[b * step_w];
#pragma unroll
            for (int m = 0; m < MT; ++m) k.ex[m] = px[m][b * step_x];
        } else if constexpr (SCALED) {
            if (how.w_blocks) k.ew = exponent(w, orow, b);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if (how.x_blocks) k.ex[m] = exponent(x, trow[m], b);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) k.fw[e] = scale_bits(w, min(o0 + lg * 4 + e, O - 1), b);
#pragma unroll
            for (int m = 0; m < MT; ++m) k.fx[m] = scale_bits(x, trow[m], b);
        }
    };
    auto request = [&](Block& k, int b) __attribute__((always_inline)) {      // a whole block
#pragma unroll
        for (int h = 0; h < 2; ++h) k.w[h] = *reinterpret_cast<const piece16_any*>(wr + (int64_t)b * 128 + 16 * h);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) k.x[m][h] = *reinterpret_cast<const piece16_any*>(xr[m] + (int64_t)b * 128 + 16 * h);
        scales(k, b);
    };
    // BRIEF: both operands become bf16 with their scales in them, as in the general kernel, and a wavefront that has met exponents which that does
    // not hold exactly makes its sums again
    ScaleRange met;                                  // as in the general kernel: this lane's scales (24 x 4096 x 4096: 11.5 us, 25 with a scale of 2^-126)
    bool exact = true;
    auto multiply = [&](auto CAREFUL, Block& k) __attribute__((always_inline)) {
        if constexpr (SCALED) {
            if (!how.w_blocks) k.ew = along_w;
            if (!how.x_blocks)
#pragma unroll
                for (int m = 0; m < MT; ++m) k.ex[m] = along_x[m];
        }
        if constexpr (!SCALED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) met.take(scale_of(w, k.fw[e]));
#pragma unroll
            for (int m = 0; m < MT; ++m) met.take(scale_of(x, k.fx[m]));
        }
        const intx8 a = words8(k.w[0], k.w[1]);
        if constexpr (BRIEF && !CAREFUL.value) {
            exact &= !beyond_bf16(k.ew);
#pragma unroll
            for (int m = 0; m < MT; ++m) exact &= !beyond_bf16(k.ex[m]);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const bf16x8_t aw = scaled8(a[2 * s], a[2 * s + 1], k.ew);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const intx8 b = words8(k.x[m][0], k.x[m][1]);
                    acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw, scaled8(b[2 * s], b[2 * s + 1], k.ex[m]), acc[m], 0, 0, 0);
                }
            }
            return;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const intx8 b = words8(k.x[m][0], k.x[m][1]);
            if constexpr (SCALED && !WIDE) {
                acc[m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[m], 0, 0, 0, (int)k.ew, 0, (int)k.ex[m]);
            } else {
                const floatx4 p = block_sum<WIDE>(a, b);
                if constexpr (SCALED) {
                    // 32-bit results, exponents: a row of w belongs to lane lr, its results to lanes of another order
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][e] += times_exponents(p[e], (uint32_t)__shfl((int)k.ew, lg * 4 + e, 64), k.ex[m]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float sw = scale_of(w, k.fw[e]), sx = scale_of(x, k.fx[m]);
                        acc[m][e] = CAREFUL.value ? add_scaled(p[e], sw, sx, acc[m][e]) : dmmv_fma(p[e], sw * sx, acc[m][e]);
                    }
                }
            }
        }
    };
    auto one = [&](auto CAREFUL, int b) __attribute__((always_inline)) {
        Block k;
        const int left = (int)min(K - b * 128ll, (int64_t)128) - lg * 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) k.w[h] = chunk_tail(wr + (int64_t)b * 128 + 16 * h, left - 16 * h, b * 128ll + lg * 32 + 16 * h);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) k.x[m][h] = chunk_tail(xr[m] + (int64_t)b * 128 + 16 * h, left - 16 * h, b * 128ll + lg * 32 + 16 * h);
        scales(k, b);
        if (SCALED && !RING && b == b0) exponents_along();
        multiply(CAREFUL, k);
    };
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    int b = b0;
    if constexpr (RING) {
        // Whole blocks, U at least (few_in_ring): U of them are requested before the first is multiplied, and each one's place is taken by the block
        // U further on.
        const int end = min(b1, full);
        Block k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) request(k[u], b + u);
        exponents_along();
        for (; b + 2 * U <= end; b += U)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                multiply(std::false_type{}, k[u]);
                request(k[u], b + u + U);
                __builtin_amdgcn_sched_barrier(0);
            }
        // the last U to 2 U - 1
#pragma unroll
        for (int u = 0; u < U; ++u) {
            multiply(std::false_type{}, k[u]);
            if (b + u + U < end) request(k[u], b + u + U);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < U - 1; ++u) {
            if (b + u + U < end) multiply(std::false_type{}, k[u]);
            __builtin_amdgcn_sched_barrier(0);
        }
        b = end;
    } else {
        for (; b + U <= b1 && b + U <= full; b += U) {
            Block k[U];
#pragma unroll
            for (int u = 0; u < U; ++u) request(k[u], b + u);
            if (SCALED && b == b0) exponents_along();
#pragma unroll
            for (int u = 0; u < U; ++u) multiply(std::false_type{}, k[u]);
        }
    }
#pragma unroll 1
    for (; b < b1; ++b) one(std::false_type{}, b);
    if constexpr (!SCALED || BRIEF)
        if (!__all(BRIEF ? exact : met.moderate())) {
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (b = b0; b < b1; ++b) one(std::true_type{}, b);
        }
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wv][m][lane] = acc[m];
    __syncthreads();
    // wavefront m joins and stores tile m
    for (int m = wv; m < MT; m += WAVES) {
        floatx4 v = part[0][m][lane];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v += part[i][m][lane];
        const int64_t t = t0 + 16 * m + lr;
        if (t >= T_) continue;
        const float st = SCALED && !how.x_blocks ? row_scale(scale_at(x, t, 0)).rest : 1.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t o = o0 + lg * 4 + e;
            if (o >= O) continue;
            const float so = SCALED && !how.w_blocks ? row_scale(scale_at(w, o, 0)).rest : 1.0f;
            const float u = dmmv_fma(v[e] * so, st, bias ? bias[o] : 0.0f);
            if constexpr (EPI) finish1(out, t, o, O, u);
            else put_y(out.y + t * out.ldy + o, u);
        }
    }
}

// Whether blocks go in a ring: every wavefront has U whole ones at least, and where there are two tiles of tokens the registers of a ring (two workgroups a
// compute unit, three without) leave no workgroup waiting.  In bf16, us with and without it: one token of 11008 to 4096 outputs 10.0 and 12.6, of 4096 to 4096 5.7
// and 6.1, 17 of 11008 to 4096 15.0 and 17.1; with fewer blocks its first requests are for nothing, 32 of 512 to 4096 6.6 and 4.0, one of 1000 to 1000 4.6
// and 3.7; 17 of 3500 to 11008, a scale per row, 16.7 and 15.5.  33 to 64 tokens, U = 2 either way: sums by 8-bit
// instructions are faster without it (33 of 3500 to 11008 21.3 and 20.1), 8 bits of sums by 16-bit ones with it (33 of 2560 to 4096 11.5 and 12.2).
// 32-bit results have none built.
static bool few_in_ring(const dmmv_block_matrix* w, int MT) {
    const int64_t nb = ceil_div(w->cols, 128), full = w->cols / 128, U = few_ring(MT);
    return nb / 4 >= U && full - 3 * nb / 4 >= U && (MT != 2 || w->rows <= 8192);
}

template <class T, int MT, bool WIDE, bool EPI>
static dmmv_status launch_few_of(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const ProductScales& how, bool scaled, const float* bias,
                                 const ProductOut<T, EPI>& out, hipStream_t s) {
    const dim3 grid((unsigned)ceil_div(w->rows, 16), (unsigned)ceil_div(x->rows, 16 * MT));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, (int32_t)x->rows, w->rows, x->cols, layer_view(x), layer_view(w), how, bias, out);
    };
    constexpr bool rings = sizeof(T) == 2 && (MT <= 2 || WIDE);
    if (!scaled) launch(k_block_product_few<T, MT, false, WIDE, false, EPI>);
    else if (rings && few_in_ring(w, MT)) launch(k_block_product_few<T, MT, true, WIDE, rings, EPI>);
    else launch(k_block_product_few<T, MT, true, WIDE, false, EPI>);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T, bool WIDE, bool EPI>
static dmmv_status launch_few(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const ProductScales& how, bool scaled, const float* bias,
                              const ProductOut<T, EPI>& out, hipStream_t s) {
    if (x->rows <= 16) return launch_few_of<T, 1, WIDE, EPI>(x, w, how, scaled, bias, out, s);
    if (x->rows <= 32) return launch_few_of<T, 2, WIDE, EPI>(x, w, how, scaled, bias, out, s);
    return launch_few_of<T, 4, WIDE, EPI>(x, w, how, scaled, bias, out, s);
}

// scales that are the same along a row leave the sum
static bool constant_rows(const dmmv_block_matrix* q) { return !q->scales || q->scale_block_stride == 0 || q->cols <= 128; }

// rows that requests of 16 bytes can bring to the LDS, with offsets of 24 x 24 bits
static bool aligned(const dmmv_block_matrix* q) { return q->ld < 1 << 23 && q->ld % 16 == 0 && (uintptr_t)q->codes % 16 == 0; }

// y = bias and the sum of the shares, by ascending share; 8 outputs a lane
template <bool EPI>
__global__ __launch_bounds__(256) void k_block_product_join(int64_t T_, int64_t O, int32_t shares, const float* __restrict__ part,
                                                            const float* __restrict__ bias, ProductOut<bf16_t, EPI> out) {
    const int64_t t = blockIdx.x * 4ll + (threadIdx.x >> 6), o = (blockIdx.y * 64ll + (threadIdx.x & 63)) * 8;
    if (t >= T_ || (!EPI && o >= O)) return;         // (whole wavefronts; the lanes of a block of 128 stay together)
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, p[8];
#pragma unroll 4
    for (int i = 0; i < shares; ++i) {
        load8(part + (i * T_ + t) * O, o, O, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += p[e];
    }
    if (bias) {
        load8(bias, o, O, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += p[e];
    }
    if constexpr (EPI) {
        if (out.residual) load8(out.residual + t * out.ldr, o, O, p);
        finish8(out, t, o, O, v, p);
    } else {
        store8(out.y + t * out.ldy, o, O, v);
    }
}

template <class T, int MI, int NI, int WS, int NST, bool EPI>
static dmmv_status launch_tiled(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, const ProductOut<T, EPI>& out, hipStream_t s,
                                int32_t shares = 1) {
    const int64_t tiles_t = ceil_div(x->rows, 32 * MI), tiles_o = ceil_div(w->rows, 32 * NI);
    if (tiles_t > INT32_MAX / 4 / tiles_o) return fail(DMMV_ERR_SHAPE, "y: more tiles than a launch takes");
    const void* kern = (const void*)k_block_product_tiled<T, MI, NI, WS, NST, EPI>;
    constexpr int bytes = product_lds(MI, NI, sizeof(T), WS, NST, EPI);
    DMMV_TRY(ensure_dynamic_lds(kern, bytes));
    const ProductScales how = {!constant_rows(x), !constant_rows(w)};
    hipLaunchKernelGGL((k_block_product_tiled<T, MI, NI, WS, NST, EPI>), dim3((unsigned)(tiles_t * tiles_o), (unsigned)shares), dim3(256), bytes, s, x->rows,
                       w->rows, x->cols, layer_view(x), layer_view(w), how, bias, out, (int32_t)tiles_t, (int32_t)tiles_o);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

// Shares of the contraction where tiles of 128 x 128 are fewer than the compute units, by the time that a step of
// a tile takes (0.4 us), the second launch and the parts, written and read once.  33 x 4096 x 11008: 21 us with eight shares, 34 with
// one (the weights alone are 9 us); 33 x 1024 x 4096 12.3 and 15.8, 128 x 4096 x 11008 25 and 36.
static int32_t product_shares(int64_t T, int64_t O, int64_t K) {
    const int64_t tiles = ceil_div(T, 128) * ceil_div(O, 128), nb = ceil_div(K, 128);
    if (tiles <= 0 || tiles > 128) return 1;
    int32_t best = 1;
    double least = 0.4 * nb;
    for (int64_t n = 2; n * tiles <= 256 && 2 * n <= nb; ++n) {
        const double us = 0.4 * ceil_div(nb, n) + 5.0 + 8.0 * n * T * O / 4e6;
        if (us < least && (n - 1) * ceil_div(nb, n) < nb) least = us, best = (int32_t)n;         // (every share has a block)
    }
    return best;
}
static size_t product_part_bytes(int64_t T, int64_t O, int64_t K) {
    const int32_t n = product_shares(T, O, K);
    return n > 1 ? (size_t)n * T * O * 4 : 0;
}

// bf16 results by the large tiles: 256 x 256, or 128 x 128 with more stages; part: room for the shares, or NULL
template <bool EPI>
static dmmv_status product_tiled(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, const ProductOut<bf16_t, EPI>& out, float* part,
                                 hipStream_t s) {
    const int32_t shares = part ? product_shares(x->rows, w->rows, x->cols) : 1;
    if (shares > 1) {
        DMMV_TRY((launch_tiled<float, 4, 4, 0, 4, false>(x, w, nullptr, {part, w->rows}, s, shares)));
        hipLaunchKernelGGL((k_block_product_join<EPI>), dim3((unsigned)ceil_div(x->rows, 4), (unsigned)ceil_div(w->rows, 512)), dim3(256), 0, s, x->rows,
                           w->rows, shares, part, bias, out);
        DMMV_LAUNCH_CHECK();
        return DMMV_OK;
    }
    const bool along = constant_rows(w);
    int dev = 0, cus = 0;
    DMMV_HIP_CHECK(hipGetDevice(&dev));
    DMMV_HIP_CHECK(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev));
    const int64_t small = ceil_div(x->rows, 128) * ceil_div(w->rows, 128), large = ceil_div(x->rows, 256) * ceil_div(w->rows, 256);
    // a round of large tiles takes 2.25 times one of small ones (K = 4096: 46 us and 20.5; 1024 x 4096 x 11008 54 and 62 us,
    // 2048 x 4096 x 4096 51 and 44)
    if ((along || w->scale_rows == 128) && 9 * ceil_div(large, cus) < 4 * ceil_div(small, cus))
        return along ? launch_tiled<bf16_t, 8, 8, 2, 2, EPI>(x, w, bias, out, s) : launch_tiled<bf16_t, 8, 8, 1, 2, EPI>(x, w, bias, out, s);
    return launch_tiled<bf16_t, 4, 4, 0, 4, EPI>(x, w, bias, out, s);
}

// Rows that are no multiple of 16 codes are laid out for the large tiles where the general kernel would
// take over some 30 us: 4096 outputs of 4095 for 11008 tokens 225 us against 660, and the other way about 500 x 1777 x 2731 two launches
// more for 20 us.  Bytes, 0 = not.
static size_t product_lay_bytes(int64_t T, int64_t O, int64_t K) {
    if (K % 16 == 0 || T <= 64 || ceil_div(K, 128) * 128 >= 1 << 23 || 2.0 * (double)T * (double)O * (double)K < 12e9) return 0;
    return (size_t)(T + O) * (size_t)(ceil_div(K, 128) * 128);
}
static bool product_shared(int64_t T, int64_t K, size_t lay) { return lay > 0 || (K % 16 == 0 && T > 32); }
static size_t product_workspace(int64_t T, int64_t O, int64_t K) {
    const size_t lay = (product_lay_bytes(T, O, K) + 255) / 256 * 256;
    return lay + (product_shared(T, K, lay) ? product_part_bytes(T, O, K) : 0);
}

// How a product is made, and the bytes that takes: what the call does and what its workspace is measured by.
struct ProductPlan {
    enum Path { FEW, TILES, LAID, GENERAL } path;
    bool scaled;
    size_t lay, bytes;                   // codes laid out (whole 256 bytes), all
};
static ProductPlan product_plan(const dmmv_block_matrix* x, const dmmv_block_matrix* w, bool f32) {
    const int64_t T = x->rows, O = w->rows, K = x->cols;
    ProductPlan p = {ProductPlan::GENERAL, (constant_rows(x) || x->scale_type == DMMV_E8M0) && (constant_rows(w) || w->scale_type == DMMV_E8M0), 0, 0};
    // Few tokens, us by registers and by tiles (T x O x K): 32 x 4096 x 4096 9.9 and 12.7, 24 x 8192 x 4096 15.3 and 16.1, 32 x 8192 x 4096
    // 17.5 and 16.1, 24 x 11008 x 4096 21 and 16.5, 24 x 8192 x 8192 27.5 and 26; few outputs of a long contraction 24 x 4096 x 8192 15.2 and 26,
    // 24 x 4096 x 11008 17.6 and 34; 64 x 4096 x 4096 16.4 and 13.8; where the large tiles do not apply, 64 (32 bits): 17.4 and 19.3, 128: 32.5 and 20.
    const bool tiles = !f32 && p.scaled && aligned(x) && aligned(w);
    const bool wide = T > 16 && O >= 8192 && (double)T * (double)O * (double)K >= 9e8;
    if (T <= (!tiles ? 64 : wide ? 16 : 32)) {
        p.path = ProductPlan::FEW;
        return p;
    }
    const size_t lay = product_lay_bytes(T, O, K);
    if (tiles) p.path = ProductPlan::TILES;
    else if (!f32 && p.scaled && lay > 0) p.path = ProductPlan::LAID;
    else return p;
    if (p.path == ProductPlan::LAID) p.lay = (lay + 255) / 256 * 256;
    p.bytes = p.lay + (product_shared(T, K, lay) ? product_part_bytes(T, O, K) : 0);
    return p;
}

template <class T, bool WIDE, bool EPI>
static dmmv_status product(const ProductPlan& plan, const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, const ProductOut<T, EPI>& out,
                           void* ws, hipStream_t s) {
    const ProductScales how = {!constant_rows(x), !constant_rows(w)};
    const bool scaled = plan.scaled;
    if (plan.path == ProductPlan::FEW) return launch_few<T, WIDE, EPI>(x, w, how, scaled, bias, out, s);
    float* part = plan.bytes > plan.lay ? reinterpret_cast<float*>(static_cast<char*>(ws) + plan.lay) : nullptr;
    if constexpr (sizeof(T) == 2) {
        if (plan.path == ProductPlan::TILES) return product_tiled<EPI>(x, w, bias, out, part, s);
        if (plan.path == ProductPlan::LAID) {
            dmmv_block_matrix lx = *x, lw = *w;
            lx.ld = lw.ld = ceil_div(x->cols, 128) * 128;
            lx.codes = ws;
            lw.codes = static_cast<uint8_t*>(ws) + x->rows * lx.ld;
            DMMV_TRY(layer_lay_codes(x, static_cast<uint8_t*>(lx.codes), lx.ld, s));
            DMMV_TRY(layer_lay_codes(w, static_cast<uint8_t*>(lw.codes), lw.ld, s));
            return product_tiled<EPI>(&lx, &lw, bias, out, part, s);
        }
    }
    const int64_t tiles_t = ceil_div(x->rows, 64), tiles_o = ceil_div(w->rows, 64);
    if (tiles_t > INT32_MAX / 4 / tiles_o) return fail(DMMV_ERR_SHAPE, "y: more tiles than a launch takes");
    const dim3 grid((unsigned)(tiles_t * tiles_o));
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, x->rows, w->rows, x->cols, layer_view(x), layer_view(w), how, bias, out, (int32_t)tiles_t,
                           (int32_t)tiles_o);
    };
    const bool one_each = tiles_t * tiles_o <= 256;
    if (sizeof(T) == 2) scaled ? launch(k_block_product<T, true, 1, EPI>) : launch(k_block_product<T, false, 3, EPI>);
    else if (one_each) scaled ? launch(k_block_product<T, true, 1, EPI>) : launch(k_block_product<T, false, sizeof(T) == 4 ? 1 : 3, EPI>);
    else scaled ? launch(k_block_product<T, true, sizeof(T) == 4 ? 4 : 1, EPI>) : launch(k_block_product<T, false, 3, EPI>);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

// The same with what follows it.  8 bits come from the kernel that has whole blocks of 128 outputs of a row (tiles, shares); the others write
// v in 32 bits, `v` bytes further on in the workspace.  8 bits of up to 64 tokens come from the 16-bit instructions, which sum in 32 bits: by the
// 8-bit ones a number in some 500 goes to the other neighbour on the 8-bit grid.  What that costs, in 8 bits with SiLU and weights from memory, us here and by the
// rule of product_plan: one token of 4096 by 11008 0.5 (the instructions alone); 24 tokens of 4096 to 11008 outputs 25.2 and 24.0, 32 28.4 and 23.9, 64 44.6 and 24.6;
// 64 of 11008 to 4096 33.6 and 23.6, of 4096 to 4096 18.8 and 14.8; 8192 to 8192 24 31.2 and 37.6 (the rule's own weak place), 64 56.8 and 23.4.
struct LinearPlan {
    ProductPlan product;
    size_t v, bytes;                     // where v begins (0 without one: bytes = product.bytes), all
    bool pass;                           // 8 bits by a pass over v
};
static LinearPlan linear_plan(const dmmv_block_matrix* x, const dmmv_block_matrix* w, bool f32, bool has_q) {
    LinearPlan p = {product_plan(x, w, f32), 0, 0, false};
    if (has_q && x->rows <= 64) {
        p.product.path = ProductPlan::FEW;
        p.product.lay = p.product.bytes = 0;
    }
    p.pass = has_q && (p.product.path == ProductPlan::FEW || p.product.path == ProductPlan::GENERAL);
    p.v = (p.product.bytes + 255) / 256 * 256;
    p.bytes = p.pass ? p.v + (size_t)x->rows * w->rows * 4 : p.product.bytes;
    return p;
}

template <class T>
static dmmv_status linear(const LinearPlan& plan, const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, ProductOut<T, true> out,
                          const dmmv_block_matrix* q, void* ws, hipStream_t s) {
    if (plan.pass) out.v = reinterpret_cast<float*>(static_cast<char*>(ws) + plan.v);
    else if (q) out.q = layer_view(q), out.has_q = 1;
    if constexpr (sizeof(T) == 2)
        if (!q) return product<T, false, true>(plan.product, x, w, bias, out, ws, s);
    DMMV_TRY((product<T, true, true>(plan.product, x, w, bias, out, ws, s)));
    return plan.pass ? dmmv_block_quantize(DMMV_F32, out.v, w->rows, q, s) : DMMV_OK;
}

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
    if (x->rows == 0 || w->rows == 0) return DMMV_OK;
    const ProductPlan plan = product_plan(x, w, dtype == DMMV_F32);
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, plan.bytes));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return dtype == DMMV_F32 ? product<float, true, false>(plan, x, w, bias, {static_cast<float*>(y), ldy}, workspace, s)
                             : product<bf16_t, false, false>(plan, x, w, bias, {static_cast<bf16_t*>(y), ldy}, workspace, s);
}

extern "C" size_t dmmv_block_linear_workspace_for(const dmmv_block_matrix* x, const dmmv_block_matrix* w, int32_t dtype, int32_t has_q) {
    if (layer_check_dtype(dtype) != DMMV_OK || layer_check_block(x, false, "x") != DMMV_OK || layer_check_block(w, false, "w") != DMMV_OK) return 0;
    if (x->cols != w->cols || x->rows == 0 || w->rows == 0) return 0;
    return linear_plan(x, w, dtype == DMMV_F32, has_q != 0).bytes;
}

extern "C" dmmv_status dmmv_block_linear(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, int32_t act, const void* residual,
                                         int64_t ldr, int32_t dtype, void* y, int64_t ldy, const dmmv_block_matrix* q, void* u, int64_t ldu,
                                         void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_act(act, true));
    DMMV_TRY(layer_check_block(x, false, "x"));
    DMMV_TRY(layer_check_block(w, false, "w"));
    if (x->cols != w->cols) return fail(DMMV_ERR_SHAPE, "x has %lld columns, w has %lld", (long long)x->cols, (long long)w->cols);
    const int width = layer_width(dtype);
    DMMV_TRY(layer_check_vector(bias, false, "bias"));
    if (residual) DMMV_TRY(layer_check_array(residual, x->rows, w->rows, ldr, width, "residual"));
    if (y) DMMV_TRY(layer_check_array(y, x->rows, w->rows, ldy, width, "y"));
    if (q) DMMV_TRY(layer_check_out_block(q, x->rows, w->rows, "q"));
    if (u) DMMV_TRY(layer_check_array(u, x->rows, w->rows, ldu, width, "u"));
    if (x->rows == 0 || w->rows == 0 || (!y && !q && !u)) return DMMV_OK;
    const LinearPlan plan = linear_plan(x, w, dtype == DMMV_F32, q != nullptr);
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, plan.bytes));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    auto call = [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        const ProductOut<T, true> out = {static_cast<T*>(y), ldy, static_cast<const T*>(residual), ldr, static_cast<T*>(u), ldu, nullptr, BlockView{}, act, 0};
        return linear<T>(plan, x, w, bias, out, q, workspace, s);
    };
    return dtype == DMMV_F32 ? call((float*)nullptr) : call((bf16_t*)nullptr);
}
