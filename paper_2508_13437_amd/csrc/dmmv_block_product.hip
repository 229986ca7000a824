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

// 16 codes of which `left` (any number) belong to the row, the others zero
__device__ __forceinline__ piece16 chunk_tail(const uint8_t* __restrict__ p, int left) {
    if (left >= 16) return *reinterpret_cast<const piece16_any*>(p);
    piece16 a = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < left) a[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return a;
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


// ---- large products ------------------------------------------------------------------------------
// Tile of 32 MI tokens x 32 NI outputs, 4 wavefronts (2 x 2), one block of 128 a step.  A step's codes go
// through registers into one of two LDS stages while the other is multiplied.  The rows of w are the A
// operand, so that a lane's four results are consecutive outputs of one token.
//   LDS row: 128 codes, the 16-byte chunk c of row r at c ^ (r & 7): neither the 8 lanes that write a row
//   nor the 8 rows that are read together meet in a bank.
// SCALED: power-of-two scales go into the instruction (8 bits) or the conversion to bf16 (32-bit results), four
// blocks' exponents in one register; scales that are the same along a row are left to the end.
// WTILE: the scales of w are the same for 128 rows, or for a whole row.
// Otherwise a block's sum is multiplied by its two scales in 32 bits.
struct ProductScales {
    int32_t x_blocks, w_blocks;         // SCALED: exponents per block, else constant along the row
};

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

constexpr int product_lds(int MI, int NI, int width, bool wtile) {
    const int stages = 2 * 128 * 32 * (MI + NI) + 68 * (32 * MI + (wtile ? (32 * NI + 127) / 128 : 32 * NI)), out = 32 * MI * (32 * NI * width + 16);
    return stages > out ? stages : out;
}

// a pointer that is the same in every lane, in scalar registers
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
    const uint64_t u = (uint64_t)p;
    return (const uint8_t*)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32)) << 32) |
                            (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u));
}
// 16 bytes a lane from memory (a uniform base and an offset of 32 bits each) to 1 KB of LDS at a uniform address, in the
// order of the lanes; in flight until lds_requests_done().  The instruction writes no register.
__device__ __forceinline__ void lds_request(const uint8_t* base, uint32_t off, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(base));
}
__device__ __forceinline__ void lds_requests_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <class T, int MI, int NI, bool SCALED, bool WTILE>
__global__ __launch_bounds__(256) void k_block_product_tiled(int64_t T_, int64_t O, int64_t K, BlockView x, BlockView w, ProductScales how,
                                                             const float* __restrict__ bias, T* __restrict__ y, int64_t ldy,
                                                             int32_t tiles_t, int32_t tiles_o) {
    extern __shared__ __align__(16) uint8_t lds[];
    constexpr int BM = 32 * MI, BN = 32 * NI, STAGE = 128 * (BM + BN);
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = (wv & 1) * (16 * MI), wo = (wv >> 1) * (16 * NI);
    // (a division runs on the vector unit: the tile's place goes back to scalar registers)
    const int tile_t = __builtin_amdgcn_readfirstlane((int)blockIdx.x / tiles_o), tile_o = (int)blockIdx.x - tile_t * tiles_o;
    const int64_t t0 = (int64_t)tile_t * BM, o0 = (int64_t)tile_o * BN;
    const int nb = (int)((K + 127) >> 7);

    // One request brings 8 rows of a step (1 KB) from memory to the LDS, 16 bytes a lane in the order of the lanes:
    // lane l has row l / 8 and the chunk that belongs at place l % 8 of it.  A wavefront brings 8 MI rows of x and
    // 8 NI of w.
    const uint8_t* xb = uniform(x.codes + t0 * x.ld);
    const uint8_t* wb = uniform(w.codes + o0 * w.ld);
    const uint32_t ldx = (uint32_t)x.ld, ldw = (uint32_t)w.ld;                    // below 2^23
    const uint32_t lastx = (uint32_t)min((int64_t)BM - 1, T_ - 1 - t0), lastw = (uint32_t)min((int64_t)BN - 1, O - 1 - o0);
    const int crow = lane >> 3, cchunk = (lane & 7) ^ crow;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

    floatx4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    // Exponents of SB blocks of every row of the tile, one byte each (WTILE: of every 128 rows of w), past the stages; a
    // lane has those of two steps in a register.
    constexpr int SB = 64, SROW = SB + 4, WROWS = WTILE ? ((BN + 127) / 128) : BN, NS = WTILE ? 1 : NI;
    uint8_t* scl = lds + 2 * STAGE;
    uint32_t sx[MI], sw[NS];
    if (SCALED) {                                    // what is not read from the tables is 1
        for (int i = tid; i < (BM + WROWS) * (SROW / 4); i += 256) reinterpret_cast<uint32_t*>(scl)[i] = 0x7F7F7F7Fu;
        __syncthreads();
    }
#define BP_SCALES_STAGE(kb)                                                                                     \
    {                                                                                                           \
        if (how.x_blocks) stage_exponents(x, t0, T_, 1, BM, kb, min(nb - (kb), SB), scl, SROW);                 \
        if (how.w_blocks) stage_exponents(w, o0, O, WTILE ? 128 : 1, WROWS, kb, min(nb - (kb), SB), scl + BM * SROW, SROW); \
    }
#define BP_SCALES_TAKE(kb)                                                                                      \
    {                                                                                                           \
        const uint8_t* p_ = scl + ((kb) & (SB - 1));                                                            \
        _Pragma("unroll") for (int j = 0; j < MI; ++j)                                                          \
            sx[j] = *reinterpret_cast<const uint16_t*>(p_ + (wt + 16 * j + lr) * SROW);                         \
        _Pragma("unroll") for (int i = 0; i < NS; ++i)                                                          \
            sw[i] = *reinterpret_cast<const uint16_t*>(p_ + (BM + (WTILE ? wo >> 7 : wo + 16 * i + lr)) * SROW); \
    }

    // request q of a step: 8 rows of x (q < MI) or of w
    static_assert(MI == NI && MI % 4 == 0, "quadrants of the wavefront's tile");
    // (rows' offsets are made anew each time: three instructions instead of a register)
#define BP_FRESH()            \
    uint32_t r_ = crow;       \
    asm volatile("" : "+v"(r_))
#define BP_ROW(q) ((uint32_t)(wv * 8 * MI + 8 * ((q) % MI)) + r_)
#define BP_OFF(q) ((q) < MI ? __umul24(min(BP_ROW(q), lastx), ldx) : __umul24(min(BP_ROW(q), lastw), ldw))
#define BP_PLACE(q) (((q) < MI ? 0 : BM * 128) + (wv * MI + (q) % MI) * 1024)
#define BP_BRING(kb, stage, q)                                                                                  \
    lds_request(((q) < MI ? xb : wb) + (int64_t)(kb) * 128, BP_OFF(q) + cchunk * 16u, lds0 + (stage) * STAGE + BP_PLACE(q))

    intx8 fx[MI], fw[NI];
    const int c0 = (lg ^ (lr & 7)) << 4, c1 = c0 ^ 64;
    const uint8_t* px0 = lds + (wt + lr) * 128;
    const uint8_t* pw0 = lds + BM * 128 + (wo + lr) * 128;
#define BP_FRAG(f, p, stage, i)                                                                                 \
    {                                                                                                           \
        const piece16 a_ = *reinterpret_cast<const piece16*>((p) + (stage) * STAGE + (i) * 2048 + c0);          \
        const piece16 b_ = *reinterpret_cast<const piece16*>((p) + (stage) * STAGE + (i) * 2048 + c1);          \
        f[i] = intx8{(int)a_[0], (int)a_[1], (int)a_[2], (int)a_[3], (int)b_[0], (int)b_[1], (int)b_[2], (int)b_[3]}; \
    }
#define BP_MUL(byte, i, j)                                                                                            \
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i], fx[j], acc[i][j], 0, 0, byte, (int)sw[WTILE ? 0 : (i)], byte, (int)sx[j])
    // One quadrant of the wavefront's tile in MI/2 groups: a fragment for a later quadrant, some requests, NI/2 products
#define BP_QUAD(byte, ih, jh, FRAG, REQ0, NREQ, REQ_STAGE, REQ_KB)                                                    \
    _Pragma("unroll") for (int g = 0; g < MI / 2; ++g) {                                                        \
        FRAG;                                                                                                   \
        BP_FRESH();                                                                                             \
        _Pragma("unroll") for (int q = 0; q < (NREQ); ++q) BP_BRING(REQ_KB, REQ_STAGE, (REQ0) + g * (NREQ) + q); \
        _Pragma("unroll") for (int i = 0; i < NI / 2; ++i) BP_MUL(byte, (ih) * (NI / 2) + i, (jh) * (MI / 2) + g); \
        __builtin_amdgcn_sched_barrier(0);                                                                      \
    }
#define BP_FRAG_X(stage, h) BP_FRAG(fx, px0, stage, (h) * (MI / 2) + g)
#define BP_FRAG_W(stage, h) BP_FRAG(fw, pw0, stage, (h) * (NI / 2) + g)
    // A step: four quadrants, each with one new half of fragments.  X0: the half of x that is there at the start;
    // the other half comes first, and at the end next step's w half 0 and x half 1 - X0 are there.  The barrier between
    // the second and third quadrant: every wavefront has read all of this stage, and the next stage is whole; from there
    // on this stage takes the step after next.
#define BP_STEP(P, X0, kb)                                                                                      \
    {                                                                                                           \
        const int k2_ = min((kb) + 2, last);                                                                    \
        BP_QUAD(P, 0, X0, BP_FRAG_X(P, 1 - (X0)), 0, 0, 0, 0);                                                  \
        BP_QUAD(P, 0, 1 - (X0), BP_FRAG_W(P, 1), 0, 0, 0, 0);                                                   \
        lds_requests_done();                                                                                    \
        __syncthreads();                                                                                        \
        BP_QUAD(P, 1, 1 - (X0), BP_FRAG_W(1 - (P), 0), 0, 2, P, k2_);                                           \
        BP_QUAD(P, 1, X0, BP_FRAG_X(1 - (P), 1 - (X0)), MI, 2, P, k2_);                                         \
    }

    // blocks in pairs (the loop's body is one piece of straight code, or the compiler takes the products out of it)
    const int paired = (int)(K >> 8) * 2, last = paired - 1;
    if (paired > 0) {
        {
            BP_FRESH();
#pragma unroll
            for (int q = 0; q < 2 * MI; ++q) BP_BRING(0, 0, q);
#pragma unroll
            for (int q = 0; q < 2 * MI; ++q) BP_BRING(1, 1, q);
        }
        if (SCALED) BP_SCALES_STAGE(0);
        lds_requests_done();
        __syncthreads();
#pragma unroll
        for (int g = 0; g < MI / 2; ++g) {
            BP_FRAG_W(0, 0);
            BP_FRAG_X(0, 0);
        }
        for (int kb = 0;;) {
            const int end = min(kb + SB, paired);
            for (; kb < end; kb += 2) {
                if (SCALED) BP_SCALES_TAKE(kb);
                BP_STEP(0, 0, kb);
                BP_STEP(1, 1, kb + 1);
            }
            if (kb >= paired) break;
            __syncthreads();
            if (SCALED) BP_SCALES_STAGE(kb);
            __syncthreads();
        }
        lds_requests_done();
    }
    // one whole block at most, and a last shorter one: zeros past the row's end
#pragma unroll 1
    for (int kb = paired; kb < nb; ++kb) {
        const int left = (int)(K - kb * 128ll) - cchunk * 16;
        __syncthreads();
        if (SCALED && (kb == paired && (kb & (SB - 1)) == 0)) BP_SCALES_STAGE(kb);
        {
            BP_FRESH();
#pragma unroll 1
            for (int q = 0; q < MI; ++q) {
                *reinterpret_cast<piece16*>(lds + BP_PLACE(q) + lane * 16) = chunk_tail(xb + kb * 128ll + BP_OFF(q) + cchunk * 16, left);
                const int p = q + MI;
                *reinterpret_cast<piece16*>(lds + BP_PLACE(p) + lane * 16) = chunk_tail(wb + kb * 128ll + BP_OFF(p) + cchunk * 16, left);
            }
        }
        __syncthreads();
        if (SCALED) BP_SCALES_TAKE(kb & ~1);
        if (SCALED && (kb & 1)) {
#pragma unroll
            for (int j = 0; j < MI; ++j) sx[j] >>= 8;
#pragma unroll
            for (int i = 0; i < NS; ++i) sw[i] >>= 8;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < MI / 2; ++g) {
                BP_FRAG_W(0, h);
                BP_FRAG_X(0, h);
            }
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < MI; ++j) BP_MUL(0, i, j);
    }
    __syncthreads();
    // results through the LDS: rows of the tile, stored 16 bytes a lane
    constexpr int LDO = BN * (int)sizeof(T) + 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        float bo[4], so[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t o = min(o0 + wo + 16 * i + lg * 4 + e, O - 1);
            bo[e] = bias ? bias[o] : 0.0f;
            so[e] = SCALED && !how.w_blocks ? scale_at(w, o, 0) : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < MI; ++j) {
            const float st = SCALED && !how.x_blocks ? scale_at(x, min(t0 + wt + 16 * j + lr, T_ - 1), 0) : 1.0f;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = dmmv_fma(acc[i][j][e], so[e] * st, bo[e]);
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
        T* dst = y + t * ldy + o;
        if (o + PER <= O) {
            *reinterpret_cast<piece16_any*>(dst) = v;
        } else {
            const T* one = reinterpret_cast<const T*>(lds + r * LDO + h * 16);
            for (int e = 0; e < PER && o + e < O; ++e) dst[e] = one[e];
        }
    }
}

// scales that are the same along a row leave the sum
static bool constant_rows(const dmmv_block_matrix* q) { return !q->scales || q->scale_block_stride == 0 || q->cols <= 128; }

// rows that requests of 16 bytes can bring to the LDS, with offsets of 24 x 24 bits
static bool aligned(const dmmv_block_matrix* q) { return q->ld < 1 << 23 && q->ld % 16 == 0 && (uintptr_t)q->codes % 16 == 0; }

template <class T, int MI, int NI, bool SCALED, bool WTILE>
static dmmv_status launch_tiled(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, T* y, int64_t ldy, hipStream_t s) {
    const int64_t tiles_t = ceil_div(x->rows, 32 * MI), tiles_o = ceil_div(w->rows, 32 * NI);
    if (tiles_t > INT32_MAX / tiles_o) return fail(DMMV_ERR_SHAPE, "y: more tiles than a launch takes");
    const void* kern = (const void*)k_block_product_tiled<T, MI, NI, SCALED, WTILE>;
    constexpr int bytes = product_lds(MI, NI, sizeof(T), WTILE);
    DMMV_TRY(ensure_dynamic_lds(kern, bytes));
    const ProductScales how = {!constant_rows(x), !constant_rows(w)};
    hipLaunchKernelGGL((k_block_product_tiled<T, MI, NI, SCALED, WTILE>), dim3((unsigned)(tiles_t * tiles_o)), dim3(256), bytes, s, x->rows, w->rows,
                       x->cols, layer_view(x), layer_view(w), how, bias, y, ldy, (int32_t)tiles_t, (int32_t)tiles_o);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T>
static dmmv_status product(const dmmv_block_matrix* x, const dmmv_block_matrix* w, const float* bias, T* y, int64_t ldy, hipStream_t s) {
    const bool scaled = (constant_rows(x) || x->scale_type == DMMV_E8M0) && (constant_rows(w) || w->scale_type == DMMV_E8M0);
    if constexpr (sizeof(T) == 2)
        if (scaled && aligned(x) && aligned(w)) {
            const bool wtile = constant_rows(w) || w->scale_rows == 128;
            if (x->rows >= 1024 && wtile) return launch_tiled<T, 8, 8, true, true>(x, w, bias, y, ldy, s);
            return launch_tiled<T, 4, 4, true, false>(x, w, bias, y, ldy, s);
        }
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
