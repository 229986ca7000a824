// Gradients of the product of block matrices (include/dmmv_layer.h).
//
// Both large products contract over the ROWS of a block matrix: dx = dy w over the outputs, dw = dy^T x
// over the tokens.  code * scale is exact in bf16 where scales are powers of two, so they run on
// the bf16 matrix cores without rounding the 8-bit operand; what needs 24 bits (32-bit gradients, other
// scales) is cut into three bf16 that sum to it, and the products of parts below the last bit are left out.
#include <type_traits>

#include "dmmv_layer_common.h"

namespace dmmv {

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
                if (m < M && n < N) put_y(c + m * ldc + n, acc[i][j][e]);
            }
}

// ---- large gradients ---------------------------------------------------------------------------------
// bf16 gradients and power-of-two scales, rows of whole chunks of 16 bytes, aligned: tile of 256 x 256, 4 wavefronts (2 x 2, one a SIMD,
// 128 x 128 each), 64 of the contraction a step, two LDS stages.
//   The rows of dy go straight from memory into the LDS.  dx: [m][k], the 16-byte chunk c of row m at c ^ (m & 7), read as it
//   is; dw: [k][m], chunk c of row k at c ^ 4 (k & 3), read transposed.
//   The codes go through registers: a thread has 16 of a row, converted to bf16 with the row's one scale (exact), [k][n] with
//   chunk c of row k at c ^ 4 (k & 3), read transposed.  (Scales along the contraction are the reason for converting here: a
//   fragment has 8 rows.)
//   The 4 x 32 lanes of a transposed read are 4 rows of 32 bytes; the places above put 8 such pieces on all 64 banks.
// The codes are the A operand, so that a lane's results come in fours along a row of the output.
// The loop is that of the large product: a quadrant of 16 products at a time, all else in their shadows.
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

constexpr int GT_STAGE = 65536, GT_LDS = 256 * (256 * 2 + 16) > 2 * GT_STAGE ? 256 * (256 * 2 + 16) : 2 * GT_STAGE;

// 4 x 4 results of 16 bits a lane, transposed in its group of 16 lanes
__device__ __forceinline__ piece8 read_transposed(const uint8_t* p) {
    return __builtin_bit_cast(piece8, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p));
}

template <bool TRANS, class TC>
__global__ __launch_bounds__(256) void k_block_grad_tiled(int64_t M, int64_t N, int64_t Kc, const bf16_t* __restrict__ a, int64_t lda,
                                                          BlockView b, TC* __restrict__ c, int64_t ldc, int32_t tiles_m, int32_t tiles_n) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wv & 1) * 128, wn = (wv >> 1) * 128;
    int tile_m, tile_n;
    tile_of_workgroup(tiles_m, tiles_n, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * 256, n0 = (int64_t)tile_n * 256;

    // requests of dy: 1 KB each, 8 a wavefront and step.  dx: 8 rows of 64; dw: 2 rows of 256
    const uint32_t lda2 = (uint32_t)lda * 2;
    const uint8_t* ab = reinterpret_cast<const uint8_t*>(TRANS ? a + m0 : a + m0 * lda);
    const int64_t arows = TRANS ? Kc : min(M - m0, (int64_t)256), acols = TRANS ? M - m0 : Kc;
    uint32_t offa[2];                                // TRANS: of even and odd requests
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if (TRANS) {
            const int row = lane >> 5;
            offa[p] = row * lda2 + (((lane & 31) ^ (((2 * p + row) & 3) << 2)) << 4);
        } else {
            const int row = lane >> 3;
            offa[p] = row * lda2 + (((lane & 7) ^ row) << 4);
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    auto bring = [&](int kb, int stage, int q) __attribute__((always_inline)) {      // q: 0 .. 7
        const int at = wv * 8 + q;
        if constexpr (TRANS) {
            // a buffer of the step's 64 rows: offsets stay small however many rows there are
            const int64_t row0 = (int64_t)kb * 64;
            const intx4 buf = buffer_of(ab + row0 * lda2, (uint32_t)((min(arows - row0, (int64_t)64) - 1) * lda2 + min(acols, (int64_t)256) * 2));
            lds_request(buf, offa[q & 1], (uint32_t)(2 * at) * lda2, lds0 + stage + at * 1024);
        } else {
            const intx4 buf = buffer_of(ab, (uint32_t)(arows - 1) * lda2 + (uint32_t)acols * 2);
            lds_request(buf, offa[0], (uint32_t)kb * 128 + (uint32_t)(8 * at) * lda2, lds0 + stage + at * 1024);
        }
    };
    // codes: thread has chunk tid % 16 of rows tid / 16 + 16 u
    const int brow = tid >> 4, bchunk = tid & 15;
    const int64_t bcol = n0 + bchunk * 16;
    const int64_t fb = min(bcol, N - 1) >> 7;
    const uint8_t* bb = b.codes + n0;
    const int nlast = (int)min(N - n0, (int64_t)256);
    // without scales a byte is read all the same (a branch around the load would wait for it) and not used
    const uint8_t* sp = b.scales ? static_cast<const uint8_t*>(b.scales) : b.codes;
    const int64_t srow = b.scales ? b.srow : 0, sblk = b.scales ? b.sblk : 0;
    piece16 rb[4];
    uint32_t rs[4];
    auto request = [&](int kb, int u) __attribute__((always_inline)) {
        const int64_t row = min((int64_t)kb * 64 + brow + 16 * u, Kc - 1);
        // (a chunk past the row's end gives columns that are not stored: the row's last is taken)
        rb[u] = *reinterpret_cast<const piece16*>(bb + row * b.ld + min(bchunk * 16, nlast - 16));
        rs[u] = sp[(row >> b.shift) * srow + fb * sblk];
    };
    const int bput = 32768 + brow * 512 + (((bchunk * 2) ^ ((brow & 3) << 2)) << 4);
    auto deposit = [&](int stage, int u) __attribute__((always_inline)) {
        uint8_t* p = lds + stage + bput + u * 8192;
        const uint32_t e = b.scales ? rs[u] : 127u;
        *reinterpret_cast<bf16x8_t*>(p) = scaled8((int)rb[u][0], (int)rb[u][1], e);
        *reinterpret_cast<bf16x8_t*>(p + 16) = scaled8((int)rb[u][2], (int)rb[u][3], e);
    };

    floatx16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;

    piece8 fn[4][4][2];                              // codes: [tile][16 of k][half]
    piece8 fm[4][4][2];                              // dy
    // transposed reads: group g of 16 lanes has columns 16 (g & 1) .. and rows 8 (g / 2) .. of a 32 x 16 fragment
    const int tk = (lane >> 5) * 8 + ((lane & 15) >> 2), tn = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    // (rows 16 s + 8 g + 4 h + r: the place depends on r alone; tiles of 32 columns are 64 bytes apart)
    auto transposed = [&](int base, int w0, int tile, int s, int h) __attribute__((always_inline)) {
        const int col = w0 + tn, chunk = (col >> 3) + 4 * tile, sw = (tk & 3) << 2;
        return read_transposed(lds + base + (tk + 4 * h) * 512 + s * 8192 + ((chunk ^ sw) << 4) + (col & 7) * 2);
    };
    auto frag_n = [&](int stage, int i, int s, int h) __attribute__((always_inline)) { fn[i][s][h] = transposed(stage + 32768, wn, i, s, h); };
    const int mrow = wm + (lane & 31);
    auto frag_m = [&](int stage, int j, int s, int h) __attribute__((always_inline)) {
        if constexpr (TRANS) {
            fm[j][s][h] = transposed(stage, wm, j, s, h);
        } else if (h == 0) {
            const piece16 v = *reinterpret_cast<const piece16*>(lds + stage + (mrow + 32 * j) * 128 + (((2 * s + (lane >> 5)) ^ (mrow & 7)) << 4));
            fm[j][s][0] = piece8{v[0], v[1]};
            fm[j][s][1] = piece8{v[2], v[3]};
        }
    };
    auto mul = [&](int i, int j, int s) __attribute__((always_inline)) {
        const piece16 n = {fn[i][s][0][0], fn[i][s][0][1], fn[i][s][1][0], fn[i][s][1][1]}, m = {fm[j][s][0][0], fm[j][s][0][1], fm[j][s][1][0], fm[j][s][1][1]};
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, n), __builtin_bit_cast(bf16x8_t, m), acc[i][j], 0, 0, 0);
    };
    // Products of half ih of the codes' tiles with half jh of dy's.  FM: the fragments for the next quadrant are of dy
    // (half fh, from the stage at fs), else of the codes.  NEXT: block `to` of dy (requests 4 r ..) and of the codes
    // (chunks 2 r ..; registers hold them already) go to the stage at rs, and the codes of block `to` + 1 are requested.
    auto quad = [&](auto ih, auto jh, auto FM, int fs, auto fh, auto NEXT, auto r, int to, int rs_, int then) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                mul(ih.value * 2 + (p >> 1), jh.value * 2 + (p & 1), s);
                const int slot = s * 4 + p;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int f = slot >> 1, hh = slot & 1;          // fragment f of 8, half by half
                    if (h != hh) continue;
                    if (FM.value) frag_m(fs, fh.value * 2 + (f & 1), f >> 1, h);
                    else frag_n(fs, fh.value * 2 + (f & 1), f >> 1, h);
                }
                if (NEXT.value) {
                    if ((slot & 3) == 1) bring(to, rs_, r.value * 4 + (slot >> 2));
                    if ((slot & 7) == 2) deposit(rs_, r.value * 2 + (slot >> 3));
                    if ((slot & 7) == 6) request(then, r.value * 2 + (slot >> 3));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    auto step = [&](auto P, auto Q, int to, int then) __attribute__((always_inline)) {      // P: parity, Q = 1 - P
        constexpr int cur = P.value * GT_STAGE, nxt = Q.value * GT_STAGE;
        quad(C0, P, C1, cur, Q, C0, C0, 0, 0, 0);
        quad(C0, Q, C0, cur, C1, C0, C0, 0, 0, 0);
        lds_requests_left<0>();
        __syncthreads();
        quad(C1, Q, C0, nxt, C0, C1, C0, to, cur, then);
        quad(C1, P, C1, nxt, Q, C1, C1, to, cur, then);
    };

    const int paired = (int)(Kc >> 7) * 2, last = paired - 1, nb = (int)((Kc + 63) >> 6);
    if (paired > 0) {
#pragma unroll
        for (int q = 0; q < 8; ++q) bring(0, 0, q);
#pragma unroll
        for (int q = 0; q < 8; ++q) bring(1, GT_STAGE, q);
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (k > 0) deposit((k - 1) * GT_STAGE, u);
                request(min(k, last), u);
            }
        lds_requests_left<0>();
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    frag_n(0, t, s, h);
                    frag_m(0, t, s, h);
                }
        for (int kb = 0; kb < paired; kb += 2) {
            step(C0, C1, min(kb + 2, last), min(kb + 3, last));
            step(C1, C0, min(kb + 3, last), min(kb + 4, last));
        }
        lds_requests_left<0>();
    }
    // what is left of the contraction, at most one whole block and a shorter one
#pragma unroll 1
    for (int kb = paired; kb < nb; ++kb) {
        const int left = (int)(Kc - kb * 64ll);
        __syncthreads();
#pragma unroll 1
        for (int q = 0; q < 8; ++q) {
            const int at = wv * 8 + q;
            const int row = TRANS ? 2 * at + (lane >> 5) : 8 * at + (lane >> 3);
            piece16 v = {0u, 0u, 0u, 0u};
            if constexpr (TRANS) {
                const int col = ((lane & 31) ^ ((row & 3) << 2)) * 8;
                if (row < left && m0 + col < M) v = *reinterpret_cast<const piece16*>(ab + ((int64_t)kb * 64 + row) * lda2 + col * 2);
            } else {
                const int col = ((lane & 7) ^ (row & 7)) * 8;
                if (m0 + row < M && col < left) v = *reinterpret_cast<const piece16*>(ab + (int64_t)row * lda2 + ((int64_t)kb * 64 + col) * 2);
            }
            *reinterpret_cast<piece16*>(lds + at * 1024 + lane * 16) = v;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            request(kb, u);
            if (brow + 16 * u >= left) rb[u] = piece16{0u, 0u, 0u, 0u}, rs[u] = 127u;
            deposit(0, u);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    frag_n(0, t, s, h);
                    frag_m(0, t, s, h);
                }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) mul(i, j, s);
    }
    // results through the LDS, 256 (bf16) or 128 rows (32 bits) at a time
    constexpr int W = (int)sizeof(TC), ROWS = W == 2 ? 256 : 128, LDO = 256 * W + 16, PER = 16 / W, CPR = 256 / PER;
#pragma unroll
    for (int h = 0; h < 256 / ROWS; ++h) {
        __syncthreads();
        if (ROWS == 256 || wm == 128 * h) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                        put4(reinterpret_cast<TC*>(lds + ((wm - ROWS * h) + 32 * j + (lane & 31)) * LDO) + wn + 32 * i + 8 * g + (lane >> 5) * 4, v);
                    }
        }
        __syncthreads();
        for (int q = tid; q < ROWS * CPR; q += 256) {
            const int r = q / CPR, at = q % CPR;
            const int64_t m = m0 + ROWS * h + r, n = n0 + at * PER;
            if (m >= M || n >= N) continue;
            const piece16 v = *reinterpret_cast<const piece16*>(lds + r * LDO + at * 16);
            TC* dst = c + m * ldc + n;
            if (n + PER <= N) {
                *reinterpret_cast<piece16_any*>(dst) = v;
            } else {
                const TC* one = reinterpret_cast<const TC*>(lds + r * LDO + at * 16);
                for (int e = 0; e < PER && n + e < N; ++e) dst[e] = one[e];
            }
        }
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
    if constexpr (sizeof(TA) == 2) {
        const int64_t big = ceil_div(M, 256) * ceil_div(N, 256);
        if (exact && M >= 256 && N >= 256 && (TRANS ? M : Kc) % 8 == 0 && N % 16 == 0 && lda % 8 == 0 && lda < 1 << 22 && (uintptr_t)a % 16 == 0 && b->ld % 16 == 0 &&
            (uintptr_t)b->codes % 16 == 0 && big <= INT32_MAX / 4) {
            const void* kern = (const void*)k_block_grad_tiled<TRANS, TC>;
            DMMV_TRY(ensure_dynamic_lds(kern, GT_LDS));
            hipLaunchKernelGGL((k_block_grad_tiled<TRANS, TC>), dim3((unsigned)big), dim3(256), GT_LDS, s, M, N, Kc, a, lda, layer_view(b), c,
                               ldc, (int32_t)ceil_div(M, 256), (int32_t)ceil_div(N, 256));
            DMMV_LAUNCH_CHECK();
            return DMMV_OK;
        }
    }
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
