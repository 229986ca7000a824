// Gradients of the product of block matrices (include/dmmv_layer.h).
//
// Both large products contract over the ROWS of a block matrix: dx = dy w over the outputs, dw = dy^T x
// over the tokens.  code * scale is exact in bf16 where scales are powers of two, so they run on
// the bf16 matrix cores without rounding the 8-bit operand; what needs 24 bits (32-bit gradients, other
// scales) is cut into three bf16 that sum to it, and the products of parts below the last bit are left out.
#include <type_traits>

#include "dmmv_layer_common.h"

namespace dmmv {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));

// 4 x 4 numbers of 16 bits a lane, transposed in its group of 16 lanes
__device__ __forceinline__ piece8 read_transposed(const uint8_t* p) {
    return __builtin_bit_cast(piece8, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)p));
}

// C[m][n] = sum_k A(m, k) B(k, n), A(m, k) = a[m][k] or (TRANS) a[k][m], B a block matrix [k][n].
// PA, PB: bf16 parts that an operand is cut into.  Any sizes, strides and scales.  LAID (TA bf16, PA > 1): `a` is laid out as PA parts
// `plane` numbers apart, the smallest first, with zeros up to a multiple of 128 rows and columns.
// 64 x 64 tile, 4 wavefronts of 32 x 32, 64 of k a step, requested two steps ahead, two LDS stages; KS groups of 4 wavefronts
// and `slices` workgroups share the contraction where the tiles alone do not fill the chip (the groups are joined
// in order here, the slices by k_block_grad_join).
//   LDS rows of 64 numbers, 128 bytes: [k][.] with the 16-byte chunk c of row k at c ^ 2 (k & 3), read transposed;
//   [m][k] with chunk c of row m at c ^ (m & 7), read as it is.
// The codes are the A operand of the instruction, so that a lane's results come in fours along a row of C.
// Bound by the LDS and the waits of wavefronts in step, the more parts the more: 2048^3 bf16 50 us (345 TFLOP/s); dx of 777 x 1365 x 1003 in
// 32 bits 23 us, 1.3 us a step and 7 for start, join and end.  32-bit scales per block (three parts of the codes): dx and dw of 4096^3 bf16 1510 us.  Requesting all of a step's fragments ahead of the next
// step's writes was no faster.
template <class TA, bool TRANS, int PA, int PB, int KS, class TC>
__global__ __launch_bounds__(256 * KS) void k_block_grad(int64_t M, int64_t N, int64_t Kc, const TA* __restrict__ a, int64_t lda, BlockView b,
                                                         TC* __restrict__ c, int64_t ldc, int32_t tiles_m, int32_t tiles_n, int32_t slices,
                                                         float* __restrict__ part, int64_t plane) {
    constexpr int STAGE = (PA + PB) * 8192;
    constexpr bool LAID = sizeof(TA) == 2 && PA > 1;
    constexpr int RA = LAID ? PA : 1;
    extern __shared__ __align__(16) uint8_t lds_all[];
    const int tid = threadIdx.x & 255, lane = tid & 63;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint8_t* lds = lds_all + group * (2 * STAGE);
    const int wm = (wv & 1) * 32, wn = (wv >> 1) * 32;
    const int tiles = tiles_m * tiles_n, slice = __builtin_amdgcn_readfirstlane((int)blockIdx.x / tiles), tile = (int)blockIdx.x - slice * tiles;
    const int tile_m = __builtin_amdgcn_readfirstlane(tile / tiles_n), tile_n = tile - tile_m * tiles_n;
    const int64_t m0 = tile_m * 64ll, n0 = tile_n * 64ll;
    // this group's share of the steps; all groups have the same barriers
    const int nb = (int)((Kc + 63) >> 6), share = (nb + slices * KS - 1) / (slices * KS);
    const int first = min((slice * KS + group) * share, nb), end = min(first + share, nb);

    const int row = tid >> 3, col = (tid & 7) * 8;   // rows row, row + 32 of a step, 8 columns
    struct Step {
        Raw8<TA> a[2][RA];
        Raw8<uint8_t> b[2];
        uint32_t s[2];
    };
    // Whole steps of rows of 8 numbers and more, and what is addressed number by number: the last step, short rows.
    const bool short_rows = (!LAID && (TRANS ? M : Kc) < 8) || N < 8;
    const int full = short_rows ? 0 : LAID ? nb : (int)(Kc >> 6), lastw = max(full - 1, 0);
    const int a_cut = TRANS && !LAID ? (int)((m0 + col) - min(m0 + col, M - 8)) : 0, b_cut = (int)((n0 + col) - min(n0 + col, N - 8));    // as raw_settle's `moved`
    const int64_t blk = (min(n0 + col, N - 1) >> 7) * b.sblk;
    const TA* ap[2];
    const uint8_t* bp[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        ap[u] = TRANS ? a + (row + 32 * u) * lda + (m0 + col - a_cut) : a + (LAID ? m0 + row + 32 * u : min(m0 + row + 32 * u, M - 1)) * lda + col;
        bp[u] = b.codes + (LAID ? 0 : (row + 32 * u) * b.ld) + (n0 + col - b_cut);
    }
    const int64_t a_step = TRANS ? 64 * lda : 64, b_step = 64 * b.ld;
    auto scale_place = [&](int k) __attribute__((always_inline)) { return (int64_t)(k >> b.shift) * b.srow + blk; };
    auto request_a = [&](Step& r, int u, int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < RA; ++p) r.a[u][p].load(ap[u] + kb * a_step + p * plane);
    };
    auto request = [&](Step& r, int kb) __attribute__((always_inline)) {      // a whole step
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            request_a(r, u, kb);
            if constexpr (LAID) {                    // rows past the last meet zeros of `a`: the last again
                const int k = min(kb * 64 + row + 32 * u, (int)Kc - 1);
                r.b[u].load(bp[u] + k * b.ld);
                r.s[u] = *scale_word(b, scale_place(k));
            } else {
                r.b[u].load(bp[u] + kb * b_step);
                r.s[u] = *scale_word(b, scale_place(kb * 64 + row + 32 * u));
            }
        }
    };
    auto request_slow = [&](Step& r, int kb) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t k = min(kb * 64ll + row + 32 * u, Kc - 1);
            if (LAID) request_a(r, u, kb);
            else if (TRANS) raw_request(r.a[u][0], a + k * lda, m0 + col, M);
            else raw_request(r.a[u][0], a + min(m0 + row + 32 * u, M - 1) * lda, kb * 64ll + col, Kc);
            raw_request(r.b[u], (const uint8_t*)b.codes + k * b.ld, n0 + col, N);
            r.s[u] = *scale_word(b, scale_place((int)k));
        }
    };
    auto deposit = [&](Step& r, int kb, int stage, bool slow) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t k = kb * 64ll + row + 32 * u;
            if (!slow) {
                if (TRANS && a_cut > 0) {
                    if (a_cut >= 8) r.a[u][0] = Raw8<TA>{};
                    else r.a[u][0].right(a_cut);
                }
                if (b_cut > 0) {
                    if (b_cut >= 8) r.b[u] = Raw8<uint8_t>{};
                    else r.b[u].right(b_cut);
                }
            } else {
                if (!LAID) {
                    if (TRANS) raw_settle(r.a[u][0], m0 + col, M, k < Kc);
                    else raw_settle(r.a[u][0], kb * 64ll + col, Kc, true);
                }
                raw_settle(r.b[u], n0 + col, N, k < Kc);
            }
            const uint32_t sbits = word_bits(b, scale_place((int)min(k, Kc - 1)), r.s[u]);
            const int rr = row + 32 * u;
            uint8_t* pa = lds + stage * STAGE + rr * 128 + (((tid & 7) ^ (TRANS ? (rr & 3) << 1 : rr & 7)) << 4);
            uint8_t* pb = lds + stage * STAGE + PA * 8192 + rr * 128 + (((tid & 7) ^ ((rr & 3) << 1)) << 4);
            if constexpr (PA == 1) {
                *reinterpret_cast<piece16*>(pa) = r.a[u][0].v;
            } else if constexpr (LAID) {
#pragma unroll
                for (int i = 0; i < PA; ++i) *reinterpret_cast<piece16*>(pa + i * 8192) = r.a[u][PA - 1 - i].v;
            } else {
                float v[8];
                piece16 w[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = r.a[u][0].get(e);
                split8<3>(v, w);
#pragma unroll
                for (int i = 0; i < 3; ++i) *reinterpret_cast<piece16*>(pa + i * 8192) = w[i];
            }
            if constexpr (PB == 1) {                 // exponents: exact
                *reinterpret_cast<bf16x8_t*>(pb) = scaled8((int)r.b[u].v[0], (int)r.b[u].v[1], b.e8m0 ? (LAID || k < Kc ? sbits : 127u) : 127u);
            } else {
                float v[8];
                piece16 w[3];
                decode8(r.b[u].v, k < Kc ? scale_of(b, sbits) : 0.0f, v);
                split8<3>(v, w);
#pragma unroll
                for (int i = 0; i < 3; ++i) *reinterpret_cast<piece16*>(pb + i * 8192) = w[i];
            }
        }
    };
    floatx16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
    const int tk = (lane >> 5) * 8 + ((lane & 15) >> 2), tn = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
    auto transposed = [&](const uint8_t* base, int w0, int s) __attribute__((always_inline)) {
        piece8 h[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            h[i] = read_transposed(base + (16 * s + tk + 4 * i) * 128 + ((((w0 + tn) >> 3) ^ ((tk & 3) << 1)) << 4) + (tn & 7) * 2);
        return __builtin_bit_cast(bf16x8_t, piece16{h[0][0], h[0][1], h[1][0], h[1][1]});
    };
    auto multiply = [&](int stage) __attribute__((always_inline)) {
        const uint8_t* pa = lds + stage * STAGE;
        const uint8_t* pb = pa + PA * 8192;
        const int mr = wm + (lane & 31);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf16x8_t fm[PA], fn[PB];
#pragma unroll
            for (int p = 0; p < PA; ++p) {
                if constexpr (TRANS) fm[p] = transposed(pa + p * 8192, wm, s);
                else fm[p] = *reinterpret_cast<const bf16x8_t*>(pa + p * 8192 + mr * 128 + (((2 * s + (lane >> 5)) ^ (mr & 7)) << 4));
            }
#pragma unroll
            for (int p = 0; p < PB; ++p) fn[p] = transposed(pb + p * 8192, wn, s);
            constexpr int PM = PA > PB ? PA : PB;     // parts p, r with p + r >= PM are below 24 bits
#pragma unroll
            for (int p = PA - 1; p >= 0; --p)
#pragma unroll
                for (int r = PB - 1; r >= 0; --r)
                    if (p + r < PM) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fn[r], fm[p], acc, 0, 0, 0);
        }
    };
    // Requests are made without a condition, or a use would wait for all of them; those past the end ask for the last whole
    // step again.  Every group has the same barriers.
    Step r0, r1;
    const int e1 = min(end, full);
    if (full > 0) {
        request(r0, min(first, lastw));
        request(r1, min(first + 1, lastw));
        deposit(r0, min(first, lastw), 0, false);
        request(r0, min(first + 2, lastw));
        __syncthreads();
        for (int k = 0; k < share; k += 2) {
            const int kb = first + k;
            deposit(r1, min(kb + 1, lastw), 1, false);
            request(r1, min(kb + 3, lastw));
            if (kb < e1) multiply(0);
            __syncthreads();
            deposit(r0, min(kb + 2, lastw), 0, false);
            request(r0, min(kb + 4, lastw));
            if (kb + 1 < e1) multiply(1);
            __syncthreads();
        }
    }
    const int slow = short_rows ? share : full < nb ? 1 : 0;
#pragma unroll 1
    for (int i = 0; i < slow; ++i) {
        const int kb = short_rows ? first + i : full;
        if (kb < end && kb >= first) {
            request_slow(r0, kb);
            deposit(r0, kb, 0, true);
        }
        __syncthreads();
        if (kb < end && kb >= first) multiply(0);
        __syncthreads();
    }
    if constexpr (KS > 1) {
        floatx4* join = reinterpret_cast<floatx4*>(lds_all);     // [KS - 1][4][256]
        if (group > 0)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                join[((group - 1) * 4 + g) * 256 + tid] = floatx4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int q = 1; q < KS; ++q)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[v] += join[((q - 1) * 4 + (v >> 2)) * 256 + tid][v & 3];
    }
    const int64_t m = m0 + wm + (lane & 31);
    if (m >= M) return;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int64_t n = n0 + wn + 8 * g + (lane >> 5) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= N) continue;
            if (slices > 1) part[((int64_t)slice * M + m) * N + n + e] = acc[4 * g + e];
            else put_y(c + m * ldc + n + e, acc[4 * g + e]);
        }
    }
}

// c = the sum of the slices, by ascending slice
template <class TC>
__global__ __launch_bounds__(256) void k_block_grad_join(int64_t M, int64_t N, int32_t slices, const float* __restrict__ part,
                                                         TC* __restrict__ c, int64_t ldc) {
    const int64_t i = blockIdx.x * 256ll + threadIdx.x;
    if (i >= M * N) return;
    float s = part[i];
    for (int p = 1; p < slices; ++p) s += part[p * M * N + i];
    put_y(c + (i / N) * ldc + i % N, s);
}

// ---- large gradients ---------------------------------------------------------------------------------
// Rows of whole chunks of 16 bytes, aligned, power-of-two scales: tile of 256 x 256, 4 wavefronts (2 x 2, one a SIMD,
// 128 x 128 each), 64 of the contraction a step, two LDS stages.
//   The rows of dy go straight from memory into the LDS.  dx: [m][k], the 16-byte chunk c of row m at c ^ (m & 7) ^ (m / 16 & 1),
//   read as it is; dw: [half][k][128 m], chunk c of row k at c ^ 4 (k & 3), read transposed.
//   The codes go through registers: a thread has 16 of a row, converted to bf16 with the row's one scale (exact), [k][n] with
//   chunk c of row k at c ^ 4 (k & 3), read transposed.  (Scales along the contraction are the reason for converting here: a
//   fragment has 8 rows.)
//   The 4 x 32 lanes of a transposed read are 4 rows of 32 bytes; the places above put 8 such pieces on all 64 banks,
//   and 16 rows of dx that are read together too.
// The codes are the A operand, so that a lane's results come in fours along a row of the output.
// dy may come as several bf16 parts that sum to it (`planes`, `plane` numbers apart): the contraction then runs over all.
// The loop is that of the large product: a quadrant of 16 products at a time, all else in their shadows.
// 4096 x 11008 x 4096 bf16, calls one after another: dx 282 to 289 us (1.28 to 1.31 PFLOP/s), dw 322 to 335 (its 180 MB of results and the
// transposed reads of both operands).  Under the profiler 315 and 369, the matrix unit busy for 60 and 49 % of the cycles.
constexpr int GT_STAGE = 65536, GT_LDS = 256 * (256 * 2 + 16) > 2 * GT_STAGE ? 256 * (256 * 2 + 16) : 2 * GT_STAGE;

template <bool TRANS, class TC>
__global__ __launch_bounds__(256) void k_block_grad_tiled(int64_t M, int64_t N, int64_t Kc, const bf16_t* __restrict__ a, int64_t lda,
                                                          int32_t planes, int64_t plane, BlockView b, int64_t brows, TC* __restrict__ c, int64_t ldc,
                                                          int32_t tiles_m, int32_t tiles_n) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wv & 1) * 128, wn = (wv >> 1) * 128;
    int tile_m, tile_n;
    tile_of_workgroup(tiles_m, tiles_n, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * 256, n0 = (int64_t)tile_n * 256;

    // requests of dy: 1 KB each, 8 a wavefront and step.  dx: 8 rows of 64; dw: 4 rows of one half of the wavefronts' columns
    const uint32_t lda2 = (uint32_t)lda * 2;
    const uint8_t* ab = reinterpret_cast<const uint8_t*>(TRANS ? a + m0 : a + m0 * lda);
    const int64_t arows = TRANS ? Kc : min(M - m0, (int64_t)256), acols = TRANS ? (M - m0 + 7) & ~7ll : Kc;   // (rows of whole chunks)
    const intx4 first = buffer_of(ab, 0);            // (in scalar registers)
    const uint64_t abase = ((uint64_t)(uint32_t)first[1] << 32) | (uint32_t)first[0];
    const uint32_t abytes = (uint32_t)__builtin_amdgcn_readfirstlane(
        (int)(TRANS ? 63u * lda2 + (uint32_t)min(acols, (int64_t)256) * 2 : (uint32_t)(arows - 1) * lda2 + (uint32_t)acols * 2));
    // dw: a lane's place (16 to a row) holds this chunk of the half's 16: 8 of each 128 columns
    const int tchunk = (lane & 15) ^ ((lane >> 4) << 2), tcol = ((tchunk >> 3) * 16 + (tchunk & 7)) * 8;
    // (dx: the place of a chunk also goes by bit 4 of the row, which is the request's)
    const uint32_t offa[2] = {TRANS ? (lane >> 4) * lda2 + tcol * 2 : (lane >> 3) * lda2 + (((lane & 7) ^ (lane >> 3)) << 4),
                              (lane >> 3) * lda2 + (((lane & 7) ^ (lane >> 3) ^ 1) << 4)};
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int steps = (int)(Kc >> 7) * 2;            // of one part, in pairs
    // step f of all parts: step f % steps of part f / steps (three at most)
    auto part_of = [&](int f) __attribute__((always_inline)) { return (f >= steps ? 1 : 0) + (f >= 2 * steps ? 1 : 0); };
    // request i (of 4) of this wavefront for half h of the wavefronts' rows (columns) of the tile, 64 each
    auto bring = [&](int f, int stage, auto h, int i) __attribute__((always_inline)) {
        const int p = part_of(f), kb = f - p * steps;
        // (the buffer begins with the part, dw: with the step's 64 rows, so that offsets stay small; all whole)
        const uint64_t at64 = abase + (uint64_t)p * (uint64_t)(plane * 2) + (TRANS ? (uint64_t)(uint32_t)kb * (uint64_t)(64u * lda2) : 0ull);
        const intx4 buf = {(int)(uint32_t)at64, (int)(uint32_t)(at64 >> 32) & 0xFFFF, (int)abytes, 0x00020000};
        if constexpr (TRANS) {
            const int at = wv * 4 + i;
            lds_request(buf, offa[0], (uint32_t)(4 * at) * lda2 + h.value * 128, lds0 + stage + h.value * 16384 + at * 1024);
        } else {
            const int at = (wv >> 1) * 16 + h.value * 8 + (wv & 1) * 4 + i;
            lds_request(buf, offa[(i >> 1) & 1], (uint32_t)kb * 128 + (uint32_t)(8 * at) * lda2, lds0 + stage + at * 1024);
        }
    };
    // codes: thread has chunk tid % 16 of rows tid / 16 + 16 u
    const int brow = tid >> 4, bchunk = tid & 15;
    const int64_t bcol = n0 + bchunk * 16;
    const uint32_t fb = (uint32_t)(min(bcol, N - 1) >> 7);
    const int nlast = ((int)min(N - n0, (int64_t)256) + 15) & ~15;
    // (a chunk past the row's end gives columns that are not stored: the row's last is taken)
    const uint32_t bld = (uint32_t)b.ld, boff = (uint32_t)min(bchunk * 16, nlast - 16);
    const intx4 bfirst = buffer_of(b.codes + n0, 0);
    typedef const __attribute__((address_space(1))) uint8_t* global_bytes;         // (of an address put together: not a flat access)
    const global_bytes bb = (global_bytes)(((uint64_t)(uint32_t)bfirst[1] << 32) | (uint32_t)bfirst[0]);
    // without scales a byte is read all the same (a branch around the load would wait for it) and not used
    const global_bytes sp = (global_bytes)(b.scales ? static_cast<const uint8_t*>(b.scales) : b.codes);
    const uint32_t srow = b.scales ? (uint32_t)b.srow : 0u, soff = b.scales ? fb * (uint32_t)b.sblk : 0u, each = b.shift ? 0u : srow;
    const int blast = (int)brows - 1;
    piece16 rb[4];
    uint32_t rs[4];
    auto request = [&](int step_of, int u) __attribute__((always_inline)) {
        // (rows past the last meet zeros of dy: the last one is read, of the last step that has any)
        const int kb = min(step_of, blast >> 6);
        const uint32_t r = (uint32_t)min(brow + 16 * u, blast - kb * 64);
        rb[u] = *(const __attribute__((address_space(1))) piece16*)(bb + (uint64_t)(uint32_t)kb * (uint64_t)(64u * bld) + (__umul24(r, bld) + boff));
        rs[u] = (sp + (uint64_t)(((uint32_t)kb * 64u) >> b.shift) * srow)[__umul24(r, each) + soff];
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
            const int chunk = (wm >> 7) * 8 + (j & 1) * 4 + (tn >> 3);
            fm[j][s][h] = read_transposed(lds + stage + (j >> 1) * 16384 + (tk + 4 * h + 16 * s) * 256 + ((chunk ^ ((tk & 3) << 2)) << 4) + (tn & 7) * 2);
        } else if (h == 0) {
            const piece16 v = *reinterpret_cast<const piece16*>(lds + stage + (mrow + 32 * j) * 128 + (((2 * s + (lane >> 5)) ^ (mrow & 7) ^ ((mrow >> 4) & 1)) << 4));
            fm[j][s][0] = piece8{v[0], v[1]};
            fm[j][s][1] = piece8{v[2], v[3]};
        }
    };
    auto mul = [&](int i, int j, int s) __attribute__((always_inline)) {
        const piece16 n = {fn[i][s][0][0], fn[i][s][0][1], fn[i][s][1][0], fn[i][s][1][1]}, m = {fm[j][s][0][0], fm[j][s][0][1], fm[j][s][1][0], fm[j][s][1][1]};
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, n), __builtin_bit_cast(bf16x8_t, m), acc[i][j], 0, 0, 0);
    };
    const int paired = steps * planes, last = paired - 1, nb = (int)((Kc + 63) >> 6);
    // Products of half ih of the codes' tiles with half jh of dy's.  FM: the fragments for the next quadrant are of dy
    // (half fh, from the stage at fs), else of the codes.  Requests 2 r .. for half rh of dy's block `to` go to the stage at rs.
    // NEXT: the codes of a block (chunks 2 r ..; registers hold them already) go to the stage at rs, and those of block `then` are
    // requested.
    auto quad = [&](auto ih, auto jh, auto FM, int fs, auto fh, auto NEXT, auto r, auto rh, int to, int rs_, int then) __attribute__((always_inline)) {
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
                if ((slot & 7) == 1) bring(to, rs_, rh, r.value * 2 + (slot >> 3));
                if (NEXT.value) {
                    if ((slot & 7) == 2) deposit(rs_, r.value * 2 + (slot >> 3));
                    if ((slot & 7) == 6) request(then - part_of(then) * steps, r.value * 2 + (slot >> 3));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    // As in the large product: of block j's rows (columns) of dy those that are read first, half j & 1, are requested a half step
    // before the others, with a barrier in the middle and at the end of a step.
    auto step = [&](auto P, auto Q, int to, int then) __attribute__((always_inline)) {      // P: parity, Q = 1 - P; to: this step + 2
        constexpr int cur = P.value * GT_STAGE, nxt = Q.value * GT_STAGE;
        quad(C0, P, C1, cur, Q, C0, C0, P, min(to - 1, last), nxt, 0);
        quad(C0, Q, C0, cur, C1, C0, C1, P, min(to - 1, last), nxt, 0);
        lds_requests_left<4>();
        __syncthreads();
        quad(C1, Q, C0, nxt, C0, C1, C0, P, min(to, last), cur, then);
        quad(C1, P, C1, nxt, Q, C1, C1, P, min(to, last), cur, then);
        lds_requests_left<8>();                      // (12 have followed: 4 of dy, the codes and their scales)
        __syncthreads();
    };

    if (paired > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bring(0, 0, C0, i);
            bring(0, 0, C1, i);
            bring(1, GT_STAGE, C1, i);               // its other half follows in the first step
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (k > 0) deposit((k - 1) * GT_STAGE, u);
                request(min(k, last) - part_of(min(k, last)) * steps, u);
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
            step(C0, C1, kb + 2, min(kb + 3, last));
            step(C1, C0, kb + 3, min(kb + 4, last));
        }
        lds_requests_left<0>();
    }
    // what is left of the contraction of one part, at most one whole block and a shorter one (several are padded to whole pairs)
#pragma unroll 1
    for (int kb = steps; kb < nb; ++kb) {
        const int left = (int)(Kc - kb * 64ll);
        __syncthreads();
#pragma unroll 1
        for (int q = 0; q < 8; ++q) {
            const int at = wv * 8 + q;
            const int row = TRANS ? 4 * (at & 15) + (lane >> 4) : 8 * at + (lane >> 3);
            piece16 v = {0u, 0u, 0u, 0u};
            if constexpr (TRANS) {
                const int col = tcol + (at >> 4) * 64;
                if (row < left && m0 + col < M) v = *reinterpret_cast<const piece16*>(ab + ((int64_t)kb * 64 + row) * lda2 + col * 2);
            } else {
                const int col = ((lane & 7) ^ (row & 7) ^ ((row >> 4) & 1)) * 8;
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

// dy as PARTS bf16 parts that sum to it (32 bits, or bf16 times scales of 32 bits; two keep 16 bits, for results in bf16: what they cut off
// is under 2^-15 of sum |dy w|, where dy itself has been rounded to 2^-8 and dx will be, and a third part costs half as much again), or as
// it is, [Tp][Op] each with zeros in the margin.  A scale that is the same along a row of the block matrix belongs to
// a place of the contraction: BY 1, a column of dy (dx); BY 2, a row (dw).  Bound by memory at large sizes; 777 x 1365 6.6 us.
template <class T, int PARTS, int BY>
__global__ __launch_bounds__(256) void k_block_lay_gradient(int64_t rows, int64_t cols, const T* __restrict__ dy, int64_t ld, BlockView b,
                                                            uint16_t* __restrict__ out, int64_t Tp, int64_t Op) {
    const int64_t row = blockIdx.x * 4ll + (threadIdx.x >> 6), col = (blockIdx.y * 64ll + (threadIdx.x & 63)) * 8;
    if (col >= Op) return;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (row < rows && col < cols) load8(dy + row * ld, col, cols, v);
    if constexpr (BY != 0) {
        const float s = BY == 2 && row < rows ? scale_at(b, row, 0) : 1.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (BY == 1) v[e] = row < rows && col + e < cols ? v[e] * scale_at(b, col + e, 0) : 0.0f;
            else v[e] *= s;
        }
    }
    piece16 w[3];
    if constexpr (PARTS == 1) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) w[0][e >> 1] = bf16_bits(v[e]) | (bf16_bits(v[e + 1]) << 16);      // exact
    } else {
        split8<PARTS>(v, w);
    }
#pragma unroll
    for (int k = 0; k < PARTS; ++k) *reinterpret_cast<piece16*>(out + (PARTS - 1 - k) * Tp * Op + row * Op + col) = w[k];      // smallest first
}

// A strip of 512 columns and every gridDim.y-th group of 4 rows.  4096 x 11008 bf16: 14.7 us, 6.1 TB/s.
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

// Up to 2048 rows: one launch.  A workgroup takes 64 columns, its 16 wavefronts every 16th row each in 8 chains, joined in order.
// (777 x 1365 in 32 bits: one launch of 5 us instead of two of 4.8.)
constexpr int64_t BIAS_ROWS = 2048;
__device__ __forceinline__ float number(float v) { return v; }
__device__ __forceinline__ float number(bf16_t v) { return bf16_value(v.u); }
template <class T>
__global__ __launch_bounds__(1024) void k_block_bias(int64_t rows, int64_t cols, const T* __restrict__ dy, int64_t lddy, float* __restrict__ out) {
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t j = min(blockIdx.x * 64ll + lane, cols - 1);
    float c[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    int64_t r = w;
    for (; r + 112 < rows; r += 128)
#pragma unroll
        for (int u = 0; u < 8; ++u) c[u] += number(dy[(r + 16 * u) * lddy + j]);
#pragma unroll
    for (int u = 0; u < 8; ++u)
        if (r + 16 * u < rows) c[u] += number(dy[(r + 16 * u) * lddy + j]);
    float s = ((c[0] + c[1]) + (c[2] + c[3])) + ((c[4] + c[5]) + (c[6] + c[7]));
    sh[w][lane] = s;
    __syncthreads();
    if (w != 0 || blockIdx.x * 64ll + lane >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sh[i][lane];
    out[j] = s;
}

static int64_t bias_strips(int64_t T, int64_t O) {
    int64_t s = 1024 / ceil_div(O, 512);
    if (s < 1) s = 1;
    const int64_t most = ceil_div(T, 4);
    return most < s ? most : s;
}
// Slices of the contraction of a product of 64 x 64 tiles: where the tiles are fewer than the compute units (256), enough for
// all, with four steps of 64 for each of a workgroup's two groups.
static int32_t grad_slices(int64_t M, int64_t N, int64_t Kc) {
    const int64_t tiles = ceil_div(M, 64) * ceil_div(N, 64), most = Kc / 512;
    if (tiles <= 0 || tiles >= 256) return 1;
    int64_t s = 256 / tiles;
    if (s > most) s = most;
    return (int32_t)(s < 1 ? 1 : s);
}
static size_t grad_part_bytes(int64_t M, int64_t N, int64_t Kc) {
    const int32_t s = grad_slices(M, N, Kc);
    return s > 1 ? ((size_t)s * M * N * 4 + 255) / 256 * 256 : 0;
}
// Large tiles or small ones?  us by the rates measured: small tiles 260 TFLOP/s with one part and 145 with three products for
// one; large 1.4 us a step of 64 and round of 256 tiles, laying out 4 TB/s and two launches.  (All three gradients, small and
// large, us: 2048 x 2048 x 1024 bf16 69 and 90; 2048^3 in 32 bits 245 and 289; dx of 2048 x 4096 x 1024 with a scale
// per row 133 and 61; 4096^3 in 32 bits 2380 and 715.)
static bool large_tiles(int64_t M, int64_t N, int64_t Kc, int parts, double lay_bytes) {
    const double small = 2.0 * M * N * Kc / (parts == 1 ? 260e6 : 145e6);
    const int64_t rounds = ceil_div(ceil_div(M, 256) * ceil_div(N, 256), 256);
    const double large = 1.4 * rounds * parts * ceil_div(Kc, 64) + lay_bytes / 4e6 + (lay_bytes > 0 ? 10 : 0);
    return large < small;
}
static int64_t up(int64_t n, int64_t to) { return ceil_div(n, to) * to; }
// Small tiles of 32-bit gradients: dy laid out in parts first (once for dx and dw), or cut by every workgroup?  With a scale per row
// always, as the scales go into dy and three products are left of six (2707 x 975 x 671, dx: 47 us against 83).  Exponents:
// where the kernel's last step is a part of one (777 x 1365 x 1003: 55 us against 62; 1400 x 1403 x 1100 79 and 89; but 64^3 23
// and 20), or the product is large (1500 x 1024 x 1024 63 and 62, 1024^3 43 and 41).
static size_t lay_small_bytes(int64_t T, int64_t O) { return T >= 64 && O >= 64 ? (size_t)(3 * up(T, 128) * up(O, 128) * 2) : 0; }
static bool lay_small(int64_t T, int64_t O, int64_t K, bool exact) {
    const double work = (double)T * (double)O * (double)K;
    return lay_small_bytes(T, O) > 0 && (!exact || (work >= 5e7 && (T % 64 || O % 64)) || work >= 1.6e9);
}
// dy laid out (three parts at most), then the codes of w or x
static size_t lay_bytes(int64_t T, int64_t O, int64_t K) {
    const double lay = 2.0 * T * O;
    const bool dx = large_tiles(T, K, O, 1, lay), dw = large_tiles(O, K, T, 1, lay), dx3 = large_tiles(T, K, O, 3, lay), dw3 = large_tiles(O, K, T, 3, lay);
    if (!dx && !dw && !dx3 && !dw3) return 0;
    const int64_t rows = T > O ? T : O;
    return (size_t)((dx3 || dw3 ? 3 : 1) * up(T, 128) * up(O, 128) * 2) + (size_t)(rows * up(K, 16));
}
static size_t bias_bytes(int64_t T, int64_t O) { return T > 0 && O > 0 ? ((size_t)bias_strips(T, O) * O * 4 + 255) / 256 * 256 : 0; }
// Any call of these sizes; dx, dw and dbias use the same bytes one after the other
static size_t backward_workspace(int64_t T, int64_t O, int64_t K) {
    if (T <= 0 || O <= 0) return 0;
    size_t n = bias_bytes(T, O);
    const size_t small = lay_small_bytes(T, O), gx = small + grad_part_bytes(T, K, O), gw = small + grad_part_bytes(O, K, T), lay = K > 0 ? (lay_bytes(T, O, K) + 255) / 256 * 256 : 0;
    if (gx > n) n = gx;
    if (gw > n) n = gw;
    return lay > n ? lay : n;
}

// How a gradient is made, and the bytes that takes: what the call does and what its workspace is measured by.
struct GradPlan {
    enum Path { NOTHING, DIRECT, LAID, LAID_SMALL, GENERAL } path;
    bool exact, codes_aligned;           // scales that are powers of two; rows of whole aligned chunks
    int parts;                           // bf16 parts of dy
    size_t bytes;
};
// trans: dw [O][K] from x [T][K]; else dx [T][K] from w [O][K]
static GradPlan grad_plan(bool trans, int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t ld, const dmmv_block_matrix* b) {
    GradPlan p = {GradPlan::NOTHING, false, false, 1, 0};
    const int64_t M = trans ? O : T, Kc = trans ? T : O;
    if (M == 0 || K == 0) return p;
    const bool f32 = dtype == DMMV_F32, f32_result = f32 || trans;
    p.exact = !b->scales || b->scale_type == DMMV_E8M0;
    p.codes_aligned = K % 16 == 0 && b->ld % 16 == 0 && (uintptr_t)b->codes % 16 == 0 && b->ld < 1 << 23;
    // (offsets of 24 x 24 bits, of 32 bits along a row)
    const bool near = !b->scales || (b->scale_row_stride < 1 << 23 && b->scale_block_stride < 1 << 23 && ceil_div(K, 128) * b->scale_block_stride < 1 << 30);
    const bool dy_aligned = O % 8 == 0 && ld % 8 == 0 && ld < 1 << 22 && (uintptr_t)dy % 16 == 0;
    if (!f32 && p.exact && near && p.codes_aligned && dy_aligned && large_tiles(M, K, Kc, 1, 0.0)) {
        p.path = GradPlan::DIRECT;
        return p;
    }
    const bool rowwise = !p.exact && (b->scale_block_stride == 0 || K <= 128);
    p.parts = f32 ? 3 : p.exact ? 1 : f32_result ? 3 : 2;
    const int64_t Tp = up(T, 128), Op = up(O, 128);
    const bool fits = K < 1 << 22 && Op < 1 << 22 && Tp <= 1 << 25 && Kc > 0;
    if ((p.exact ? near : rowwise) && fits && large_tiles(M, K, Kc, p.parts, 2.0 * T * O) && large_tiles(M, K, Kc, p.parts == 1 ? 1 : 3, 2.0 * T * O)) {
        p.path = GradPlan::LAID;
        p.bytes = (size_t)p.parts * Tp * Op * 2 + (p.codes_aligned ? 0 : (size_t)Kc * up(K, 16));
    } else if (f32 && (p.exact || rowwise) && fits && lay_small(T, O, K, p.exact)) {
        p.path = GradPlan::LAID_SMALL;
        p.bytes = lay_small_bytes(T, O) + grad_part_bytes(M, K, Kc);
    } else {
        p.path = GradPlan::GENERAL;
        p.bytes = grad_part_bytes(M, K, Kc);
    }
    return p;
}
// a call with these arguments (checked)
static size_t backward_needs(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy, const dmmv_block_matrix* x,
                             const dmmv_block_matrix* w, bool dx, bool dw) {
    size_t n = bias_bytes(T, O);
    const size_t a = dx ? grad_plan(false, dtype, T, O, K, dy, lddy, w).bytes : 0, b = dw ? grad_plan(true, dtype, T, O, K, dy, lddy, x).bytes : 0;
    if (a > n) n = a;
    return b > n ? b : n;
}

template <class TA, bool TRANS, int PA, int PB, class TC>
static dmmv_status grad_any(int64_t M, int64_t N, int64_t Kc, const TA* a, int64_t lda, const BlockView& b, TC* c, int64_t ldc,
                            float* part, hipStream_t s, int64_t plane = 0) {
    const int64_t tiles_m = ceil_div(M, 64), tiles_n = ceil_div(N, 64);
    const int32_t slices = grad_slices(M, N, Kc);
    if (tiles_m > INT32_MAX / 4 / tiles_n) return fail(DMMV_ERR_SHAPE, "gradient: more tiles than a launch takes");
    auto launch = [&](auto groups) {
        constexpr int KS = decltype(groups)::value, bytes = KS * 2 * (PA + PB) * 8192;
        DMMV_TRY(ensure_dynamic_lds((const void*)k_block_grad<TA, TRANS, PA, PB, KS, TC>, bytes));
        hipLaunchKernelGGL((k_block_grad<TA, TRANS, PA, PB, KS, TC>), dim3((unsigned)(tiles_m * tiles_n * slices)), dim3(256 * KS), bytes, s, M, N,
                           Kc, a, lda, b, c, ldc, (int32_t)tiles_m, (int32_t)tiles_n, slices, part, plane);
        DMMV_LAUNCH_CHECK();
        return DMMV_OK;
    };
    // Two groups a workgroup (one workgroup a compute unit) where the tiles are no more than the compute units, else two
    // workgroups of one group (three parts, 396 tiles of 13 steps: 24.6 us against 35.5).
    if (PA + PB <= 4 && tiles_m * tiles_n <= 256) {
        if constexpr (PA + PB <= 4) DMMV_TRY(launch(std::integral_constant<int, 2>{}));
    } else {
        DMMV_TRY(launch(std::integral_constant<int, 1>{}));
    }
    if (slices > 1) {
        hipLaunchKernelGGL((k_block_grad_join<TC>), dim3((unsigned)ceil_div(M * N, 256)), dim3(256), 0, s, M, N, slices, part, c, ldc);
        DMMV_LAUNCH_CHECK();
    }
    return DMMV_OK;
}

template <bool TRANS, class TC>
static dmmv_status grad_tiled(int64_t M, int64_t N, int64_t Kc, const bf16_t* a, int64_t lda, int planes, int64_t plane, const BlockView& b,
                              int64_t brows, TC* c, int64_t ldc, hipStream_t s) {
    const int64_t tiles_m = ceil_div(M, 256), tiles_n = ceil_div(N, 256);
    if (tiles_m > INT32_MAX / 4 / tiles_n) return fail(DMMV_ERR_SHAPE, "gradient: more tiles than a launch takes");
    DMMV_TRY(ensure_dynamic_lds((const void*)k_block_grad_tiled<TRANS, TC>, GT_LDS));
    hipLaunchKernelGGL((k_block_grad_tiled<TRANS, TC>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), GT_LDS, s, M, N, Kc, a, lda, planes, plane, b,
                       brows, c, ldc, (int32_t)tiles_m, (int32_t)tiles_n);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class TA, int PARTS, int BY>
static dmmv_status lay_gradient(int64_t T, int64_t O, const TA* dy, int64_t ld, const BlockView& b, uint16_t* out, hipStream_t s) {
    const int64_t Tp = up(T, 128), Op = up(O, 128);
    hipLaunchKernelGGL((k_block_lay_gradient<TA, PARTS, BY>), dim3((unsigned)(Tp / 4), (unsigned)ceil_div(Op, 512)), dim3(256), 0, s, T, O, dy, ld, b, out, Tp, Op);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

// TRANS: c = dw [O][K] from x [T][K]; else dx [T][K] from w [O][K].  ws: the call's workspace; laid: dy lies there in PA parts
// without scales.
template <class TA, bool TRANS, class TC>
static dmmv_status grad(int64_t T, int64_t O, int64_t K, const TA* dy, int64_t ld, const dmmv_block_matrix* b, TC* c, int64_t ldc, char* ws,
                        bool* laid, hipStream_t s) {
    constexpr int PA = sizeof(TA) == 4 ? 3 : 1;
    const GradPlan plan = grad_plan(TRANS, PA == 3 ? DMMV_F32 : DMMV_BF16, T, O, K, dy, ld, b);
    const int64_t M = TRANS ? O : T, Kc = TRANS ? T : O, Tp = up(T, 128), Op = up(O, 128);
    uint16_t* lay = reinterpret_cast<uint16_t*>(ws);
    BlockView v = layer_view(b);
    // dy in parts, at the workspace's start; scales that are the same along a row go into it
    auto lay_out = [&]() {
        constexpr int BY = TRANS ? 2 : 1;
        if (plan.exact && *laid) return DMMV_OK;
        *laid = plan.exact;
        if (plan.exact) return lay_gradient<TA, PA, 0>(T, O, dy, ld, v, lay, s);
        BlockView by = v;
        v.scales = nullptr;
        if (plan.parts == 2) return lay_gradient<TA, 2, BY>(T, O, dy, ld, by, lay, s);
        return lay_gradient<TA, 3, BY>(T, O, dy, ld, by, lay, s);
    };
    switch (plan.path) {
    case GradPlan::NOTHING: return DMMV_OK;
    case GradPlan::DIRECT:
        if constexpr (PA == 1) return grad_tiled<TRANS, TC>(M, K, Kc, dy, ld, 1, 0, v, Kc, c, ldc, s);
        break;
    case GradPlan::LAID:
        DMMV_TRY(lay_out());
        if (!plan.codes_aligned) {
            const int64_t Kp = up(K, 16);
            uint8_t* to = reinterpret_cast<uint8_t*>(lay + (size_t)plan.parts * Tp * Op);
            DMMV_TRY(layer_lay_codes(b, to, Kp, s));
            v.codes = to;
            v.ld = Kp;
        }
        return grad_tiled<TRANS, TC>(M, K, TRANS ? Tp : Op, reinterpret_cast<const bf16_t*>(lay), Op, plan.parts, Tp * Op, v, Kc, c, ldc, s);
    case GradPlan::LAID_SMALL:
        if constexpr (PA == 3) {
            DMMV_TRY(lay_out());
            return grad_any<bf16_t, TRANS, 3, 1, TC>(M, K, Kc, reinterpret_cast<const bf16_t*>(lay), Op, v, c, ldc,
                                                     reinterpret_cast<float*>(ws + lay_small_bytes(T, O)), s, Tp * Op);
        }
        break;
    case GradPlan::GENERAL: break;
    }
    *laid = false;                                   // the slices go there
    float* part = reinterpret_cast<float*>(ws);
    return plan.exact ? grad_any<TA, TRANS, PA, 1, TC>(M, K, Kc, dy, ld, v, c, ldc, part, s)
                      : grad_any<TA, TRANS, PA, 3, TC>(M, K, Kc, dy, ld, v, c, ldc, part, s);
}

template <class T>
static dmmv_status backward(int64_t Tn, int64_t O, int64_t K, const T* dy, int64_t lddy, const dmmv_block_matrix* x,
                            const dmmv_block_matrix* w, T* dx, int64_t lddx, float* dw, int64_t lddw, float* dbias, void* ws, hipStream_t s) {
    bool laid = false;
    if (dx) DMMV_TRY((grad<T, false, T>(Tn, O, K, dy, lddy, w, dx, lddx, static_cast<char*>(ws), &laid, s)));
    if (dw) DMMV_TRY((grad<T, true, float>(Tn, O, K, dy, lddy, x, dw, lddw, static_cast<char*>(ws), &laid, s)));
    if (dbias && O > 0 && Tn <= BIAS_ROWS) {
        hipLaunchKernelGGL((k_block_bias<T>), dim3((unsigned)ceil_div(O, 64)), dim3(1024), 0, s, Tn, O, dy, lddy, dbias);
        DMMV_LAUNCH_CHECK();
    } else if (dbias && O > 0) {
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

static dmmv_status check_backward(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy, const dmmv_block_matrix* x,
                                  const dmmv_block_matrix* w, const void* dx, int64_t lddx, const float* dw, int64_t lddw) {
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
    return DMMV_OK;
}

extern "C" size_t dmmv_block_backward_workspace_for(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy, const dmmv_block_matrix* x,
                                                    const dmmv_block_matrix* w, const void* dx, const float* dw) {
    alignas(16) static const float wanted[4] = {};   // (any place will do for results that are asked for)
    dx = dx ? wanted : nullptr;
    dw = dw ? wanted : nullptr;
    if (check_backward(dtype, T, O, K, dy, lddy, x, w, dx, K, dw, K) != DMMV_OK) return 0;
    return backward_needs(dtype, T, O, K, dy, lddy, x, w, dx, dw);
}

extern "C" dmmv_status dmmv_block_backward(int32_t dtype, int64_t T, int64_t O, int64_t K, const void* dy, int64_t lddy,
                                           const dmmv_block_matrix* x, const dmmv_block_matrix* w, void* dx, int64_t lddx, float* dw,
                                           int64_t lddw, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(check_backward(dtype, T, O, K, dy, lddy, x, w, dx, lddx, dw, lddw));
    if ((uintptr_t)dbias % 4) return fail(DMMV_ERR_SHAPE, "dbias is not aligned to its elements");
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, backward_needs(dtype, T, O, K, dy, lddy, x, w, dx, dw)));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dtype == DMMV_F32)
        return backward(T, O, K, static_cast<const float*>(dy), lddy, x, w, static_cast<float*>(dx), lddx, dw, lddw, dbias, workspace, s);
    return backward(T, O, K, static_cast<const bf16_t*>(dy), lddy, x, w, static_cast<bf16_t*>(dx), lddx, dw, lddw, dbias, workspace, s);
}
