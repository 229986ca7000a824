// Layer norm, forward and backward (include/dmmv_layer.h).
//
// Both passes are bound by memory: some ten operations for each element that is read.  A team of
// threads (a wavefront, or a whole workgroup for long rows) holds its row in registers, so the row is
// read once and the variance is the sum of squared deviations from the mean, not a difference of sums.
// A lane has 8 consecutive columns of every chunk, 16 lanes a block of 128: the 8-bit results need no
// exchange but the block's maximum.  Rows beyond the registers are walked three times instead.
#include "dmmv_layer_common.h"

namespace dmmv {

// one array of a row that is there or not, and the 8-bit outputs
template <class T>
struct NormOut {
    T* y;
    int64_t ldy;
    BlockView q, xq;
    int32_t has_q, has_xq;
};

// sum over the TPR threads of a team, in every thread; `sh` [TPR / 64]
template <int TPR>
__device__ __forceinline__ float team_sum(float v, float* sh) {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        const int w = threadIdx.x >> 6;
        __syncthreads();                     // the last round's values have been read
        if ((threadIdx.x & 63) == 0) sh[w] = v;
        __syncthreads();
        v = sh[0];
#pragma unroll
        for (int i = 1; i < TPR / 64; ++i) v += sh[i];
    }
    return v;
}

template <class T>
__device__ __forceinline__ void put_q(const BlockView& q, int64_t row, int64_t col, int64_t cols, const float (&v)[8]) {
    const uint32_t b = scale_byte(row16_max(max8_bits(v)));
    if (col < cols) {
        store8_codes(q.codes + row * q.ld, col, cols, encode8(v, b));
        if ((threadIdx.x & 15) == 0) scale_put(q, row, col >> 7, b);
    }
}

// v = (x - mean) rstd gamma + beta of 8 columns, zero past the row's end
__device__ __forceinline__ void norm8(const float (&x)[8], int64_t col, int64_t cols, float mu, float rs,
                                      const float* __restrict__ gamma, const float* __restrict__ beta, float (&v)[8]) {
    float g[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { g[e] = 1.0f; b[e] = 0.0f; }
    if (gamma) load8(gamma, col, cols, g);
    if (beta) load8(beta, col, cols, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < cols ? dmmv_fma((x[e] - mu) * rs, g[e], b[e]) : 0.0f;
}

// TPR threads a row, CH chunks of 8 TPR columns in registers: a row is read once, the two sums and the results come from the
// registers.  A wavefront a row up to 1024 columns (sums by DPP alone, four rows a workgroup), then a workgroup a row.
// Bound by memory and by the wait for a row before its two sums, in which nothing is requested: 4096 x 4096 bf16, y alone 16.5 us (4.1 TB/s with
// everything read and written once), the 8-bit result alone 18.0 (2.8), y and xq 18.6 (4.5), the 8-bit result and xq 21.7 (3.1).
template <class T, int TPR, int CH>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_layernorm(int64_t rows, int64_t cols, const T* __restrict__ x, int64_t ldx,
                                                                     const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                     float eps, NormOut<T> o, float* __restrict__ mean,
                                                                     float* __restrict__ rstd) {
    __shared__ float sh[TPR / 64];
    constexpr int TEAMS = TPR < 256 ? 256 / TPR : 1;
    const int team = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t row = blockIdx.x * (int64_t)TEAMS + team;
    if (row >= rows) return;                 // whole wavefronts; with TPR > 64 there is one team and none leaves
    const T* xr = x + row * ldx;
    const float n = (float)cols;
    float v[CH][8], s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) load8(xr, (c * TPR + t) * 8ll, cols, v[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[c][e];
    const float mu = team_sum<TPR>(s, sh) / n;
    s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = (c * TPR + t) * 8ll + e < cols ? v[c][e] - mu : 0.0f;
            s = dmmv_fma(d, d, s);
        }
    const float rs = 1.0f / __builtin_sqrtf(team_sum<TPR>(s, sh) / n + eps);
    if (t == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = rs;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = (c * TPR + t) * 8ll;
        if (o.has_xq) put_q<T>(o.xq, row, col, cols, v[c]);
        float w[8];
        norm8(v[c], col, cols, mu, rs, gamma, beta, w);
        if (o.y) store8(o.y + row * o.ldy, col, cols, w);
        if (o.has_q) put_q<T>(o.q, row, col, cols, w);
    }
}

// Rows of any length: one workgroup, three walks over the row (the second and third find it in the L2).  1024 x 40000 bf16:
// y 46 us (3.6 TB/s of what has to move), y and xq 53 (3.8).
template <class T>
__global__ __launch_bounds__(1024) void k_layernorm_wide(int64_t rows, int64_t cols, const T* __restrict__ x, int64_t ldx,
                                                         const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                         NormOut<T> o, float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float sh[16];
    const int64_t row = blockIdx.x;
    const T* xr = x + row * ldx;
    const float n = (float)cols;
    float s = 0.0f;
    for (int64_t col = threadIdx.x * 8ll; col < cols; col += 8192) {
        float v[8];
        load8(xr, col, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e];
    }
    const float mu = team_sum<1024>(s, sh) / n;
    s = 0.0f;
    for (int64_t col = threadIdx.x * 8ll; col < cols; col += 8192) {
        float v[8];
        load8(xr, col, cols, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = col + e < cols ? v[e] - mu : 0.0f;
            s = dmmv_fma(d, d, s);
        }
    }
    const float rs = 1.0f / __builtin_sqrtf(team_sum<1024>(s, sh) / n + eps);
    if (threadIdx.x == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = rs;
    }
    for (int64_t c0 = 0; c0 < cols; c0 += 8192) {            // every lane stays for the blocks' maxima
        const int64_t col = c0 + threadIdx.x * 8ll;
        float v[8], w[8];
        load8(xr, col, cols, v);
        if (o.has_xq) put_q<T>(o.xq, row, col, cols, v);
        norm8(v, col, cols, mu, rs, gamma, beta, w);
        if (o.y) store8(o.y + row * o.ldy, col, cols, w);
        if (o.has_q) put_q<T>(o.q, row, col, cols, w);
    }
}

// ---- backward ---------------------------------------------------------------------------------
// the norm's input: a matrix, or its 8-bit checkpoint
template <class T, bool Q8>
struct NormIn {
    const T* x;
    int64_t ldx;
    BlockView q;
    __device__ __forceinline__ void get(int64_t row, int64_t col, int64_t cols, float (&v)[8]) const {
        if constexpr (Q8) {
            if (col < cols) {
                decode8(load8_codes(q.codes + row * q.ld, col, cols), scale_at(q, row, col >> 7), v);
                if (col + 8 > cols)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = col + e < cols ? v[e] : 0.0f;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.0f;
            }
        } else {
            load8(x + row * ldx, col, cols, v);
        }
    }
};

// eight numbers of the input as they are stored
template <class T, bool Q8>
struct RawIn {
    Raw8<T> x;
    __device__ __forceinline__ void request(const NormIn<T, Q8>& in, int64_t row, int64_t col, int64_t cols) {
        raw_request(x, in.x + row * in.ldx, col, cols);
    }
    __device__ __forceinline__ void get(const NormIn<T, Q8>&, int64_t, int64_t col, int64_t cols, float (&v)[8]) {
        raw_settle(x, col, cols, col < cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x.get(e);
    }
};
template <class T>
struct RawIn<T, true> {
    Raw8<uint8_t> x;
    uint32_t s;
    __device__ __forceinline__ void request(const NormIn<T, true>& in, int64_t row, int64_t col, int64_t cols) {
        raw_request(x, (const uint8_t*)in.q.codes + row * in.q.ld, col, cols);
        s = *scale_word(in.q, (row >> in.q.shift) * in.q.srow + (col >> 7) * in.q.sblk);
    }
    __device__ __forceinline__ void get(const NormIn<T, true>& in, int64_t row, int64_t col, int64_t cols, float (&v)[8]) {
        raw_settle(x, col, cols, col < cols);
        const uint32_t bits = word_bits(in.q, (row >> in.q.shift) * in.q.srow + (col >> 7) * in.q.sblk, s);
        decode8(x.v, scale_of(in.q, bits), v);
        if (col + 8 > cols)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = col + e < cols ? v[e] : 0.0f;
    }
};

// Rows of up to 8192 columns: a team of TPR threads holds a row (its a and h) in registers between the two sums and dx, and keeps
// its columns' share of dgamma and dbeta over all the rows it takes; the THREADS / TPR teams of a workgroup join theirs at the
// end, in order, in the LDS.  Everything is read once, and the next row is requested before this one's sums are waited for.
// Few workgroups (256 of 1024 threads) keep the parts few: 4096 x 4096 bf16 21.3 us (4.7 TB/s), from the checkpoint 22.6, then 3.9
// for the sum of the parts.
template <class T, bool Q8, int TPR, int THREADS>
__global__ __launch_bounds__(THREADS) void k_layernorm_grad(int64_t rows, int64_t cols, const T* __restrict__ dy, int64_t lddy, NormIn<T, Q8> in,
                                                            const float* __restrict__ gamma, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, T* __restrict__ dx, int64_t lddx,
                                                            float* __restrict__ part) {
    constexpr int TEAMS = THREADS / TPR, WAVES = TPR / 64;
    // (8 columns a thread: with 16 the registers of 1024 threads do not hold the next row as well)
    __shared__ float2 sh[2][TEAMS][WAVES];
    __shared__ float join[TPR * 8];
    const int team = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const float inv_n = 1.0f / (float)cols;
    const int64_t col = t * 8ll;
    float g[8], dg[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { g[e] = 1.0f; dg[e] = db[e] = 0.0f; }
    if (gamma) load8(gamma, col, cols, g);
    // the row after this one is requested before this one's sums are waited for
    Raw8<T> nd;
    RawIn<T, Q8> nx;
    float nmu, nrs;
    auto request = [&](int64_t r0) __attribute__((always_inline)) {
        const int64_t row = min(r0 + team, rows - 1);
        nmu = mean[row];
        nrs = rstd[row];
        if (col >= cols) return;                     // (whole wavefronts but one)
        raw_request(nd, dy + row * lddy, col, cols);
        nx.request(in, row, col, cols);
    };
    request(blockIdx.x * (int64_t)TEAMS);
    int parity = 0;
    for (int64_t r0 = blockIdx.x * (int64_t)TEAMS; r0 < rows; r0 += gridDim.x * (int64_t)TEAMS, parity ^= 1) {
        const bool there = r0 + team < rows;
        const int64_t row = there ? r0 + team : rows - 1;
        const float mu = nmu, rs = nrs;
        float a[8], h[8];
        raw_settle(nd, col, cols, col < cols);
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = nd.get(e);
        nx.get(in, row, col, cols, h);
        request(r0 + gridDim.x * (int64_t)TEAMS);    // (past the last: the last again)
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = (h[e] - mu) * rs;
        // past the row's end dy is zero, and so is what follows from it, if h is not infinite
        if (col + 8 > cols)
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = col + e < cols ? h[e] : 0.0f;
        if (there)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = a[e];
                dg[e] = dmmv_fma(d, h[e], dg[e]);
                db[e] += d;
                a[e] = d * g[e];
                s1 += a[e];
                s2 = dmmv_fma(a[e], h[e], s2);
            }
        if (!dx) continue;
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (WAVES > 1) {
            // (two sets in turn: one barrier a row)
            if ((t & 63) == 0) sh[parity][team][t >> 6] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { s1 += sh[parity][team][w].x; s2 += sh[parity][team][w].y; }
        }
        s1 *= inv_n;
        s2 *= inv_n;
        if (!there) continue;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = rs * ((a[e] - s1) - h[e] * s2);
        if (col < cols) store8(dx + row * lddx, col, cols, w);
    }
    if (!part) return;
    float* p = part + blockIdx.x * 2ll * cols;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        float* v = b ? db : dg;
        for (int w = 1; w < TEAMS; ++w) {
            __syncthreads();
            if (team == w)
#pragma unroll
                for (int e = 0; e < 8; ++e) join[e * TPR + t] = v[e];
            __syncthreads();
            if (team == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += join[e * TPR + t];
        }
        if (team == 0 && col < cols) {
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = v[e];
            store8(p + b * cols, col, cols, o);
        }
    }
}

// ---- longer rows: the sums first, then strips of columns ------------------------------------------
// Sums of a row: s[row] = {sum a / n, sum a h / n}.  2048 x 16384 bf16: 14.8 us, 9 TB/s from the caches and memory.
template <class T, bool Q8>
__global__ __launch_bounds__(256) void k_layernorm_grad_sums(int64_t cols, const T* __restrict__ dy, int64_t lddy, NormIn<T, Q8> in,
                                                             const float* __restrict__ gamma, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, float2* __restrict__ sums) {
    __shared__ float sh[4];
    const int64_t row = blockIdx.x;
    const float mu = mean[row], rs = rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t col = threadIdx.x * 8ll; col < cols; col += 2048) {
        float d[8], v[8], g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        load8(dy + row * lddy, col, cols, d);
        in.get(row, col, cols, v);
        if (gamma) load8(gamma, col, cols, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = d[e] * g[e], h = col + e < cols ? (v[e] - mu) * rs : 0.0f;
            s1 += a;
            s2 = dmmv_fma(a, h, s2);
        }
    }
    s1 = team_sum<256>(s1, sh);
    s2 = team_sum<256>(s2, sh);
    if (threadIdx.x == 0) sums[row] = make_float2(s1 / (float)cols, s2 / (float)cols);
}

// A strip of 2048 columns and every gridDim.y-th row: dx and this workgroup's share of dgamma, dbeta.  The same size: 28.7 us,
// 7.0 TB/s, as dy and x are still in the chip's last cache.
template <class T, bool Q8>
__global__ __launch_bounds__(256) void k_layernorm_grad_apply(int64_t rows, int64_t cols, const T* __restrict__ dy, int64_t lddy,
                                                              NormIn<T, Q8> in, const float* __restrict__ gamma,
                                                              const float* __restrict__ mean, const float* __restrict__ rstd,
                                                              const float2* __restrict__ sums, T* __restrict__ dx, int64_t lddx,
                                                              float* __restrict__ part) {
    const int64_t col = (blockIdx.x * 256ll + threadIdx.x) * 8;
    if (col >= cols) return;
    float g[8] = {1, 1, 1, 1, 1, 1, 1, 1}, dg[8] = {}, db[8] = {};
    if (gamma) load8(gamma, col, cols, g);
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float mu = mean[row], rs = rstd[row];
        float d[8], v[8], w[8];
        load8(dy + row * lddy, col, cols, d);
        in.get(row, col, cols, v);
        float2 s = make_float2(0.0f, 0.0f);
        if (dx) s = sums[row];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float h = (v[e] - mu) * rs;
            w[e] = rs * ((d[e] * g[e] - s.x) - h * s.y);
            dg[e] = dmmv_fma(d[e], h, dg[e]);
            db[e] += d[e];
        }
        if (dx) store8(dx + row * lddx, col, cols, w);
    }
    if (part) {
        float* p = part + blockIdx.y * 2ll * cols;
        store8(p, col, cols, dg);
        store8(p + cols, col, cols, db);
    }
}

// ---- host ---------------------------------------------------------------------------------------
// Parts of the sums over rows.  Rows in registers: a workgroup of 1024 threads a compute unit; while those would have fewer than
// two rounds of rows, workgroups of 256 (or of a row, where it needs more), 512 at most.
constexpr int64_t NORM_REGS = 8192;
static int norm_team(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }
static bool norm_small(int64_t rows, int64_t cols) { return rows < 512 * (1024 / norm_team(cols)); }
static int64_t norm_strips(int64_t rows, int64_t cols) {
    if (cols <= NORM_REGS) {
        const int team = norm_team(cols), threads = norm_small(rows, cols) ? (team < 256 ? 256 : team) : 1024;
        const int64_t n = ceil_div(rows, threads / team), most = norm_small(rows, cols) ? 512 : 256;
        return n < most ? n : most;
    }
    int64_t s = 1024 / ceil_div(cols, 2048);
    if (s < 1) s = 1;
    return rows < s ? rows : s;
}
static size_t norm_workspace(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return 0;
    const size_t sums = cols <= NORM_REGS ? 0 : ((size_t)rows * 8 + 255) / 256 * 256;
    return sums + (size_t)norm_strips(rows, cols) * 2 * cols * 4;
}

template <class T>
static dmmv_status norm_forward(int64_t rows, int64_t cols, const T* x, int64_t ldx, const float* gamma, const float* beta,
                                float eps, const NormOut<T>& o, float* mean, float* rstd, hipStream_t stream) {
#define NORM_LAUNCH(TPR, CH)                                                                                         \
    hipLaunchKernelGGL((k_layernorm<T, TPR, CH>), dim3((unsigned)ceil_div(rows, TPR < 256 ? 256 / TPR : 1)),         \
                       dim3(TPR < 256 ? 256 : TPR), 0, stream, rows, cols, x, ldx, gamma, beta, eps, o, mean, rstd)
    if (cols <= 512) NORM_LAUNCH(64, 1);
    else if (cols <= 1024) NORM_LAUNCH(64, 2);
    else if (cols <= 2048) NORM_LAUNCH(256, 1);
    else if (cols <= 4096) NORM_LAUNCH(256, 2);
    else if (cols <= 8192) NORM_LAUNCH(256, 4);
    else if (cols <= 16384) NORM_LAUNCH(1024, 2);
    else
        hipLaunchKernelGGL((k_layernorm_wide<T>), dim3((unsigned)rows), dim3(1024), 0, stream, rows, cols, x, ldx, gamma, beta,
                           eps, o, mean, rstd);
#undef NORM_LAUNCH
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

template <class T, bool Q8>
static dmmv_status norm_backward(int64_t rows, int64_t cols, const T* dy, int64_t lddy, const NormIn<T, Q8>& in, const float* gamma,
                                 const float* mean, const float* rstd, T* dx, int64_t lddx, float* dgamma, float* dbeta,
                                 char* ws, hipStream_t stream) {
    if (cols <= NORM_REGS) {
        float* parts = reinterpret_cast<float*>(ws);
        float* to = dgamma || dbeta ? parts : nullptr;
        const int64_t n = norm_strips(rows, cols);
#define NORM_GRAD(TPR, THREADS)                                                                                                  \
    hipLaunchKernelGGL((k_layernorm_grad<T, Q8, TPR, THREADS>), dim3((unsigned)n), dim3(THREADS), 0, stream, rows, cols, dy, lddy, in, gamma, \
                       mean, rstd, dx, lddx, to)
        const bool small = norm_small(rows, cols);
        if (cols <= 512) { if (small) NORM_GRAD(64, 256); else NORM_GRAD(64, 1024); }
        else if (cols <= 1024) { if (small) NORM_GRAD(128, 256); else NORM_GRAD(128, 1024); }
        else if (cols <= 2048) { if (small) NORM_GRAD(256, 256); else NORM_GRAD(256, 1024); }
        else if (cols <= 4096) { if (small) NORM_GRAD(512, 512); else NORM_GRAD(512, 1024); }
        else NORM_GRAD(1024, 1024);
#undef NORM_GRAD
        DMMV_LAUNCH_CHECK();
        return to ? layer_sum_parts(parts, n, 2 * cols, dgamma, cols, dbeta, stream) : DMMV_OK;
    }
    float2* sums = reinterpret_cast<float2*>(ws);
    float* part = reinterpret_cast<float*>(ws + ((size_t)rows * 8 + 255) / 256 * 256);
    const int64_t strips = norm_strips(rows, cols);
    if (dx) {
        hipLaunchKernelGGL((k_layernorm_grad_sums<T, Q8>), dim3((unsigned)rows), dim3(256), 0, stream, cols, dy, lddy, in, gamma,
                           mean, rstd, sums);
        DMMV_LAUNCH_CHECK();
    }
    hipLaunchKernelGGL((k_layernorm_grad_apply<T, Q8>), dim3((unsigned)ceil_div(cols, 2048), (unsigned)strips), dim3(256), 0, stream,
                       rows, cols, dy, lddy, in, gamma, mean, rstd, sums, dx, lddx, dgamma || dbeta ? part : nullptr);
    DMMV_LAUNCH_CHECK();
    if (dgamma || dbeta) DMMV_TRY(layer_sum_parts(part, strips, 2 * cols, dgamma, cols, dbeta, stream));
    return DMMV_OK;
}

template <class T>
static dmmv_status norm_backward_of(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                    const dmmv_block_matrix* xq, const float* gamma, const float* mean, const float* rstd,
                                    void* dx, int64_t lddx, float* dgamma, float* dbeta, void* ws, hipStream_t s) {
    if (xq) {
        const NormIn<T, true> in{nullptr, 0, layer_view(xq)};
        return norm_backward<T, true>(rows, cols, static_cast<const T*>(dy), lddy, in, gamma, mean, rstd, static_cast<T*>(dx), lddx,
                                      dgamma, dbeta, static_cast<char*>(ws), s);
    }
    const NormIn<T, false> in{static_cast<const T*>(x), ldx, BlockView{}};
    return norm_backward<T, false>(rows, cols, static_cast<const T*>(dy), lddy, in, gamma, mean, rstd, static_cast<T*>(dx), lddx,
                                   dgamma, dbeta, static_cast<char*>(ws), s);
}

static dmmv_status check_vector(const float* p, bool needed, const char* what) {
    if (needed && !p) return fail(DMMV_ERR_NULL, "%s is NULL", what);
    if ((uintptr_t)p % 4) return fail(DMMV_ERR_SHAPE, "%s is not aligned to its elements", what);
    return DMMV_OK;
}

static dmmv_status check_out_block(const dmmv_block_matrix* q, int64_t rows, int64_t cols, const char* what) {
    DMMV_TRY(layer_check_block(q, true, what));
    if (q->rows != rows || q->cols != cols) return fail(DMMV_ERR_SHAPE, "%s is not %lld x %lld", what, (long long)rows, (long long)cols);
    if (q->scale_rows != 1) return fail(DMMV_ERR_UNSUPPORTED, "%s: a row's blocks have scales of their own (scale_rows 1)", what);
    return DMMV_OK;
}

}  // namespace dmmv

using namespace dmmv;

extern "C" dmmv_status dmmv_layernorm(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const float* gamma,
                                      const float* beta, float eps, void* y, int64_t ldy, const dmmv_block_matrix* q,
                                      const dmmv_block_matrix* xq, float* mean, float* rstd, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(rows, cols, "x"));
    if (!(eps >= 0.0f) || eps > 3.0e38f) return fail(DMMV_ERR_DOMAIN, "eps must be finite and not negative");
    const int w = layer_width(dtype);
    DMMV_TRY(layer_check_array(x, rows, cols, ldx, w, "x"));
    if (y) DMMV_TRY(layer_check_array(y, rows, cols, ldy, w, "y"));
    if (q) DMMV_TRY(check_out_block(q, rows, cols, "q"));
    if (xq) DMMV_TRY(check_out_block(xq, rows, cols, "xq"));
    DMMV_TRY(check_vector(gamma, false, "gamma"));
    DMMV_TRY(check_vector(beta, false, "beta"));
    DMMV_TRY(check_vector(mean, false, "mean"));
    DMMV_TRY(check_vector(rstd, false, "rstd"));
    if (rows == 0) return DMMV_OK;             // (rows without columns: mean and rstd are 0 / 0)
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (dtype == DMMV_F32) {
        const NormOut<float> o{static_cast<float*>(y), ldy, layer_view(q), layer_view(xq), q != nullptr, xq != nullptr};
        return norm_forward(rows, cols, static_cast<const float*>(x), ldx, gamma, beta, eps, o, mean, rstd, s);
    }
    const NormOut<bf16_t> o{static_cast<bf16_t*>(y), ldy, layer_view(q), layer_view(xq), q != nullptr, xq != nullptr};
    return norm_forward(rows, cols, static_cast<const bf16_t*>(x), ldx, gamma, beta, eps, o, mean, rstd, s);
}

extern "C" size_t dmmv_layernorm_workspace_bytes(int64_t rows, int64_t cols) {
    if (layer_check_sizes(rows, cols, "x") != DMMV_OK) return 0;
    return norm_workspace(rows, cols);
}

extern "C" dmmv_status dmmv_layernorm_backward(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* x,
                                               int64_t ldx, const dmmv_block_matrix* xq, const float* gamma, const float* mean,
                                               const float* rstd, void* dx, int64_t lddx, float* dgamma, float* dbeta,
                                               void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(rows, cols, "x"));
    const int w = layer_width(dtype);
    const bool empty = rows == 0 || cols == 0;
    if (x && xq) return fail(DMMV_ERR_NULL, "only one of x and xq can be given");
    if (!x && !xq && !empty) return fail(DMMV_ERR_NULL, "x and xq are both NULL");
    DMMV_TRY(layer_check_array(dy, rows, cols, lddy, w, "dy"));
    if (x) DMMV_TRY(layer_check_array(x, rows, cols, ldx, w, "x"));
    if (xq) {
        DMMV_TRY(layer_check_block(xq, false, "xq"));
        if (xq->rows != rows || xq->cols != cols)
            return fail(DMMV_ERR_SHAPE, "xq is not %lld x %lld", (long long)rows, (long long)cols);
    }
    if (dx) DMMV_TRY(layer_check_array(dx, rows, cols, lddx, w, "dx"));
    DMMV_TRY(check_vector(gamma, false, "gamma"));
    DMMV_TRY(check_vector(mean, !empty, "mean"));
    DMMV_TRY(check_vector(rstd, !empty, "rstd"));
    DMMV_TRY(check_vector(dgamma, false, "dgamma"));
    DMMV_TRY(check_vector(dbeta, false, "dbeta"));
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, norm_workspace(rows, cols)));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (cols == 0 || (!dx && !dgamma && !dbeta)) return DMMV_OK;
    if (rows == 0) return layer_sum_parts(nullptr, 0, 2 * cols, dgamma, cols, dbeta, s);     // sums over no rows
    if (dtype == DMMV_F32)
        return norm_backward_of<float>(rows, cols, dy, lddy, x, ldx, xq, gamma, mean, rstd, dx, lddx, dgamma, dbeta, workspace, s);
    return norm_backward_of<bf16_t>(rows, cols, dy, lddy, x, ldx, xq, gamma, mean, rstd, dx, lddx, dgamma, dbeta, workspace, s);
}
