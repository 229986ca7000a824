// The norms on both sides of a residual connection, its gate and scale, forward and backward (include/dmmv_layer.h).
//
//   p = post(f),  v = alpha h + gate p,  y = pre(v)
//
// As in the layer norm, a team of threads holds its row in registers, a lane 8 consecutive columns of every chunk: f and h are read once,
// v and y written once, and the norm of v is that of its 32-bit values.  Bound by memory, and by the wait for a row before its sums.
#include "dmmv_layer_common.h"

namespace dmmv {

// a norm as kernels take it
struct NormView {
    const float* gamma;
    const float* beta;
    float eps;
    int32_t kind;                        // 0 none, 1 layer norm, 2 RMS norm: no mean
};

static NormView norm_view(const dmmv_norm* n) { return n ? NormView{n->gamma, n->beta, n->eps, n->rms ? 2 : 1} : NormView{nullptr, nullptr, 0.0f, 0}; }

// a gate for every `per` rows, 1 without one
struct GateView {
    const float* g;
    int64_t ld;
    uint32_t per;
};

struct Stats {
    float mu, rs;
};

template <class T>
struct ResidualIn {
    const T* f;
    int64_t ldf;
    const T* h;
    int64_t ldh;
    float alpha;
    GateView gate;
    NormView post, pre;
};
template <class T>
struct ResidualOut {
    T* h;
    int64_t ldh;
    T* y;
    int64_t ldy;
    BlockView q;
    int32_t has_q;
    float *post_mean, *post_rstd, *mean, *rstd;
};

// (x - mean) rstd gamma + beta of 8 columns, zero past the row's end
__device__ __forceinline__ void norm8(const float (&x)[8], int64_t col, int64_t cols, Stats st, const NormView& n, float (&v)[8]) {
    float g[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { g[e] = 1.0f; b[e] = 0.0f; }
    if (n.gamma) load8(n.gamma, col, cols, g);
    if (n.beta) load8(n.beta, col, cols, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < cols ? dmmv_fma((x[e] - st.mu) * st.rs, g[e], b[e]) : 0.0f;
}

// v = alpha h + gate p of 8 columns, in the place of h; zero past the row's end
template <class T>
__device__ __forceinline__ void combine8(const ResidualIn<T>& in, int64_t col, int64_t cols, const float (&p)[8], const float (&gate)[8], float (&h)[8]) {
    if (in.gate.g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = col + e < cols ? dmmv_fma(gate[e], p[e], in.alpha * h[e]) : 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = col + e < cols ? dmmv_fma(in.alpha, h[e], p[e]) : 0.0f;
    }
}

__device__ __forceinline__ void put_stats(float* mean, float* rstd, int64_t row, Stats st) {
    if (mean) mean[row] = st.mu;
    if (rstd) rstd[row] = st.rs;
}

// Sum over the TPR threads of a team in every thread, by one barrier: the wavefronts' sums go to `sh` (a place that no wavefront still reads), in turn
// to the lanes, and a tree over them.
template <int TPR>
__device__ __forceinline__ float team_total(float v, float (&sh)[TPR / 64]) {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        constexpr int WAVES = TPR / 64;
        static_assert(WAVES <= 16, "sixteen lanes");
        const int t = threadIdx.x % TPR;
        if ((t & 63) == 0) sh[t >> 6] = v;
        __syncthreads();
        v = sh[t & (WAVES - 1)];
        v += dpp_mov<DPP_QUAD_XOR1>(v);
        if constexpr (WAVES > 2) v += dpp_mov<DPP_QUAD_XOR2>(v);
        if constexpr (WAVES > 4) v += dpp_mov<DPP_ROW_HALF_MIRROR>(v);
        if constexpr (WAVES > 8) v += dpp_mov<DPP_ROW_MIRROR>(v);
    }
    return v;
}

// mean (of a layer norm) and 1 / sqrt(sum of squared deviations / n + eps) of a row in registers
template <int TPR, int CH>
__device__ __forceinline__ Stats stats_of(const float (&v)[CH][8], int t, int64_t cols, const NormView& n, float (&sh)[2][TPR / 64]) {
    Stats st = {0.0f, 0.0f};
    const float len = (float)cols;
    float s = 0.0f;
    if (n.kind == 1) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[c][e];
        st.mu = team_total<TPR>(s, sh[0]) / len;
        s = 0.0f;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = (c * TPR + t) * 8ll + e < cols ? v[c][e] - st.mu : 0.0f;
            s = dmmv_fma(d, d, s);
        }
    st.rs = 1.0f / __builtin_sqrtf(team_total<TPR>(s, sh[1]) / len + n.eps);
    return st;
}

__device__ __forceinline__ void load_or(const float* __restrict__ p, float value, int64_t col, int64_t cols, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = value;
    if (p) load8(p, col, cols, v);
}
__device__ __forceinline__ void load_gate(const GateView& gate, int64_t row, int64_t col, int64_t cols, float (&g)[8]) {
    load_or(gate.g ? gate.g + ((uint32_t)row / gate.per) * gate.ld : nullptr, 1.0f, col, cols, g);
}

// TPR threads a row, CH chunks of 8 TPR columns in registers.  The gammas and the gate are requested with the row, so that no load waits for the sums
// (they come from the L2 for every row; a workgroup that kept them in registers over its rows had too few rows on their way: 31 us).  4096 x 4096
// bf16: both norms RMS and a gate 27.7 us (4.8 TB/s), without the norm after the block 22.3 (6.0), one row 3.6; in 32 bits 51 (5.3).
template <class T, int TPR, int CH>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void k_residual_norm(int64_t rows, int64_t cols, ResidualIn<T> in, ResidualOut<T> o) {
    __shared__ float sh[2][2][TPR / 64];
    constexpr int TEAMS = TPR == 64 ? 4 : 1;
    const int team = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const int64_t row = blockIdx.x * (int64_t)TEAMS + team;
    if (row >= rows) return;                 // whole wavefronts; with TPR > 64 there is one team and none leaves
    float f[CH][8], v[CH][8], g0[CH][8], gate[CH][8], g1[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) load8(in.f + row * in.ldf, (c * TPR + t) * 8ll, cols, f[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c) load8(in.h + row * in.ldh, (c * TPR + t) * 8ll, cols, v[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = (c * TPR + t) * 8ll;
        load_or(in.post.gamma, 1.0f, col, cols, g0[c]);
        load_gate(in.gate, row, col, cols, gate[c]);
        load_or(in.pre.gamma, 1.0f, col, cols, g1[c]);
    }
    Stats st = {0.0f, 0.0f};
    if (in.post.kind) {
        st = stats_of<TPR, CH>(f, t, cols, in.post, sh[0]);
        if (t == 0) put_stats(o.post_mean, o.post_rstd, row, st);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = (c * TPR + t) * 8ll;
        if (in.post.kind) {
            float b[8];
            load_or(in.post.beta, 0.0f, col, cols, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[c][e] = dmmv_fma((f[c][e] - st.mu) * st.rs, g0[c][e], b[e]);
        }
        combine8(in, col, cols, f[c], gate[c], v[c]);
        if (o.h) store8(o.h + row * o.ldh, col, cols, v[c]);
    }
    if (!in.pre.kind) return;
    st = stats_of<TPR, CH>(v, t, cols, in.pre, sh[1]);
    if (t == 0) put_stats(o.mean, o.rstd, row, st);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t col = (c * TPR + t) * 8ll;
        float b[8];
        load_or(in.pre.beta, 0.0f, col, cols, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = col + e < cols ? dmmv_fma((v[c][e] - st.mu) * st.rs, g1[c][e], b[e]) : 0.0f;
        if (o.y) store8(o.y + row * o.ldy, col, cols, v[c]);
        if (o.has_q) put_q<T>(o.q, row, col, cols, v[c]);
    }
}

// Rows of any length: one workgroup, a walk over the row for every sum and one for the results.  1024 x 40000 bf16, both norms RMS: 119 us (2.8 TB/s
// of what has to move; f and h come from the L2 or the chip's last cache for the later walks).
template <class T>
__global__ __launch_bounds__(1024) void k_residual_norm_wide(int64_t, int64_t cols, ResidualIn<T> in, ResidualOut<T> o) {
    __shared__ float sh[16];
    const int64_t row = blockIdx.x;
    const float len = (float)cols;
    Stats st = {0.0f, 0.0f}, sv = {0.0f, 0.0f};
    auto value = [&](int64_t col, float (&v)[8]) __attribute__((always_inline)) {
        float f[8], p[8], gate[8];
        load8(in.f + row * in.ldf, col, cols, f);
        load8(in.h + row * in.ldh, col, cols, v);
        load_gate(in.gate, row, col, cols, gate);
        if (!in.post.kind) {
            combine8(in, col, cols, f, gate, v);
            return;
        }
        norm8(f, col, cols, st, in.post, p);
        combine8(in, col, cols, p, gate, v);
    };
    auto walk = [&](const NormView& n, Stats& s, auto get) __attribute__((always_inline)) {
        float a = 0.0f;
        if (n.kind == 1) {
            for (int64_t col = threadIdx.x * 8ll; col < cols; col += 8192) {
                float v[8];
                get(col, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) a += v[e];
            }
            s.mu = team_sum<1024>(a, sh) / len;
            a = 0.0f;
        }
        for (int64_t col = threadIdx.x * 8ll; col < cols; col += 8192) {
            float v[8];
            get(col, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = col + e < cols ? v[e] - s.mu : 0.0f;
                a = dmmv_fma(d, d, a);
            }
        }
        s.rs = 1.0f / __builtin_sqrtf(team_sum<1024>(a, sh) / len + n.eps);
    };
    if (in.post.kind) {
        walk(in.post, st, [&](int64_t col, float (&v)[8]) { load8(in.f + row * in.ldf, col, cols, v); });
        if (threadIdx.x == 0) put_stats(o.post_mean, o.post_rstd, row, st);
    }
    if (in.pre.kind) {
        walk(in.pre, sv, value);
        if (threadIdx.x == 0) put_stats(o.mean, o.rstd, row, sv);
    }
    for (int64_t c0 = 0; c0 < cols; c0 += 8192) {            // every lane stays for the blocks' maxima
        const int64_t col = c0 + threadIdx.x * 8ll;
        float v[8], w[8];
        value(col, v);
        if (o.h) store8(o.h + row * o.ldh, col, cols, v);
        if (!in.pre.kind) continue;
        norm8(v, col, cols, sv, in.pre, w);
        if (o.y) store8(o.y + row * o.ldy, col, cols, w);
        if (o.has_q) put_q<T>(o.q, row, col, cols, w);
    }
}

// ---- backward ---------------------------------------------------------------------------------
//   n = (v - mean) rstd,  a = dy gamma,  e = dh + rstd (a - sum a / cols - n sum(a n) / cols)        [the sum of a: layer norm]
//   m = (f - post_mean) post_rstd,  p = m post_gamma + post_beta,  d = gate e,  b = d post_gamma
//   dh' = alpha e,  df = post_rstd (b - sum b / cols - m sum(b m) / cols)
//   dgamma = sum dy n,  dbeta = sum dy,  dgate = sum e p over the gate's rows,  dpost_gamma = sum d m,  dpost_beta = sum d
template <class T>
struct ResidualGrad {
    // what is not there points to something that is, and is not used
    const T *dy, *dv, *f, *v;
    int64_t lddy, lddv, ldf, ldv;
    int32_t has_dv, need_f;
    float alpha;
    GateView gate;
    NormView post, pre;
    const float *post_mean, *post_rstd, *mean, *rstd;
    T *df, *dh;
    int64_t lddf, lddh;
    float* dgate;                        // groups that a team has for itself are written where they belong
    int64_t lddgate;
    float* part;                         // [workgroup][4][cols]: GradSums, or where groups are not split the gates' products with the last two
    int32_t sums;                        // which of them are wanted, by bits
};

// Which rows a workgroup has.  split: `per` rows of one gate group, its teams in turn, and `each` workgroups a group; else every team has
// `per` rows, which are whole groups.
struct RowStrips {
    int64_t n, per, each;
    bool split;
};
struct TeamRows {
    int64_t at, end;
    int step;
};
__device__ __forceinline__ TeamRows team_rows(const RowStrips& s, int64_t rows, uint32_t gate_rows, int team, int teams) {
    if (s.split) {
        const uint32_t b = blockIdx.x, g = b / (uint32_t)s.each, i = b - g * (uint32_t)s.each;
        const int64_t g0 = (int64_t)g * gate_rows, g1 = min(g0 + gate_rows, rows), r0 = min(g0 + i * s.per, g1);
        return {r0 + team, min(r0 + s.per, g1), teams};
    }
    const int64_t r0 = min(((int64_t)blockIdx.x * teams + team) * s.per, rows);
    return {r0, min(r0 + s.per, rows), 1};
}

// What a column's sums over rows are made of:  sum dy n,  sum dy,  A = sum e m,  B = sum e.  Within a gate group, dgate = post_gamma A +
// post_beta B, and a group's share of dpost_gamma and dpost_beta is gate A and gate B.
struct GradSums {
    float dy_n[8], dy[8], e_m[8], e[8];
};
// a group of a team's own has ended: its gate's gradient, and what it adds to those of the norm after the block
template <class T>
__device__ __forceinline__ void end_group(const ResidualGrad<T>& a, int64_t row, int64_t col, int64_t cols, GradSums& s, float (&to_gamma)[8], float (&to_beta)[8]) {
    float g[8], b[8];
    if (a.dgate) {
        load_or(a.post.gamma, 1.0f, col, cols, g);
        load_or(a.post.beta, 0.0f, col, cols, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = dmmv_fma(g[e], s.e_m[e], b[e] * s.e[e]);
        store8(a.dgate + ((uint32_t)row / a.gate.per) * a.lddgate, col, cols, g);
    }
    load_gate(a.gate, row, col, cols, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        to_gamma[e] = dmmv_fma(g[e], s.e_m[e], to_gamma[e]);
        to_beta[e] = dmmv_fma(g[e], s.e[e], to_beta[e]);
        s.e_m[e] = s.e[e] = 0.0f;
    }
}
// gate post_gamma of a row
template <class T>
__device__ __forceinline__ void load_factor(const ResidualGrad<T>& a, int64_t row, int64_t col, int64_t cols, float (&f)[8]) {
    float g[8];
    load_gate(a.gate, row, col, cols, f);
    load_or(a.post.gamma, 1.0f, col, cols, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= g[e];
}

// Rows of up to 4096 columns (8192 in bf16): a team of TPR threads holds a row in registers between the two pairs of sums, and keeps its columns' share of the
// sums over rows; the teams of a workgroup join theirs at the end, in order, in the LDS.  Everything is read once, and the next row is requested before
// this one's sums are waited for.  SPLIT: a workgroup has rows of one gate group only.  BETAS: sum dy or sum e are wanted.
// Registers decide: with 128 two workgroups share a compute unit and one computes while the other waits for its sums (4096 x 4096 bf16, both norms RMS and a
// gate: 43 us, 4.7 TB/s; 65 with 187 registers).  The shares' way to memory and their join are 9 us of 51; both norms with betas 59.  2048 x 8192: 54 us.
template <class T, int TPR, int THREADS, bool SPLIT, bool BETAS>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 && SPLIT ? 4 : 2) void k_residual_norm_grad(int64_t rows, int32_t cols, ResidualGrad<T> a, RowStrips strips) {
    constexpr int TEAMS = THREADS / TPR, WAVES = TPR / 64;
    __shared__ float2 sh[2][2][TEAMS][WAVES];
    __shared__ float join[TEAMS > 1 ? TPR * 8 : 1];
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), t = threadIdx.x % TPR;
    const float inv_n = 1.0f / (float)cols;
    const int32_t col = t * 8;
    const bool in = col < cols;
    float g1[8], factor[8], to_gamma[SPLIT ? 1 : 8], to_beta[SPLIT ? 1 : 8];
    load_or(a.pre.gamma, 1.0f, col, cols, g1);
    GradSums sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sum.dy_n[e] = sum.dy[e] = sum.e_m[e] = sum.e[e] = 0.0f;
        if constexpr (!SPLIT) to_gamma[e] = to_beta[e] = 0.0f;
    }
    const TeamRows r = team_rows(strips, rows, a.gate.per, team, TEAMS);
    const int64_t last = rows - 1;
    int64_t row = r.at;
    load_factor(a, min(row, last), col, cols, factor);
    const int32_t passes = (int32_t)((strips.per + r.step - 1) / r.step);           // the same for all teams
    Raw8<T> rdy = {}, rdv = {}, rf = {}, rv = {};
    float nmu1 = 0.0f, nrs1 = 0.0f, nmu0 = 0.0f, nrs0 = 1.0f;
    auto request = [&](int64_t at) __attribute__((always_inline)) {
        const int64_t q = min(at, last);
        if (a.pre.kind) { nmu1 = a.pre.kind == 1 ? a.mean[q] : 0.0f; nrs1 = a.rstd[q]; }
        if (a.post.kind) { nmu0 = a.post.kind == 1 ? a.post_mean[q] : 0.0f; nrs0 = a.post_rstd[q]; }
        if (!in) return;                             // (whole wavefronts but one)
        raw_request(rdy, a.dy + q * a.lddy, col, cols);
        raw_request(rdv, a.dv + q * a.lddv, col, cols);
        raw_request(rf, a.f + q * a.ldf, col, cols);
        raw_request(rv, a.v + q * a.ldv, col, cols);
    };
    // sums over the row of two numbers; two sets in turn: one barrier
    auto both = [&](int set, int parity, float& s1, float& s2) __attribute__((always_inline)) {
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (WAVES > 1) {
            if ((t & 63) == 0) sh[set][parity][team][t >> 6] = make_float2(s1, s2);
            __syncthreads();
            // (the wavefronts' sums in turn over the lanes, and a tree over them)
            const float2 w = sh[set][parity][team][t & (WAVES - 1)];
            s1 = w.x + dpp_mov<DPP_QUAD_XOR1>(w.x);
            s2 = w.y + dpp_mov<DPP_QUAD_XOR1>(w.y);
            if constexpr (WAVES > 2) { s1 += dpp_mov<DPP_QUAD_XOR2>(s1); s2 += dpp_mov<DPP_QUAD_XOR2>(s2); }
            if constexpr (WAVES > 4) { s1 += dpp_mov<DPP_ROW_HALF_MIRROR>(s1); s2 += dpp_mov<DPP_ROW_HALF_MIRROR>(s2); }
            if constexpr (WAVES > 8) { s1 += dpp_mov<DPP_ROW_MIRROR>(s1); s2 += dpp_mov<DPP_ROW_MIRROR>(s2); }
            static_assert(WAVES <= 16, "sixteen lanes");
        }
        s1 *= inv_n;
        s2 *= inv_n;
    };
    request(row);
    int parity = 0;
    for (int32_t p = 0; p < passes; ++p, row += r.step, parity ^= 1) {
        const bool there = row < r.end;
        const float mu1 = nmu1, rs1 = nrs1, mu0 = nmu0, rs0 = nrs0;
        // this row as it is stored: numbers are made of it wherever they are used, which takes fewer registers than holding them
        raw_settle(rdy, col, cols, in && a.pre.kind);
        raw_settle(rdv, col, cols, in && a.has_dv);
        raw_settle(rf, col, cols, in && a.need_f);
        raw_settle(rv, col, cols, in && a.pre.kind);
        const Raw8<T> cdy = rdy, cdv = rdv, cf = rf, cv = rv;
        request(row + r.step);                       // (past the last: the last again)
        // past the row's end dy and dv are zero, and so is what follows from them, if the rest is finite
        const int32_t left = cols - col;
        auto n_of = [&](int e) __attribute__((always_inline)) { return e < left ? (cv.get(e) - mu1) * rs1 : 0.0f; };
        auto m_of = [&](int e) __attribute__((always_inline)) { return e < left ? (cf.get(e) - mu0) * rs0 : 0.0f; };
        float x[8];                                  // e
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = cdv.get(e);
        if (a.pre.kind) {
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float b = cdy.get(e) * g1[e];
                s1 += b;
                s2 = dmmv_fma(b, n_of(e), s2);
            }
            both(0, parity, s1, s2);
            if (a.pre.kind == 2) s1 = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float dy = cdy.get(e), n = n_of(e);
                if (there) {
                    sum.dy_n[e] = dmmv_fma(dy, n, sum.dy_n[e]);
                    if constexpr (BETAS) sum.dy[e] += dy;
                }
                x[e] = e < left ? dmmv_fma(rs1, (dy * g1[e] - s1) - n * s2, x[e]) : 0.0f;
            }
        }
        if (there)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum.e_m[e] = dmmv_fma(x[e], m_of(e), sum.e_m[e]);
                if constexpr (BETAS) sum.e[e] += x[e];
            }
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = x[e] * factor[e];
        if (a.post.kind) {
            float s3 = 0.0f, s4 = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s3 += d[e];
                s4 = dmmv_fma(d[e], m_of(e), s4);
            }
            both(1, parity, s3, s4);
            if (a.post.kind == 2) s3 = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = rs0 * ((d[e] - s3) - m_of(e) * s4);
        }
        if (there && in) {
            if (a.df) store8(a.df + row * a.lddf, col, cols, d);
            if (a.dh) {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = a.alpha * x[e];
                store8(a.dh + row * a.lddh, col, cols, d);
            }
        }
        if constexpr (!SPLIT)
            if (there && ((uint32_t)(row + 1) % a.gate.per == 0 || row == last)) {
                if (in) end_group(a, row, col, cols, sum, to_gamma, to_beta);
                if (row + 1 < r.end) load_factor(a, row + 1, col, cols, factor);
            }
    }
    if (!a.part) return;
    float* to = a.part + blockIdx.x * 4ll * cols;
    auto put = [&](int i, float (&v)[8]) __attribute__((always_inline)) {
        if constexpr (TEAMS > 1)
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
        if (team == 0 && in) store8(to + i * (int64_t)cols, col, cols, v);
    };
    if (a.sums & 1) put(0, sum.dy_n);
    if (a.sums & 2) put(1, sum.dy);
    if constexpr (SPLIT) {
        if (a.sums & 4) put(2, sum.e_m);
        if (a.sums & 8) put(3, sum.e);
    } else {
        if (a.sums & 4) put(2, to_gamma);
        if (a.sums & 8) put(3, to_beta);
    }
}

// ---- longer rows: the sums over the row first, then strips of columns ------------------------------
// s[row] = {sum a, sum a n, sum b, sum b m} / cols (the first and third 0 for RMS norms).  2048 x 16384 bf16, both norms RMS: 157 us with the
// next kernel and the join, which read everything once more from the chip's last cache; 78 if it were read once.
template <class T>
__global__ __launch_bounds__(256) void k_residual_norm_grad_sums(int64_t cols, ResidualGrad<T> a, floatx4* __restrict__ sums) {
    __shared__ float sh[4];
    const int64_t row = blockIdx.x;
    const float inv_n = 1.0f / (float)cols;
    const float mu1 = a.pre.kind == 1 ? a.mean[row] : 0.0f, rs1 = a.pre.kind ? a.rstd[row] : 0.0f;
    const float mu0 = a.post.kind == 1 ? a.post_mean[row] : 0.0f, rs0 = a.post.kind ? a.post_rstd[row] : 1.0f;
    floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.pre.kind) {
        for (int64_t col = threadIdx.x * 8ll; col < cols; col += 2048) {
            float d[8], v[8], g[8] = {1, 1, 1, 1, 1, 1, 1, 1};
            load8(a.dy + row * a.lddy, col, cols, d);
            load8(a.v + row * a.ldv, col, cols, v);
            if (a.pre.gamma) load8(a.pre.gamma, col, cols, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float b = d[e] * g[e], n = col + e < cols ? (v[e] - mu1) * rs1 : 0.0f;
                s[0] += b;
                s[1] = dmmv_fma(b, n, s[1]);
            }
        }
        s[0] = a.pre.kind == 1 ? team_sum<256>(s[0], sh) * inv_n : 0.0f;
        s[1] = team_sum<256>(s[1], sh) * inv_n;
    }
    if (a.post.kind) {
        for (int64_t col = threadIdx.x * 8ll; col < cols; col += 2048) {
            float x[8], y[8], g[8] = {1, 1, 1, 1, 1, 1, 1, 1}, e8[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (a.has_dv) load8(a.dv + row * a.lddv, col, cols, e8);
            if (a.pre.kind) {
                load8(a.dy + row * a.lddy, col, cols, x);
                load8(a.v + row * a.ldv, col, cols, y);
                if (a.pre.gamma) load8(a.pre.gamma, col, cols, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) e8[e] = dmmv_fma(rs1, (x[e] * g[e] - s[0]) - (y[e] - mu1) * rs1 * s[1], e8[e]);
            }
            load_gate(a.gate, row, col, cols, g);
            load8(a.f + row * a.ldf, col, cols, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = 1.0f;
            if (a.post.gamma) load8(a.post.gamma, col, cols, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = col + e < cols;
                const float b = in ? g[e] * e8[e] * y[e] : 0.0f, m = in ? (x[e] - mu0) * rs0 : 0.0f;
                s[2] += b;
                s[3] = dmmv_fma(b, m, s[3]);
            }
        }
        s[2] = a.post.kind == 1 ? team_sum<256>(s[2], sh) * inv_n : 0.0f;
        s[3] = team_sum<256>(s[3], sh) * inv_n;
    }
    if (threadIdx.x == 0) sums[row] = s;
}

// 2048 columns of a strip of rows, one team: the results and the share of the sums over rows
template <class T, bool SPLIT>
__global__ __launch_bounds__(256) void k_residual_norm_grad_apply(int64_t rows, int64_t cols, ResidualGrad<T> a, RowStrips strips,
                                                                  const floatx4* __restrict__ sums) {
    const int64_t col = (blockIdx.y * 256ll + threadIdx.x) * 8;
    if (col >= cols) return;
    float g1[8], factor[8], to_gamma[8], to_beta[8];
    load_or(a.pre.gamma, 1.0f, col, cols, g1);
    GradSums sum;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum.dy_n[e] = sum.dy[e] = sum.e_m[e] = sum.e[e] = to_gamma[e] = to_beta[e] = 0.0f;
    const TeamRows r = team_rows(strips, rows, a.gate.per, 0, 1);
    load_factor(a, min(r.at, rows - 1), col, cols, factor);
    for (int64_t row = r.at; row < r.end; ++row) {
        floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        if (sums) s = sums[row];
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0}, n[8] = {0, 0, 0, 0, 0, 0, 0, 0}, m[8] = {0, 0, 0, 0, 0, 0, 0, 0}, e8[8] = {0, 0, 0, 0, 0, 0, 0, 0}, d[8];
        if (a.has_dv) load8(a.dv + row * a.lddv, col, cols, e8);
        if (a.pre.kind) {
            const float mu1 = a.pre.kind == 1 ? a.mean[row] : 0.0f, rs1 = a.rstd[row];
            load8(a.dy + row * a.lddy, col, cols, x);
            load8(a.v + row * a.ldv, col, cols, n);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[e] = (n[e] - mu1) * rs1;
                sum.dy_n[e] = dmmv_fma(x[e], n[e], sum.dy_n[e]);
                sum.dy[e] += x[e];
                e8[e] = dmmv_fma(rs1, (x[e] * g1[e] - s[0]) - n[e] * s[1], e8[e]);
            }
        }
        const float mu0 = a.post.kind == 1 ? a.post_mean[row] : 0.0f, rs0 = a.post.kind ? a.post_rstd[row] : 1.0f;
        if (a.need_f) load8(a.f + row * a.ldf, col, cols, m);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = (m[e] - mu0) * rs0;
            sum.e_m[e] = dmmv_fma(e8[e], m[e], sum.e_m[e]);
            sum.e[e] += e8[e];
            d[e] = e8[e] * factor[e];
            if (a.post.kind) d[e] = rs0 * ((d[e] - s[2]) - m[e] * s[3]);
            e8[e] *= a.alpha;
        }
        if (a.df) store8(a.df + row * a.lddf, col, cols, d);
        if (a.dh) store8(a.dh + row * a.lddh, col, cols, e8);
        if constexpr (!SPLIT)
            if ((uint32_t)(row + 1) % a.gate.per == 0 || row == rows - 1) {
                end_group(a, row, col, cols, sum, to_gamma, to_beta);
                if (row + 1 < r.end) load_factor(a, row + 1, col, cols, factor);
            }
    }
    if (!a.part) return;
    float* to = a.part + blockIdx.x * 4ll * cols;
    if (a.sums & 1) store8(to, col, cols, sum.dy_n);
    if (a.sums & 2) store8(to + cols, col, cols, sum.dy);
    if (a.sums & 4) store8(to + 2 * cols, col, cols, SPLIT ? sum.e_m : to_gamma);
    if (a.sums & 8) store8(to + 3 * cols, col, cols, SPLIT ? sum.e : to_beta);
}

// Sums of the workgroups' shares: rows 0 to 3 of the grid the norms' parameters over all of them (those of the norm after the block times
// the gate of each share, where groups are split), row 4 + g the gate of group g over its `each`.  64 columns a workgroup, every 16th share a
// wavefront, joined in order.
struct ResidualSums {
    float* out[4];                       // dgamma, dbeta, dpost_gamma, dpost_beta
    float* dgate;
    int64_t lddgate;
    const float *gate, *post_gamma, *post_beta;
    int64_t ldgate;
};
__global__ __launch_bounds__(1024) void k_residual_norm_join(const float* __restrict__ part, int64_t n, int64_t each, int64_t cols, int32_t first, ResidualSums o) {
    __shared__ float sh[16][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, seg = first + (int)blockIdx.y;
    const int64_t j = blockIdx.x * 64ll + lane, g = seg - 4;
    float* out = seg < 4 ? o.out[seg] : o.dgate + g * o.lddgate;
    if (!out) return;                                // (the whole workgroup)
    const int64_t p0 = seg < 4 ? 0 : g * each, p1 = seg < 4 ? n : p0 + each;
    const float *A = part + (seg < 4 ? seg : 2) * cols + j, *B = part + 3 * cols + j;
    // (a single group's gate once, at the end)
    const bool gates = seg >= 2 && seg < 4 && o.gate && each > 0, gated = gates && n > each, both = seg >= 4 && o.post_beta;
    float ga = 1.0f, gb = 0.0f;
    if (gates && !gated && j < cols) ga = o.gate[j];
    if (seg >= 4 && j < cols) {
        if (o.post_gamma) ga = o.post_gamma[j];
        if (both) gb = o.post_beta[j];
    }
    float c[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](int u, int64_t p) __attribute__((always_inline)) {
        float v = A[p * 4 * cols];
        if (gated) v *= o.gate[((uint32_t)p / (uint32_t)each) * o.ldgate + j];
        if (both) v = dmmv_fma(ga, v, gb * B[p * 4 * cols]);
        c[u] += v;
    };
    if (j < cols) {
        int64_t p = p0 + w;
        for (; p + 112 < p1; p += 128)               // eight shares requested together, a chain of sums for each
#pragma unroll
            for (int u = 0; u < 8; ++u) add(u, p + 16 * u);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (p + 16 * u < p1) add(u, p + 16 * u);
    }
    float s = ((c[0] + c[1]) + (c[2] + c[3])) + ((c[4] + c[5]) + (c[6] + c[7]));
    sh[w][lane] = s;
    __syncthreads();
    if (w != 0 || j >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sh[i][lane];
    out[j] = both ? s : s * ga;
}

// ---- host ---------------------------------------------------------------------------------------
static bool residual_regs(int64_t cols, bool bf16) { return cols <= (bf16 ? 8192 : 4096); }
static int residual_team(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }

// Gradients: the threads of a workgroup (4096 x 4096 bf16: 51 us with 512 workgroups of 512, 52.6 with 256 of 1024, which have fewer shares to join
// but wait for one another).
static int residual_threads(int64_t cols) { return residual_team(cols) == 1024 ? 1024 : 512; }

// Rows per workgroup: some 256 of 1024 threads or 512 of fewer; groups that are longer are split, more than 1024 groups go to teams whole.
static RowStrips residual_strips(int64_t rows, int64_t cols, int64_t gate_rows, bool bf16) {
    const int64_t groups = ceil_div(rows, gate_rows);
    RowStrips s;
    s.split = groups <= 1024;
    const bool regs = residual_regs(cols, bf16);
    const int threads = residual_threads(cols);
    const int64_t want = regs ? (threads == 1024 ? 256 : 512) : (1024 / ceil_div(cols, 2048) > 1 ? 1024 / ceil_div(cols, 2048) : 1);
    const int64_t teams = regs ? threads / residual_team(cols) : 1;
    if (s.split) {
        int64_t each = want / groups, most = ceil_div(gate_rows, teams);
        if (each < 1) each = 1;
        if (each > most) each = most;
        s.per = ceil_div(gate_rows, each);
        s.each = ceil_div(gate_rows, s.per);
        s.n = groups * s.each;
    } else {
        s.per = ceil_div(groups, want * teams) * gate_rows;
        s.each = 0;
        s.n = ceil_div(rows, s.per * teams);
    }
    return s;
}
static size_t residual_sums_bytes(int64_t rows, int64_t cols, bool bf16) { return residual_regs(cols, bf16) ? 0 : ((size_t)rows * 16 + 255) / 256 * 256; }
static size_t residual_workspace_of(int64_t rows, int64_t cols, int64_t gate_rows, bool bf16) {
    return residual_sums_bytes(rows, cols, bf16) + (size_t)residual_strips(rows, cols, gate_rows, bf16).n * 4 * cols * 4;
}
static size_t residual_workspace(int64_t rows, int64_t cols, int64_t gate_rows) {
    if (rows <= 0 || cols <= 0) return 0;
    const size_t a = residual_workspace_of(rows, cols, gate_rows, false), b = residual_workspace_of(rows, cols, gate_rows, true);
    return a > b ? a : b;
}

static dmmv_status check_launch(int64_t groups, int threads) {
    return groups * threads <= UINT32_MAX ? DMMV_OK : fail(DMMV_ERR_SHAPE, "f: more rows than a launch takes");
}

template <class T>
static dmmv_status residual_forward(int64_t rows, int64_t cols, const ResidualIn<T>& in, const ResidualOut<T>& o, hipStream_t stream) {
    auto launch = [&](auto kernel, int threads, int64_t groups) -> dmmv_status {
        DMMV_TRY(check_launch(groups, threads));
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3((unsigned)threads), 0, stream, rows, cols, in, o);
        DMMV_LAUNCH_CHECK();
        return DMMV_OK;
    };
    // 8 columns a thread as long as a workgroup has 512: 4096 x 4096 bf16 with both norms and a gate 27.7 us, 30.7 with 256 threads of 16, the 8-bit
    // result alone 26.6 and 30.0; but 2048 x 8192 35 us with 1024 threads of 8, 29.6 with 512 of 16
    if (cols <= 512) return launch(k_residual_norm<T, 64, 1>, 256, ceil_div(rows, 4));
    if (cols <= 1024) return launch(k_residual_norm<T, 128, 1>, 128, rows);
    if (cols <= 2048) return launch(k_residual_norm<T, 256, 1>, 256, rows);
    if (cols <= 4096) return launch(k_residual_norm<T, 512, 1>, 512, rows);
    if (cols <= 8192) return launch(k_residual_norm<T, 512, 2>, 512, rows);
    if (cols <= 16384) return launch(k_residual_norm<T, 1024, 2>, 1024, rows);
    return launch(k_residual_norm_wide<T>, 1024, rows);
}

template <class T>
static dmmv_status residual_backward(int64_t rows, int64_t cols, ResidualGrad<T> a, const ResidualSums& o, char* ws, hipStream_t stream) {
    const int64_t groups = ceil_div(rows, (int64_t)a.gate.per);
    constexpr bool bf16 = sizeof(T) == 2;
    const RowStrips s = residual_strips(rows, cols, a.gate.per, bf16);
    a.sums = 0;
    for (int i = 0; i < 4; ++i) a.sums |= (o.out[i] ? 1 : 0) << i;
    const bool gates = s.split && o.dgate;           // gates' gradients by the join
    if (gates) a.sums |= o.post_beta ? 12 : 4;
    a.dgate = s.split ? nullptr : o.dgate;
    a.lddgate = o.lddgate;
    a.part = a.sums ? reinterpret_cast<float*>(ws + residual_sums_bytes(rows, cols, bf16)) : nullptr;
    if (residual_regs(cols, bf16)) {
        const bool betas = o.out[1] || o.out[3] || (o.dgate && o.post_beta);         // sums of dy or e are wanted
        auto launch = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)s.n), dim3((unsigned)threads), 0, stream, rows, (int32_t)cols, a, s);
        };
#define RESIDUAL_SPLIT(TPR, THREADS) \
    betas ? launch(k_residual_norm_grad<T, TPR, THREADS, true, true>, THREADS) : launch(k_residual_norm_grad<T, TPR, THREADS, true, false>, THREADS);
#define RESIDUAL_GRAD(TPR, THREADS)                                                              \
    if (s.split) RESIDUAL_SPLIT(TPR, THREADS)                                                    \
    else launch(k_residual_norm_grad<T, TPR, THREADS, false, true>, THREADS);
        if (cols <= 512) { RESIDUAL_GRAD(64, 512) }
        else if (cols <= 1024) { RESIDUAL_GRAD(128, 512) }
        else if (cols <= 2048) { RESIDUAL_GRAD(256, 512) }
        else if (cols <= 4096) { RESIDUAL_GRAD(512, 512) }
        else if constexpr (bf16) { RESIDUAL_GRAD(1024, 1024) }
#undef RESIDUAL_SPLIT
#undef RESIDUAL_GRAD
        DMMV_LAUNCH_CHECK();
    } else {
        DMMV_TRY(check_launch(rows, 256));
        if (cols > 65535 * 2048) return fail(DMMV_ERR_SHAPE, "f: longer rows than a launch takes");
        floatx4* sums = a.pre.kind || a.post.kind ? reinterpret_cast<floatx4*>(ws) : nullptr;
        if (sums) {
            hipLaunchKernelGGL((k_residual_norm_grad_sums<T>), dim3((unsigned)rows), dim3(256), 0, stream, cols, a, sums);
            DMMV_LAUNCH_CHECK();
        }
        auto kernel = s.split ? k_residual_norm_grad_apply<T, true> : k_residual_norm_grad_apply<T, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)s.n, (unsigned)ceil_div(cols, 2048)), dim3(256), 0, stream, rows, cols, a, s, sums);
        DMMV_LAUNCH_CHECK();
    }
    if (!a.sums) return DMMV_OK;
    const bool parameters = o.out[0] || o.out[1] || o.out[2] || o.out[3];
    const int first = parameters ? 0 : 4, rows_y = (gates ? 4 + (int)groups : 4) - first;
    hipLaunchKernelGGL(k_residual_norm_join, dim3((unsigned)ceil_div(cols, 64), (unsigned)rows_y), dim3(1024), 0, stream, a.part, s.n, s.each, cols, first, o);
    DMMV_LAUNCH_CHECK();
    return DMMV_OK;
}

static dmmv_status check_norm(const dmmv_norm* n, const char* what) {
    if (!n) return DMMV_OK;
    if (!(n->eps >= 0.0f) || n->eps > 3.0e38f) return fail(DMMV_ERR_DOMAIN, "%s: eps must be finite and not negative", what);
    if (n->rms != 0 && n->rms != 1) return fail(DMMV_ERR_DOMAIN, "%s: rms is not 0 or 1", what);
    DMMV_TRY(layer_check_vector(n->gamma, false, what));
    return layer_check_vector(n->beta, false, what);
}
static dmmv_status check_gate(int64_t rows, int64_t cols, int64_t gate_rows, const float* gate, int64_t ld, const char* what) {
    if (!gate) return DMMV_OK;
    if (gate_rows < 1) return fail(DMMV_ERR_SHAPE, "gate_rows is not positive");
    return layer_check_array(gate, rows ? ceil_div(rows, gate_rows) : 0, cols, ld, 4, what);
}
// rows of a gate group as kernels take them; without a gate there is one group
static uint32_t group_rows(int64_t rows, bool gated, int64_t gate_rows) {
    return (uint32_t)(!gated || gate_rows > rows ? (rows > 0 ? rows : 1) : gate_rows);
}

template <class T>
static dmmv_status residual_backward_of(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* dv, int64_t lddv, const void* f, int64_t ldf,
                                        const void* v, int64_t ldv, float alpha, const GateView& gate, const dmmv_norm* post, const dmmv_norm* pre,
                                        const float* post_mean, const float* post_rstd, const float* mean, const float* rstd, void* df, int64_t lddf,
                                        void* dh, int64_t lddh, const ResidualSums& o, void* ws, hipStream_t s) {
    ResidualGrad<T> a = {};
    const void* some = dv ? dv : dy;
    const int64_t ld = dv ? lddv : lddy;
    auto take = [&](const T*& to, int64_t& to_ld, const void* p, int64_t p_ld) {
        to = static_cast<const T*>(p ? p : some);
        to_ld = p ? p_ld : ld;
    };
    a.need_f = post || o.dgate;
    take(a.dy, a.lddy, pre ? dy : nullptr, lddy);
    take(a.dv, a.lddv, dv, lddv);
    take(a.f, a.ldf, a.need_f ? f : nullptr, ldf);
    take(a.v, a.ldv, pre ? v : nullptr, ldv);
    a.has_dv = dv != nullptr;
    a.alpha = alpha;
    a.gate = gate;
    a.post = norm_view(post);
    a.pre = norm_view(pre);
    a.post_mean = post_mean; a.post_rstd = post_rstd; a.mean = mean; a.rstd = rstd;
    a.df = static_cast<T*>(df);
    a.dh = static_cast<T*>(dh);
    a.lddf = lddf;
    a.lddh = lddh;
    return residual_backward<T>(rows, cols, a, o, static_cast<char*>(ws), s);
}

}  // namespace dmmv

using namespace dmmv;

extern "C" dmmv_status dmmv_residual_norm(int32_t dtype, int64_t rows, int64_t cols, const void* f, int64_t ldf, const void* h, int64_t ldh, float alpha,
                                          const float* gate, int64_t ldgate, int64_t gate_rows, const dmmv_norm* post, const dmmv_norm* pre, void* v,
                                          int64_t ldv, void* y, int64_t ldy, const dmmv_block_matrix* q, float* post_mean, float* post_rstd, float* mean,
                                          float* rstd, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(rows, cols, "f"));
    if (!(alpha >= -3.0e38f && alpha <= 3.0e38f)) return fail(DMMV_ERR_DOMAIN, "alpha must be finite");
    DMMV_TRY(check_norm(post, "post"));
    DMMV_TRY(check_norm(pre, "pre"));
    if (!pre && (y || q)) return fail(DMMV_ERR_NULL, "y and q need pre");
    const int w = layer_width(dtype);
    DMMV_TRY(layer_check_array(f, rows, cols, ldf, w, "f"));
    DMMV_TRY(layer_check_array(h, rows, cols, ldh, w, "h"));
    DMMV_TRY(check_gate(rows, cols, gate_rows, gate, ldgate, "gate"));
    if (v) DMMV_TRY(layer_check_array(v, rows, cols, ldv, w, "v"));
    if (y) DMMV_TRY(layer_check_array(y, rows, cols, ldy, w, "y"));
    if (q) DMMV_TRY(layer_check_out_block(q, rows, cols, "q"));
    for (const float* p : {post_mean, post_rstd, mean, rstd}) DMMV_TRY(layer_check_vector(p, false, "a statistic"));
    if (rows == 0) return DMMV_OK;             // (rows without columns: the statistics are 0 / 0)
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const GateView g = {gate, ldgate, group_rows(rows, gate != nullptr, gate_rows)};
    auto call = [&](auto* type) {
        using T = std::remove_pointer_t<decltype(type)>;
        const ResidualIn<T> in{static_cast<const T*>(f), ldf, static_cast<const T*>(h), ldh, alpha, g, norm_view(post), norm_view(pre)};
        const ResidualOut<T> o{static_cast<T*>(v), ldv, static_cast<T*>(y), ldy, layer_view(q), q != nullptr, post_mean, post_rstd, mean, rstd};
        return residual_forward<T>(rows, cols, in, o, s);
    };
    return dtype == DMMV_F32 ? call((float*)nullptr) : call((bf16_t*)nullptr);
}

extern "C" size_t dmmv_residual_norm_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows) {
    if (layer_check_sizes(rows, cols, "f") != DMMV_OK) return 0;
    return residual_workspace(rows, cols, group_rows(rows, gate_rows > 0, gate_rows));
}

extern "C" dmmv_status dmmv_residual_norm_backward(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* dv, int64_t lddv,
                                                   const void* f, int64_t ldf, const void* v, int64_t ldv, float alpha, const float* gate, int64_t ldgate,
                                                   int64_t gate_rows, const dmmv_norm* post, const dmmv_norm* pre, const float* post_mean,
                                                   const float* post_rstd, const float* mean, const float* rstd, void* df, int64_t lddf, void* dh,
                                                   int64_t lddh, float* dgate, int64_t lddgate, float* dpost_gamma, float* dpost_beta, float* dgamma,
                                                   float* dbeta, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(rows, cols, "f"));
    if (!(alpha >= -3.0e38f && alpha <= 3.0e38f)) return fail(DMMV_ERR_DOMAIN, "alpha must be finite");
    DMMV_TRY(check_norm(post, "post"));
    DMMV_TRY(check_norm(pre, "pre"));
    const bool empty = rows == 0 || cols == 0;
    if ((dy != nullptr) != (pre != nullptr) && !empty) return fail(DMMV_ERR_NULL, "dy comes with pre, and pre with dy");
    if (!dy && !dv && !empty) return fail(DMMV_ERR_NULL, "dy and dv are both NULL");
    if (dgate && !gate) return fail(DMMV_ERR_NULL, "dgate without gate");
    if ((dgamma || dbeta) && !pre) return fail(DMMV_ERR_NULL, "dgamma and dbeta need pre");
    if ((dpost_gamma || dpost_beta) && !post) return fail(DMMV_ERR_NULL, "dpost_gamma and dpost_beta need post");
    const int w = layer_width(dtype);
    if (dy) DMMV_TRY(layer_check_array(dy, rows, cols, lddy, w, "dy"));
    if (dv) DMMV_TRY(layer_check_array(dv, rows, cols, lddv, w, "dv"));
    if (post || dgate) DMMV_TRY(layer_check_array(f, rows, cols, ldf, w, "f"));
    if (pre) DMMV_TRY(layer_check_array(v, rows, cols, ldv, w, "v"));
    DMMV_TRY(check_gate(rows, cols, gate_rows, gate, ldgate, "gate"));
    if (post) {
        DMMV_TRY(layer_check_vector(post_mean, !empty && !post->rms, "post_mean"));
        DMMV_TRY(layer_check_vector(post_rstd, !empty, "post_rstd"));
    }
    if (pre) {
        DMMV_TRY(layer_check_vector(mean, !empty && !pre->rms, "mean"));
        DMMV_TRY(layer_check_vector(rstd, !empty, "rstd"));
    }
    if (df) DMMV_TRY(layer_check_array(df, rows, cols, lddf, w, "df"));
    if (dh) DMMV_TRY(layer_check_array(dh, rows, cols, lddh, w, "dh"));
    if (dgate) DMMV_TRY(check_gate(rows, cols, gate_rows, dgate, lddgate, "dgate"));
    for (const float* p : {dpost_gamma, dpost_beta, dgamma, dbeta}) DMMV_TRY(layer_check_vector(p, false, "a gradient"));
    const uint32_t per = group_rows(rows, gate != nullptr, gate_rows);
    DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, residual_workspace(rows, cols, per)));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const ResidualSums o = {{dgamma, dbeta, dpost_gamma, dpost_beta}, dgate, lddgate, gate, post ? post->gamma : nullptr, post ? post->beta : nullptr, ldgate};
    if (cols == 0 || (!df && !dh && !dgate && !dpost_gamma && !dpost_beta && !dgamma && !dbeta)) return DMMV_OK;
    if (rows == 0) {                           // sums over no rows; no gates
        hipLaunchKernelGGL(k_residual_norm_join, dim3((unsigned)ceil_div(cols, 64), 4), dim3(1024), 0, s, nullptr, (int64_t)0, (int64_t)0, cols, 0, o);
        DMMV_LAUNCH_CHECK();
        return DMMV_OK;
    }
    const GateView g = {gate, ldgate, per};
    return dtype == DMMV_F32 ? residual_backward_of<float>(rows, cols, dy, lddy, dv, lddv, f, ldf, v, ldv, alpha, g, post, pre, post_mean, post_rstd, mean, rstd,
                                                           df, lddf, dh, lddh, o, workspace, s)
                             : residual_backward_of<bf16_t>(rows, cols, dy, lddy, dv, lddv, f, ldf, v, ldv, alpha, g, post, pre, post_mean, post_rstd, mean, rstd,
                                                            df, lddf, dh, lddh, o, workspace, s);
}
