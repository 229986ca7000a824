// Backward through an activation, with the gradient of the bias before it (include/dmmv_layer.h).
#include "dmmv_activation.h"

namespace dmmv {

dmmv_status layer_check_act(int32_t act, bool none) {
    if (act < (none ? DMMV_ACT_NONE : DMMV_ACT_RELU) || act > DMMV_ACT_SILU) return fail(DMMV_ERR_DOMAIN, "act %d is no activation", act);
    return DMMV_OK;
}

// du = dy act'(u): a lane 8 columns of every row of its strip, TPR lanes a row; the sums over the strip's rows of a column stay in the lane
// and are joined over the workgroup's rows in the LDS, in order.  Bound by memory: 4096 x 11008 bf16
// GELU 56 us (4.8 TB/s; 103 with the library's erfc and exp), and 5 for the sum of the parts.
template <class T, int ACT, int TPR>
__global__ __launch_bounds__(256) void k_activation_backward(int64_t rows, int64_t cols, int64_t per, uint32_t strips, const T* __restrict__ dy, int64_t lddy,
                                                             const T* __restrict__ u, int64_t ldu, T* __restrict__ du, int64_t lddu,
                                                             float* __restrict__ part) {
    constexpr int TEAMS = 256 / TPR;
    __shared__ float join[TEAMS > 1 ? 256 * 8 : 1];
    const int team = threadIdx.x / TPR, t = threadIdx.x % TPR;
    const uint32_t piece = blockIdx.x / strips, strip = blockIdx.x - piece * strips;
    const int64_t col = (piece * (int64_t)TPR + t) * 8;
    const int64_t r0 = strip * per, r1 = min(r0 + per, rows);
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (col < cols) {
        // two rows requested at a time
        Raw8<T> d[2], x[2];
        auto request = [&](int k, int64_t row) __attribute__((always_inline)) {
            const int64_t q = min(row, rows - 1);
            raw_request(d[k], dy + q * lddy, col, cols);
            raw_request(x[k], u + q * ldu, col, cols);
        };
        auto take = [&](int k, int64_t row) __attribute__((always_inline)) {
            if (row >= r1) return;
            raw_settle(d[k], col, cols, true);
            raw_settle(x[k], col, cols, true);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = d[k].get(e) * act_slope<ACT>(x[k].get(e));
                s[e] += v[e];
            }
            if (du) store8(du + row * lddu, col, cols, v);
        };
        request(0, r0 + team);
        for (int64_t row = r0 + team; row < r1; row += 2 * TEAMS) {
            request(1, row + TEAMS);
            take(0, row);
            request(0, row + 2 * TEAMS);
            take(1, row + TEAMS);
        }
    }
    if (!part) return;
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) join[(e * TEAMS + team) * TPR + t] = s[e];
        __syncthreads();
        if (team) return;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            for (int w = 1; w < TEAMS; ++w) s[e] += join[(e * TEAMS + w) * TPR + t];
    }
    if (col < cols) store8(part + strip * cols, col, cols, s);
}

// Strips of rows: some 1536 workgroups (4096 x 11008 bf16 64 us, 68 with 2048, 72 with 1024), a strip at least eight rounds of the workgroup's rows.
static int act_lanes(int64_t cols) { return cols <= 128 ? 16 : cols <= 512 ? 64 : 256; }
static int64_t act_rows(int64_t rows, int64_t cols) {
    const int64_t lanes = act_lanes(cols), teams = 256 / lanes, want = ceil_div(1536, ceil_div(cols, 8 * lanes));
    const int64_t per = ceil_div(rows, want), least = 8 * teams;
    return per > least ? per : least;
}
static size_t act_workspace(int64_t rows, int64_t cols) {
    return rows <= 0 || cols <= 0 ? 0 : (size_t)ceil_div(rows, act_rows(rows, cols)) * cols * 4;
}

template <class T>
static dmmv_status act_backward(int64_t rows, int64_t cols, const T* dy, int64_t lddy, const T* u, int64_t ldu, int32_t act, T* du, int64_t lddu,
                                float* dbias, float* part, hipStream_t s) {
    const int64_t per = act_rows(rows, cols), n = ceil_div(rows, per);
    const int lanes = act_lanes(cols);
    const dim3 grid((unsigned)(n * ceil_div(cols, 8 * lanes)));             // (at most some 1536 and 2^20)
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, rows, cols, per, (uint32_t)n, dy, lddy, u, ldu, du, lddu, dbias ? part : nullptr);
    };
#define ACT_LAUNCH(A)                                                        \
    case A:                                                                  \
        if (lanes == 16) launch(k_activation_backward<T, A, 16>);            \
        else if (lanes == 64) launch(k_activation_backward<T, A, 64>);       \
        else launch(k_activation_backward<T, A, 256>);                       \
        break;
    switch (act) {
        ACT_LAUNCH(DMMV_ACT_RELU)
        ACT_LAUNCH(DMMV_ACT_GELU)
        ACT_LAUNCH(DMMV_ACT_GELU_TANH)
        ACT_LAUNCH(DMMV_ACT_SILU)
    }
#undef ACT_LAUNCH
    DMMV_LAUNCH_CHECK();
    return dbias ? layer_sum_parts(part, n, cols, dbias, cols, nullptr, s) : DMMV_OK;
}

}  // namespace dmmv

using namespace dmmv;

extern "C" size_t dmmv_activation_workspace_bytes(int64_t rows, int64_t cols) {
    if (layer_check_sizes(rows, cols, "u") != DMMV_OK) return 0;
    return act_workspace(rows, cols);
}

extern "C" dmmv_status dmmv_activation_backward(int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* u, int64_t ldu, int32_t act,
                                                void* du, int64_t lddu, float* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
    DMMV_TRY(layer_check_dtype(dtype));
    DMMV_TRY(layer_check_sizes(rows, cols, "u"));
    DMMV_TRY(layer_check_act(act, false));
    const int w = layer_width(dtype);
    DMMV_TRY(layer_check_array(dy, rows, cols, lddy, w, "dy"));
    DMMV_TRY(layer_check_array(u, rows, cols, ldu, w, "u"));
    if (du) DMMV_TRY(layer_check_array(du, rows, cols, lddu, w, "du"));
    DMMV_TRY(layer_check_vector(dbias, false, "dbias"));
    if (dbias && cols > 1 << 27) return fail(DMMV_ERR_SHAPE, "dbias: more than 2^27 columns");
    if (dbias) DMMV_TRY(layer_check_workspace(workspace, workspace_bytes, act_workspace(rows, cols)));
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (cols == 0 || (!du && !dbias)) return DMMV_OK;
    if (rows == 0) return dbias ? layer_sum_parts(nullptr, 0, cols, dbias, cols, nullptr, s) : DMMV_OK;      // sums over no rows
    float* part = static_cast<float*>(workspace);
    if (dtype == DMMV_F32)
        return act_backward(rows, cols, static_cast<const float*>(dy), lddy, static_cast<const float*>(u), ldu, act, static_cast<float*>(du), lddu, dbias, part, s);
    return act_backward(rows, cols, static_cast<const bf16_t*>(dy), lddy, static_cast<const bf16_t*>(u), ldu, act, static_cast<bf16_t*>(du), lddu, dbias, part, s);
}
