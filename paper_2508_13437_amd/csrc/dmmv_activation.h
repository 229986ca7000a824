// The activations of a layer (include/dmmv_layer.h), on several numbers at a time: one uniform branch for all of them.
#pragma once

#include "dmmv_layer_common.h"

namespace dmmv {

dmmv_status layer_check_act(int32_t act, bool none);

#ifdef __HIPCC__

// 1 / (1 + e^-x) and 1 less that, neither from the other: e^-|x| <= 1.  Off by 1.3 |x| + 6 units of 2^-24 at most (the product with log2 e has one
// rounding, that constant 0.2; 65 units at 87), and 0 where e^-|x| is below 2^-126: the instruction has no smaller results.
struct Logistic {
    float s, rest;
};
__device__ __forceinline__ Logistic logistic(float x) {
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * -1.4426950408889634f), r = __builtin_amdgcn_rcpf(1.0f + e);
    return x < 0.0f ? Logistic{e * r, r} : Logistic{r, e * r};
}
// e^(-t^2 / 2) and the normal distribution's function at -t, t >= 0.  Their quotient falls slowly, from 1/2 as 1 / t: k times a polynomial in
// k = 1 / (1 + 0.3 t), of least largest relative error over 0 to 32 (2^-25; its sum in 32 bits 5.6 units of 2^-24, and 1/2 exactly at 0).
// The exponential's argument has two roundings and a constant's 0.2: 1.2 t^2 units more (128 measured at t = 13).
struct NormalTail {
    float e, q;
};
__device__ __forceinline__ NormalTail normal_tail(float t) {
    const float e = __builtin_amdgcn_exp2f(t * t * -0.72134752044448170f), k = __builtin_amdgcn_rcpf(dmmv_fma(0.3f, t, 1.0f));
    float p = -0.018033696338534355f;
    p = dmmv_fma(p, k, 0.0994100347161293f);
    p = dmmv_fma(p, k, -0.20012778043746948f);
    p = dmmv_fma(p, k, 0.15783672034740448f);
    p = dmmv_fma(p, k, -0.05417666584253311f);
    p = dmmv_fma(p, k, 0.08422795683145523f);
    p = dmmv_fma(p, k, 0.0819549635052681f);
    p = dmmv_fma(p, k, 0.10958808660507202f);
    p = dmmv_fma(p, k, 0.11963638663291931f);
    p = dmmv_fma(p, k, 0.11968399584293365f);
    return NormalTail{e, p * k * e};
}
constexpr float GELU_2C = 1.5957691216057308f, GELU_A = 0.044715f;       // 2 sqrt(2 / pi)

// 0 below every number that matters, so that -infinity gives act's limit there
__device__ __forceinline__ float above(float u, float least) { return __builtin_elementwise_maximum(u, least); }       // (NaN stays)

template <int ACT>
__device__ __forceinline__ float act_value(float u) {
    if constexpr (ACT == DMMV_ACT_RELU) return above(u, 0.0f);
    if constexpr (ACT == DMMV_ACT_GELU) {
        const float t = __builtin_elementwise_minimum(fabsf(u), 30.0f);
        return dmmv_fma(-t, normal_tail(t).q, above(u, 0.0f));           // u Phi(u) = max(u, 0) - |u| Phi(-|u|)
    }
    if constexpr (ACT == DMMV_ACT_GELU_TANH) {
        u = above(u, -30.0f);
        return u * logistic(GELU_2C * u * dmmv_fma(GELU_A * u, u, 1.0f)).s;
    }
    if constexpr (ACT == DMMV_ACT_SILU) {
        u = above(u, -128.0f);
        return u * logistic(u).s;
    }
    return u;
}

// The same for results of 8 significant bits, to a relative 2^-14: a third of the instructions, which are what an epilogue adds to a large
// product.  GELU is max(u, 0) - t Phi(-t) with t = |u|, and -log2 Phi(-t) is close to a parabola: a polynomial of degree 9 (least
// largest error over 0 to 13.3, 2^-15.5 of Phi; 2^-14.2 with its sums in 32 bits).  Beyond 13.3 Phi is below the type's numbers.
template <int ACT>
__device__ __forceinline__ float act_value_short(float u) {
    if constexpr (ACT == DMMV_ACT_GELU) {
        const float t = __builtin_elementwise_minimum(fabsf(u), 13.3f);
        float p = 1.8800052625778108e-09f;
        p = dmmv_fma(p, t, -1.3789509978323622e-07f);
        p = dmmv_fma(p, t, 4.445783815754112e-06f);
        p = dmmv_fma(p, t, -8.338923362316564e-05f);
        p = dmmv_fma(p, t, 0.0010188646847382188f);
        p = dmmv_fma(p, t, -0.008657238446176052f);
        p = dmmv_fma(p, t, 0.05393112078309059f);
        p = dmmv_fma(p, t, 0.4588252007961273f);
        p = dmmv_fma(p, t, 1.1509639024734497f);
        p = dmmv_fma(p, t, 1.000031590461731f);
        return dmmv_fma(-t, __builtin_amdgcn_exp2f(-p), above(u, 0.0f));
    }
    if constexpr (ACT == DMMV_ACT_GELU_TANH || ACT == DMMV_ACT_SILU) {
        constexpr float LOG2E = 1.4426950408889634f;
        u = above(u, ACT == DMMV_ACT_SILU ? -126.0f : -30.0f);
        const float x = ACT == DMMV_ACT_SILU ? -LOG2E * u : u * dmmv_fma(-LOG2E * GELU_2C * GELU_A * u, u, -LOG2E * GELU_2C);
        return u * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x));          // (beyond the range 1 / infinity)
    }
    return act_value<ACT>(u);
}
// the derivative; at infinities its limit
template <int ACT>
__device__ __forceinline__ float act_slope(float u) {
    if constexpr (ACT == DMMV_ACT_RELU) return u != u ? u : u > 0.0f ? 1.0f : 0.0f;
    // beyond 30 the slopes of GELU are 0 and 1 (their rest is below e^-430), and the products below leave the range
    if constexpr (ACT == DMMV_ACT_GELU || ACT == DMMV_ACT_GELU_TANH) u = u > 30.0f ? 30.0f : u < -30.0f ? -30.0f : u;
    if constexpr (ACT == DMMV_ACT_GELU) {
        const NormalTail n = normal_tail(fabsf(u));
        return dmmv_fma(u * 0.39894228040143268f, n.e, u < 0.0f ? n.q : 1.0f - n.q);
    }
    if constexpr (ACT == DMMV_ACT_GELU_TANH) {
        const Logistic l = logistic(GELU_2C * u * dmmv_fma(GELU_A * u, u, 1.0f));
        return dmmv_fma(u * GELU_2C * dmmv_fma(3.0f * GELU_A * u, u, 1.0f), l.s * l.rest, l.s);
    }
    // (the rest of the logistic is 0 in 32 bits beyond 104)
    u = u > 128.0f ? 128.0f : u < -128.0f ? -128.0f : u;
    const Logistic l = logistic(u);
    return dmmv_fma(u, l.s * l.rest, l.s);
}

template <bool SHORT, int M, int N>
__device__ __forceinline__ void act_values(int32_t act, float (&v)[M][N]) {
#define ACT_CASE(A)                                                                                                     \
    case A:                                                                                                             \
        _Pragma("unroll") for (int i = 0; i < M; ++i)                                                                   \
            _Pragma("unroll") for (int e = 0; e < N; ++e) v[i][e] = SHORT ? act_value_short<A>(v[i][e]) : act_value<A>(v[i][e]); \
        break;
    switch (act) {
        ACT_CASE(DMMV_ACT_RELU)
        ACT_CASE(DMMV_ACT_GELU)
        ACT_CASE(DMMV_ACT_GELU_TANH)
        ACT_CASE(DMMV_ACT_SILU)
    }
#undef ACT_CASE
}
template <bool SHORT, int N>
__device__ __forceinline__ void act_values(int32_t act, float (&v)[N]) { act_values<SHORT, 1, N>(act, reinterpret_cast<float (&)[1][N]>(v)); }

#endif  // __HIPCC__

}  // namespace dmmv
