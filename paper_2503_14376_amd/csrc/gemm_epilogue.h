// What follows a matrix product of the residual block: bias, activation, residual, the gated product, and the derivative of
// the activation for the backward pass.  All of it in fp32 on the unrounded results; one rounding where a result is stored.
#pragma once
#include "block_internal.h"
#include "row8.h"

namespace tfla {

enum { ACT_NONE = 0, ACT_SILU = 1, ACT_GELU = 2, ACT_RELU = 3 };

// act(z) and act'(z).  silu: z sigma(z), sigma (1 + z (1 - sigma)); gelu: z Phi(z), Phi + z phi; relu: (z > 0).
// For bf16 tensors sigma comes from the hardware's exponential and reciprocal (2^-16 of its value at most, most of it the rounding of
// the exponent's argument; the result is rounded to 2^-8).  Phi(-|z|) = exp(-z^2 / 2) h(|z|), h falling from 1/2 as 1 / (|z| sqrt(2 pi)), so
// that a fit of h keeps Phi's digits also where it is small: h = t P(t), t = 1 / (1 + c |z|), c and the six coefficients fitted over |z| <= 14.5 (beyond,
// exp(-z^2 / 2) leaves fp32) to the smallest error against min(2^-12 of h, 2.5e-7 / Phi(-|z|)): 2^-13 of Phi(-|z|) and 1.2e-7 absolute.  (Formula 7.1.26 of
// Abramowitz and Stegun, one term shorter, is bounded absolutely only: 1 % of Phi at z = -8, 3.7 % at -13.)
// For fp32 both come from the library's functions (erfc, which keeps Phi's digits where it is small).
template <typename DT> __device__ __forceinline__ float sigmoid(float z);
template <> __device__ __forceinline__ float sigmoid<float>(float z) {
    const float e = expf(-fabsf(z));
    return (z >= 0.0f ? 1.0f : e) / (1.0f + e);
}
template <> __device__ __forceinline__ float sigmoid<bf16_t>(float z) {
    return __builtin_amdgcn_rcpf(1.0f + fast_exp2(-1.44269504f * z));
}
// Phi(z), and exp(-z^2 / 2)
template <typename DT> __device__ __forceinline__ float normal_cdf(float z, float& e);
template <> __device__ __forceinline__ float normal_cdf<float>(float z, float& e) {
    e = expf(-0.5f * z * z);
    return 0.5f * erfcf(z * -0.70710678f);
}
template <> __device__ __forceinline__ float normal_cdf<bf16_t>(float z, float& e) {
    e = fast_exp2(-0.72134752f * z * z);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.41907025f, fabsf(z), 1.0f));
    float p = __builtin_fmaf(t, 0.05759048f, -0.2349666f);
    p = __builtin_fmaf(t, p, 0.26108308f);
    p = __builtin_fmaf(t, p, 0.07074811f);
    p = __builtin_fmaf(t, p, 0.17915755f);
    p = __builtin_fmaf(t, p, 0.16638749f);
    const float h = t * p * e;
    return z < 0.0f ? h : 1.0f - h;
}
template <typename DT> __device__ __forceinline__ float act_value(float z, int act) {
    if (act == ACT_SILU) return z * sigmoid<DT>(z);
    if (act == ACT_GELU) {
        float e;
        return z * normal_cdf<DT>(z, e);
    }
    if (act == ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    return z;
}
// value and slope
template <typename DT> __device__ __forceinline__ float act_both(float z, int act, float& slope) {
    if (act == ACT_SILU) {
        const float g = sigmoid<DT>(z);
        slope = g * (1.0f + z * (1.0f - g));
        return z * g;
    }
    if (act == ACT_GELU) {
        float e;
        const float c = normal_cdf<DT>(z, e);
        slope = __builtin_fmaf(z * 0.39894228f, e, c);
        return z * c;
    }
    if (act == ACT_RELU) {
        slope = z > 0.0f ? 1.0f : 0.0f;
        return z > 0.0f ? z : (z != z ? z : 0.0f);
    }
    slope = 1.0f;
    return z;
}

// NG groups of eight columns, group i at row m + down(i), columns n + step(i) ...: the epilogue and the stores, part by part over
// all groups, so that the loads of a part are under way together.  v: the product (of the first matrix), w: of the second (EPI_GATED).  b: which
// result of a batch.  FULL: all of the row and the columns exist.
template <typename DT, int EPI, int NG, bool FULL, typename DOWN, typename STEP>
__device__ __forceinline__ void epilogue_groups(const GemmArgs& a, int b, long m, int n, DOWN down, STEP step, float (&v)[NG][8], float (&w)[NG][8],
                                                int width = 8) {
    auto at = [&](int i) { return (m + down(i)) * a.N + n + step(i); };
    auto left = [&](int i) { return FULL ? 8 : (m + down(i) < a.M ? min(width, a.N - n - step(i)) : 0); };
    auto add = [&](const float* bias, float (&x)[NG][8]) {
        Vec8<float> t[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) t[i] = load8<float>(bias, n + step(i), left(i));
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] += t[i].v[e];
    };
    auto put = [&](void* p, const float (&x)[NG][8]) {
#pragma unroll
        for (int i = 0; i < NG; ++i) store8<DT>(p, at(i), left(i), x[i]);
    };
    auto activate = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = act_value<DT>(v[i][e], kind());
    };
    struct Silu { __device__ constexpr int operator()() const { return ACT_SILU; } };
    struct Gelu { __device__ constexpr int operator()() const { return ACT_GELU; } };
    struct Relu { __device__ constexpr int operator()() const { return ACT_RELU; } };
    if constexpr (EPI != EPI_STORE) {
        Vec8<DT> r[NG];
        if (EPI == EPI_LINEAR && a.residual) {
#pragma unroll
            for (int i = 0; i < NG; ++i) r[i] = load8<DT>(a.residual, at(i), left(i));
        }
        if (a.bias[0]) add(a.bias[0], v);
        if (a.z[0]) put(a.z[0], v);
        if constexpr (EPI == EPI_GATED) {
            if (a.bias[1]) add(a.bias[1], w);
            if (a.z[1]) put(a.z[1], w);
        }
        if (a.act == ACT_SILU) activate(Silu());
        else if (a.act == ACT_GELU) activate(Gelu());
        else if (a.act == ACT_RELU) activate(Relu());
        if constexpr (EPI == EPI_GATED) {
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] *= w[i][e];
        } else if (a.residual) {
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                float t[8];
                r[i].get(t);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] += t[e];
            }
        }
    }
    put(a.out[EPI == EPI_STORE ? b : 0], v);
}
// one group
template <typename DT, int EPI> __device__ __forceinline__ void epilogue8(const GemmArgs& a, int b, long m, int n, float (&v)[8], float (&w)[8], int width = 8) {
    float v1[1][8], w1[1][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { v1[0][e] = v[e]; w1[0][e] = w[e]; }
    if (n < a.N) epilogue_groups<DT, EPI, 1, false>(a, b, m, n, [](int) { return 0; }, [](int) { return 0; }, v1, w1, width);
}
// where the partial results of one part of the contraction lie: plane (part, result) of M rows of ld_part values
__device__ __forceinline__ float* partial_plane(const GemmArgs& a, int planes, int part, int plane) {
    return a.part + ((long)part * planes + plane) * a.M * a.ld_part;
}

}  // namespace tfla
