// What follows a matrix product of the residual block: bias, activation, residual, the gated product, and the derivative of
// the activation for the backward pass.  All of it in fp32 on the unrounded results; one rounding where a result is stored.
#pragma once
#include "block_internal.h"
#include "row8.h"

namespace tfla {

enum { ACT_NONE = 0, ACT_SILU = 1, ACT_GELU = 2, ACT_RELU = 3 };

// act(z) and act'(z).  silu: z sigma(z), sigma (1 + z (1 - sigma)); gelu: z Phi(z), Phi + z phi; relu: (z > 0).
__device__ __forceinline__ float sigmoid_f32(float z) {
    const float e = expf(-fabsf(z));
    return (z >= 0.0f ? 1.0f : e) / (1.0f + e);
}
__device__ __forceinline__ float act_value(float z, int act) {
    if (act == ACT_SILU) return z * sigmoid_f32(z);
    if (act == ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
    if (act == ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
    if (act == ACT_SILU) {
        const float g = sigmoid_f32(z);
        return g * (1.0f + z * (1.0f - g));
    }
    if (act == ACT_GELU) return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * expf(-0.5f * z * z) * 0.39894228f;
    if (act == ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    return 1.0f;
}

// Eight columns n, n + 1, ... of row m: the epilogue and the stores.  v: the product (of the first matrix), w: of the second
// (EPI_GATED).  b: which result of a batch.
template <typename DT, int EPI>
__device__ __forceinline__ void epilogue8(const GemmArgs& a, int b, long m, int n, float (&v)[8], float (&w)[8]) {
    if (m >= a.M || n >= a.N) return;
    const int left = a.N - n;
    const long at = m * a.N + n;
    if constexpr (EPI == EPI_STORE) {
        store8<DT>(a.out[b], at, left, v);
    } else if constexpr (EPI == EPI_LINEAR) {
        if (a.bias[0]) {
            float t[8];
            load8<float>(a.bias[0], n, left).get(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += t[e];
        }
        if (a.z[0]) store8<DT>(a.z[0], at, left, v);
        if (a.act != ACT_NONE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = act_value(v[e], a.act);
        }
        if (a.residual) {
            float t[8];
            load8<DT>(a.residual, at, left).get(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += t[e];
        }
        store8<DT>(a.out[0], at, left, v);
    } else if constexpr (EPI == EPI_GATED) {
        if (a.bias[0]) {
            float t[8];
            load8<float>(a.bias[0], n, left).get(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += t[e];
        }
        if (a.bias[1]) {
            float t[8];
            load8<float>(a.bias[1], n, left).get(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] += t[e];
        }
        if (a.z[0]) store8<DT>(a.z[0], at, left, v);
        if (a.z[1]) store8<DT>(a.z[1], at, left, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = act_value(v[e], a.act) * w[e];
        store8<DT>(a.out[0], at, left, v);
    }
}
// the partial results of one part of the contraction: plane (part, result) of M rows of ld_part values
__device__ __forceinline__ void partial8(const GemmArgs& a, int planes, int part, int plane, long m, int n, const float (&v)[8]) {
    if (m >= a.M || n >= a.N) return;
    float* p = a.part + (((long)part * planes + plane) * a.M + m) * a.ld_part + n;
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

}  // namespace tfla
