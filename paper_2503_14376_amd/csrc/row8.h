// Eight consecutive elements of a row at any element address, as floats.  The compiler turns a copy of unknown alignment
// into one 16-byte access (the target runs with unaligned access enabled), so aligned rows lose nothing.
#pragma once
#include "tfla_device.h"

namespace tfla {

template <typename DT> struct Vec8;
template <> struct Vec8<bf16_t> {
    u32x4 w;
    __device__ __forceinline__ void zero() { w = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void load(const void* base, long idx) {
        __builtin_memcpy(&w, reinterpret_cast<const bf16_t*>(base) + idx, 16);
    }
    // the first n (0..8) elements, zeros behind them
    __device__ __forceinline__ void load_tail(const void* base, long idx, int n) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(base) + idx;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t lo = 2 * e < n ? p[2 * e] : 0u, hi = 2 * e + 1 < n ? p[2 * e + 1] : 0u;
            w[e] = lo | (hi << 16);
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = bf16_lo_to_f32(w[e]); x[2 * e + 1] = bf16_hi_to_f32(w[e]); }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
    }
    __device__ __forceinline__ void store(void* base, long idx) const {
        __builtin_memcpy(reinterpret_cast<bf16_t*>(base) + idx, &w, 16);
    }
    __device__ __forceinline__ void store_tail(void* base, long idx, int n) const {
        uint16_t* p = reinterpret_cast<uint16_t*>(base) + idx;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
};
template <> struct Vec8<float> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
    __device__ __forceinline__ void load(const void* base, long idx) {
        const float* p = reinterpret_cast<const float*>(base) + idx;
        f32x4 a, b;
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 4, 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    }
    __device__ __forceinline__ void load_tail(const void* base, long idx, int n) {
        const float* p = reinterpret_cast<const float*>(base) + idx;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.0f;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = v[e];
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[e];
    }
    __device__ __forceinline__ void store(void* base, long idx) const {
        float* p = reinterpret_cast<float*>(base) + idx;
        f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        __builtin_memcpy(p, &a, 16);
        __builtin_memcpy(p + 4, &b, 16);
    }
    __device__ __forceinline__ void store_tail(void* base, long idx, int n) const {
        float* p = reinterpret_cast<float*>(base) + idx;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = v[e];
    }
};

// the same with the number of elements that exist (n <= 0: none, n >= 8: all)
template <typename DT> __device__ __forceinline__ Vec8<DT> load8(const void* base, long idx, int n) {
    Vec8<DT> r;
    if (n >= 8) r.load(base, idx);
    else if (n > 0) r.load_tail(base, idx, n);
    else r.zero();
    return r;
}
template <typename DT> __device__ __forceinline__ void store8(void* base, long idx, int n, const float (&x)[8]) {
    Vec8<DT> r;
    r.set(x);
    if (n >= 8) r.store(base, idx);
    else if (n > 0) r.store_tail(base, idx, n);
}

}  // namespace tfla
