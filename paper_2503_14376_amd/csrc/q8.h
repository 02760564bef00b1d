// Numbers in 8 bits: e4m3 codes with one power of two per group of 128.  For a group with the largest finite magnitude A the exponent
// e is the least integer >= -127 with A <= 448 2^e; its scale is the byte e + 127 (e8m0) and a code is RNE(v 2^-e), which the
// conversion instruction rounds once, the scaling being exact.  Infinities and NaN become the code NaN.  The matrix unit takes
// these scales as they are (v_mfma_scale), so that a product needs no other instruction for them.
#pragma once
#include "tfla_device.h"

namespace tfla {

constexpr int Q8_GROUP = 128;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// magnitudes are compared as their bits; what is not finite does not count
__device__ __forceinline__ uint32_t q8_magnitude(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
// The largest of N: by their bits alone, and with the test of each only in a wavefront that holds one that is not finite (of four
// instructions a value two and a half are saved)
template <int N> __device__ __forceinline__ uint32_t q8_largest(const float (&v)[N]) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) most = max(most, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    if (__any(most >= 0x7f800000u)) {
        most = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) most = max(most, q8_magnitude(v[e]));
    }
    return most;
}
// scale byte of a group with that magnitude: 448 is 1.75 2^8 (subnormal magnitudes give 0 as they should)
__device__ __forceinline__ uint32_t q8_scale(uint32_t most) {
    const int b = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u);
    return (uint32_t)(b > 0 ? b : 0);
}
// 2^e as the conversions take it: of its bits they read the exponent alone, so that the byte 0 (2^-127) needs no denormal
__device__ __forceinline__ float q8_power(uint32_t scale) { return __builtin_bit_cast(float, scale << 23); }
// four values times 2^-e -> four codes
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, float power) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, power, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, power, true));
}
__device__ __forceinline__ u32x2 q8_codes8(const float (&v)[8], float power) {
    return u32x2{q8_codes(v[0], v[1], v[2], v[3], power), q8_codes(v[4], v[5], v[6], v[7], power)};
}
// the first n (0 .. 8) of eight codes to any address
__device__ __forceinline__ void q8_store8(uint8_t* p, const u32x2& w, int n) {
    if (n >= 8) __builtin_memcpy(p, &w, 8);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
    }
}

// Maximum over groups of N neighbouring lanes (N = 16 ... 64), in every lane: as lanes_sum.
template <int N> __device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    auto dpp = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl(), 0xf, 0xf, true); };
    struct A { __device__ constexpr int operator()() const { return 0xb1; } };
    struct B { __device__ constexpr int operator()() const { return 0x4e; } };
    struct C { __device__ constexpr int operator()() const { return 0x141; } };
    struct D { __device__ constexpr int operator()() const { return 0x140; } };
    x = max(x, dpp(x, A()));
    x = max(x, dpp(x, B()));
    x = max(x, dpp(x, C()));
    x = max(x, dpp(x, D()));
    if constexpr (N >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        const uint32_t lo = p[0], hi = p[1];
        x = max(lo, hi);
    }
    if constexpr (N >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const uint32_t lo = p[0], hi = p[1];
        x = max(lo, hi);
    }
    return x;
}

}  // namespace tfla
