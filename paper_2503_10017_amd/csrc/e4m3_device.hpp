// Device-side building blocks of matrices in 8 bits (fnn_scaled): e4m3 codes, four bits of exponent and three of mantissa, with a scale for each block of 128.
#pragma once
#include "net_device.hpp"
#include "net_kernels.hpp"

namespace fnn {

enum : int { CT_E4M3 = 3 };  // an element type of operands only
template <>
struct Elem<CT_E4M3> {
    typedef uint8_t T;
    static constexpr int N = 16;
};

// Maximum over LANES neighbouring lanes (16, 32 or 64), in each of them; a NaN loses against a number.
template <int LANES>
__device__ __forceinline__ float lanes_max(float x) {
    x = __builtin_fmaxf(x, dpp_move<0xB1>(x));
    x = __builtin_fmaxf(x, dpp_move<0x4E>(x));
    x = __builtin_fmaxf(x, dpp_move<0x141>(x));
    x = __builtin_fmaxf(x, dpp_move<0x140>(x));
    if constexpr (LANES >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __builtin_fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
    if constexpr (LANES >= 64) {
        const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __builtin_fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return x;
}
// Largest magnitude of N values; with FINITE, of those that are finite.
template <bool FINITE, int N>
__device__ __forceinline__ float top_of(const float (&v)[N]) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float m = __builtin_fabsf(v[e]);
        top = __builtin_fmaxf(top, !FINITE || m < __builtin_inff() ? m : 0.f);
    }
    return top;
}
// The largest finite magnitude of a block that LANES neighbouring lanes hold: with the infinities first, which are rare.
template <int LANES, int N>
__device__ __forceinline__ float block_top(const float (&v)[N]) {
    float top = lanes_max<LANES>(top_of<false>(v));
    if (__any(top == __builtin_inff())) top = lanes_max<LANES>(top_of<true>(v));
    return top;
}

// The scale that brings the largest magnitude to 448, e4m3's largest; never so small that its reciprocal would be infinite.
struct Scale {
    float scale, over;
    __device__ __forceinline__ explicit Scale(float top) : scale(__builtin_fmaxf(top / 448.f, 0x1p-126f)), over(1.f / scale) {}
};
// v / scale as a division rounds it, from the rounded reciprocal and one correction.  The product alone would be one step off now and then, and inputs of few
// digits lie on the border of two codes often enough (bf16 activations: one code in 10^5).
__device__ __forceinline__ float over_scale(float v, const Scale& s) {
    const float q = v * s.over;
    return __builtin_fmaf(__builtin_fmaf(-q, s.scale, v), s.over, q);
}
// Four values as codes, to nearest even; infinities and NaN as NaN.  Values that are themselves computed, and so off by some units in the last place, may do without the correction.
template <bool DIVIDED = true>
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, const Scale& s) {
    auto quotient = [&](float v) { return DIVIDED ? over_scale(v, s) : v * s.over; };
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(a), quotient(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient(c), quotient(d), low, true);
}
// N codes (4 or 8) to p, of which the first `count` exist.
template <int N, bool DIVIDED = true>
__device__ __forceinline__ void store_codes(uint8_t* p, int count, const float (&v)[N], const Scale& s) {
    uint32_t raw[N / 4];
#pragma unroll
    for (int e = 0; e < N; e += 4) raw[e / 4] = four_codes<DIVIDED>(v[e], v[e + 1], v[e + 2], v[e + 3], s);
    if (count >= N) {
        __builtin_memcpy(p, raw, N);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < count) p[e] = (uint8_t)(raw[e / 4] >> (8 * (e & 3)));
    }
}

}  // namespace fnn
