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

// Magnitudes are compared by their bits, which are ordered as they are, infinity and then the NaNs last: no value has to be brought into canonical form first.
enum : uint32_t { INFINITE = 0x7F800000u };
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t x, uint32_t y) { return x > y ? x : y; }

// Maximum over LANES neighbouring lanes (16, 32 or 64), in each of them.
template <int CONTROL>
__device__ __forceinline__ uint32_t larger_of(uint32_t x) { return larger(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xF, 0xF, true)); }
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    x = larger_of<0x140>(larger_of<0x141>(larger_of<0x4E>(larger_of<0xB1>(x))));
    if constexpr (LANES >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = larger(a[0], a[1]);
    }
    if constexpr (LANES >= 64) {
        const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = larger(b[0], b[1]);
    }
    return x;
}
// Largest magnitude of N values; with FINITE, of those that are finite.
template <bool FINITE, int N>
__device__ __forceinline__ uint32_t top_of(const float (&v)[N]) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const uint32_t m = magnitude(v[e]);
        top = larger(top, !FINITE || m < INFINITE ? m : 0u);
    }
    return top;
}
// The largest finite magnitude of a block that LANES neighbouring lanes hold: with what is not finite first, which is rare.
template <int LANES, int N>
__device__ __forceinline__ uint32_t block_top(const float (&v)[N]) {
    uint32_t top = lanes_max<LANES>(top_of<false>(v));
    if (__any(top >= INFINITE)) top = lanes_max<LANES>(top_of<true>(v));
    return top;
}

// The scale that brings the largest magnitude to 448, e4m3's largest; never so small that its reciprocal would be infinite.  top / 448 is what a division rounds it to for every fp32
// number (compared for all of them): the product with the rounded reciprocal, and one correction.
struct Scale {
    float scale, over;
    bool tiny;  // of any of the wave's lanes
    // DIVIDED: with the reciprocal that over_scale needs, rounded correctly; otherwise within a unit in its last place.
    template <bool DIVIDED>
    __device__ __forceinline__ static Scale of(uint32_t bits) {
        const float top = __uint_as_float(bits), near = top * (1.f / 448.f);
        const float scale = __builtin_fmaxf(__builtin_fmaf(__builtin_fmaf(-448.f, near, top), 1.f / 448.f, near), 0x1p-126f);
        return kept<DIVIDED>(scale, DIVIDED ? 1.f / scale : __builtin_amdgcn_rcpf(scale));
    }
    template <bool DIVIDED>
    __device__ __forceinline__ static Scale kept(float scale, float over) {
        return {scale, over, DIVIDED && __any(scale < 0x1p-100f)};
    }
};
// v / scale as a division rounds it, from the rounded reciprocal and one correction.  The product alone would be one step off now and then, and inputs of few
// digits lie on the border of two codes often enough (bf16 activations: one code in 10^5).
__device__ __forceinline__ float over_scale(float v, float scale, float over) {
    const float q = v * over;
    return __builtin_fmaf(__builtin_fmaf(-q, scale, v), over, q);
}
// Four values as codes, to nearest even; infinities and NaN as NaN.  Values that are themselves computed, and so off by some units in the last place, may do without the correction.
template <bool DIVIDED = true>
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, const Scale& s) {
    float v[4] = {a, b, c, d};
    if constexpr (DIVIDED) {
        if (__builtin_expect(s.tiny, 0)) {  // corrections that would be below fp32's range
            const bool here = s.scale < 0x1p-100f;
            const float up = here ? 0x1p64f : 1.f, down = here ? 0x1p-64f : 1.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = over_scale(v[e] * up, s.scale * up, s.over * down);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = over_scale(v[e], s.scale, s.over);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= s.over;
    }
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], low, true);
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
