// Device-side building blocks of the network's operators (fnn_net.h): element types, 16-byte accesses, sums over a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fnn_device.hpp"

namespace fnn {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// How an element is stored; N elements fill 16 bytes.  Everything is computed on fp32 values.
template <int DT>
struct Elem;
template <>
struct Elem<CT_F32> {
    typedef float T;
    static constexpr int N = 4;
};
template <>
struct Elem<CT_F16> {
    typedef _Float16 T;
    static constexpr int N = 8;
};
template <>
struct Elem<CT_BF16> {
    typedef __bf16 T;
    static constexpr int N = 8;
};

// N elements as fp32 from p, of which the first `count` exist (the rest are 0).  p need only be aligned to an element: global
// memory takes 16-byte accesses at any address, and rows of odd width or stride keep one load per 16 bytes that way.
template <int DT, int N = Elem<DT>::N>
__device__ __forceinline__ void load_elems(const typename Elem<DT>::T* p, int count, float (&v)[N]) {
    typename Elem<DT>::T raw[N];
    if (count >= N) {
        __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (float)raw[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = e < count ? (float)p[e] : 0.f;
    }
}
template <int DT, int N = Elem<DT>::N>
__device__ __forceinline__ void store_elems(typename Elem<DT>::T* p, int count, const float (&v)[N]) {
    if (count >= N) {
        typename Elem<DT>::T raw[N];
#pragma unroll
        for (int e = 0; e < N; ++e) raw[e] = (typename Elem<DT>::T)v[e];
        __builtin_memcpy(p, raw, sizeof(raw));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < count) p[e] = (typename Elem<DT>::T)v[e];
    }
}

// Sum over the 64 lanes of a wave, in every lane, always in the same order.
__device__ __forceinline__ float wave_sum(float x) {
    x += dpp_move<0xB1>(x);   // quad_perm [1,0,3,2]: lane ^ 1
    x += dpp_move<0x4E>(x);   // quad_perm [2,3,0,1]: lane ^ 2
    x += dpp_move<0x141>(x);  // row_half_mirror: joins the two quads of 8 lanes
    x += dpp_move<0x140>(x);  // row_mirror: joins the two halves of a 16-lane row
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace fnn
