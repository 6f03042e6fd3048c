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

// Two values rounded to nearest even, as a vector: converted one by one, bf16 pairs take four instructions instead of one.
template <int DT>
__device__ __forceinline__ auto round_two(float a, float b) {
    typedef float two __attribute__((ext_vector_type(2)));
    typedef typename Elem<DT>::T pair __attribute__((ext_vector_type(2)));
    return __builtin_convertvector((two{a, b}), pair);
}

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
        for (int e = 0; e < N; e += 2) {
            const auto pair = round_two<DT>(v[e], v[e + 1]);
            raw[e] = pair[0];
            raw[e + 1] = pair[1];
        }
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

// ---- activations and their slopes ----
// 16-bit outputs take exp and the reciprocal from the hardware (2 units in the last place of fp32) and the normal tail from a fit of its own whose relative
// error is 1e-6 everywhere, since far to the left the tail is what GELU consists of; fp32 outputs take the library's functions.

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

template <bool FAST>
__device__ __forceinline__ float exp_of(float x) {
    if constexpr (FAST) return __builtin_amdgcn_exp2f(x * 1.44269504f);
    else return expf(x);
}
template <bool FAST>
__device__ __forceinline__ float over(float a, float b) {
    if constexpr (FAST) return a * __builtin_amdgcn_rcpf(b);
    else return a / b;
}
// Phi(-|x|), the integral of the normal density beyond |x|; exp(-x^2 / 2) comes along.  FAST: Phi(-x) exp(x^2 / 2) falls like 1 / x, and is a polynomial of
// t = 1 / (1 + 0.265 x) without a constant term.  Degree 7, its coefficients and the 0.265 are the least relative error over 0 <= x <= 14.4, where the
// exponential ends (linear programming over 1200 points): 6e-7, 9.6e-7 as computed; a step of fp16 is 1000 times that.
template <bool FAST>
__device__ __forceinline__ float normal_tail(float x, float& gauss) {
    if constexpr (FAST) {
        gauss = __builtin_amdgcn_exp2f(x * (x * -0.72134752f));
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(x), 0.265f, 1.f));
        float p = __builtin_fmaf(t, -0.06778702f, 0.19527303f);
        p = __builtin_fmaf(t, p, -0.06636281f);
        p = __builtin_fmaf(t, p, 0.14249325f);
        p = __builtin_fmaf(t, p, 0.08294662f);
        p = __builtin_fmaf(t, p, 0.10783678f);
        p = __builtin_fmaf(t, p, 0.10559984f);
        return p * t * gauss;
    } else {
        gauss = expf(-0.5f * x * x);
        return 0.5f * erfcf(0.70710678118654752f * __builtin_fabsf(x));
    }
}

// x = act(x), for N values; the choice is the same in every lane and made once.
template <bool FAST, int N>
__device__ __forceinline__ void activate(float (&x)[N], int act) {
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = x[e] < 0.f ? 0.f : x[e];
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            // x Phi(x) = max(x, 0) - |x| Phi(-|x|), whose second term is 0 long before |x| = 64 and must stay 0 at infinity
            float gauss;
            const float tail = normal_tail<FAST>(x[e], gauss);
            x[e] = __builtin_fmaf(-__builtin_fminf(__builtin_fabsf(x[e]), 64.f), tail, x[e] < 0.f ? 0.f : x[e]);
        }
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = over<FAST>(x[e], 1.f + exp_of<FAST>(-x[e]));
    }
}
// p *= act'(x)
template <bool FAST, int N>
__device__ __forceinline__ void times_slope(float (&p)[N], const float (&x)[N], int act) {
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = x[e] > 0.f ? p[e] : x[e] <= 0.f ? 0.f : x[e];  // a NaN stays one
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float gauss;
            const float tail = normal_tail<FAST>(x[e], gauss);
            p[e] *= __builtin_fmaf(x[e] * 0.39894228f, gauss, x[e] < 0.f ? tail : 1.f - tail);
        }
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float s = over<FAST>(1.f, 1.f + exp_of<FAST>(-x[e]));
            p[e] *= s * __builtin_fmaf(x[e], 1.f - s, 1.f);
        }
    }
}

// ---- matrix instructions: 32 x 32 results over a run of 16 bytes per lane, two lane halves ----
// mma32(a, b): result register v of lane (c = lane & 31, h = lane >> 5) belongs to row 8 (v / 4) + 4 h + v % 4 of a and row c of b.
template <int DT>
__device__ __forceinline__ f32x16 mma32(uint4 a, uint4 b, f32x16 acc) {
    if constexpr (DT == CT_F16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
    } else if constexpr (DT == CT_BF16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
    }
}
// The same for 16 x 16: lane (r = lane & 15, q = lane >> 4) holds 16 bytes of row r at run q; result register v belongs to row 4 q + v of a and
// row r of b.
template <int DT>
__device__ __forceinline__ f32x4 mma16(uint4 a, uint4 b, f32x4 acc) {
    if constexpr (DT == CT_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
    } else if constexpr (DT == CT_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
    }
}
// A lane's 16 results of mma32, rearranged: out[p] = the 8 consecutive rows 16 p + 8 h .. + 7 of a (p = 0, 1).
__device__ __forceinline__ void rows_of_eight(const f32x16& acc, float (&out)[2][8]) {
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[8 * p + e]), __float_as_uint(acc[8 * p + 4 + e]), false, false);
            out[p][e] = __uint_as_float(sw[0]);
            out[p][4 + e] = __uint_as_float(sw[1]);
        }
}

// 16 bytes from p, of which the first `count` elements exist; the rest are zero.  p as in load_elems.
template <int DT>
__device__ __forceinline__ uint4 load_run(const typename Elem<DT>::T* p, int count) {
    uint4 v = {0u, 0u, 0u, 0u};
    if (count >= Elem<DT>::N) {
        __builtin_memcpy(&v, p, 16);
    } else if (count > 0) {
        typename Elem<DT>::T raw[Elem<DT>::N];
#pragma unroll
        for (int e = 0; e < Elem<DT>::N; ++e) raw[e] = e < count ? p[e] : (typename Elem<DT>::T)0.f;
        __builtin_memcpy(&v, raw, 16);
    }
    return v;
}

// ---- direct loads from a buffer to LDS ----
// A buffer of `bytes` bytes from base (both the same in every lane): what lies behind it reads as zero.
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 buffer_of(const void* base, uint32_t bytes) {
    const uint64_t at = (uint64_t)base;
    i32x4 b;
    b[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)at);
    b[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xFFFF);
    b[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    b[3] = 0x00020000;
    return b;
}
__device__ __forceinline__ uint32_t lds_address(const char* lds) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds;
}
// 16 bytes per lane from `offset` in the buffer to LDS at `to` + 16 * lane (`to` the same in every lane).  Written in assembly because the compiler
// makes every later LDS read wait for a load to LDS that it knows of, whichever part of LDS it reads; whoever reads what this brings
// waits for it (vmcnt) first, and then meets the other waves at a barrier.
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(buffer) : "m0", "memory");
}
// The same with 4 bytes per lane, to `to` + 4 * lane.
__device__ __forceinline__ void load_word_to_lds(i32x4 buffer, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(buffer) : "m0", "memory");
}
// Both with a constant further on in LDS, to be had for an instruction less where several follow one another.
template <int ON>
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t offset, uint32_t to) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(buffer), "n"(ON) : "m0", "scc", "memory");
}
template <int ON>
__device__ __forceinline__ void load_word_to_lds(i32x4 buffer, uint32_t offset, uint32_t to) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(to), "v"(offset), "s"(buffer), "n"(ON) : "m0", "scc", "memory");
}
// All but this wave's last N loads have arrived (no others are under way), and its reads of LDS before them are done.
template <int N>
__device__ __forceinline__ void lds_loads_left() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}
// A barrier alone, where the waits before it were chosen by hand; no access moves across it.
__device__ __forceinline__ void meet() {
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}
// This wave's loads have arrived, and its reads of LDS before them are done.
__device__ __forceinline__ void lds_loads_arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory"); }

// ---- transposing reads of 16-bit tiles in LDS ----
// Of every 16 lanes, lanes 4 r .. 4 r + 3 name the 16 elements of row r (r = 0 .. 3), four each; lane t gets column t of the four rows.
typedef short i16x4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 read_transposed(const char* lds) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4v*)lds));
}

}  // namespace fnn
