// How the norms divide their rows among threads.
#pragma once
#include <type_traits>

#include "net_device.hpp"
#include "net_kernels.hpp"

namespace fnn {

// A row is shared by LANES threads, each of which holds CHUNKS runs of 16 bytes, LANES runs apart.  A workgroup has 256 threads, or
// LANES where that is more.
constexpr int norm_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

// Sum over the LANES threads of a row.  `slot`: LDS, one word per wave; two alternating rows of it make one barrier enough.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* slot) {
    x = wave_sum(x);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) x += slot[w];
    }
    return x;
}

// Calls f(LANES, CHUNKS) with the narrowest shape that holds a row of d elements: one wave a row as long as its registers do.
template <int DT, typename F>
hipError_t with_shape(int d, F f) {
    constexpr int N = Elem<DT>::N;
#define FNN_SHAPE(LANES, CHUNKS) \
    if (d <= LANES * CHUNKS * N) return f(std::integral_constant<int, LANES>(), std::integral_constant<int, CHUNKS>());
    FNN_SHAPE(64, 1)
    FNN_SHAPE(64, 2)
    FNN_SHAPE(64, 4)
    if constexpr (DT == CT_F32) {
        FNN_SHAPE(256, 2)
        FNN_SHAPE(256, 4)
        FNN_SHAPE(1024, 2)
        FNN_SHAPE(1024, 4)
    } else {
        FNN_SHAPE(256, 2)
        FNN_SHAPE(256, 4)
        FNN_SHAPE(1024, 2)
    }
#undef FNN_SHAPE
    return hipErrorInvalidValue;
}
template <typename F>
hipError_t with_types(int dtype, int weight_dtype, F f) {
    if (dtype == FNN_F32) return f(std::integral_constant<int, CT_F32>(), std::integral_constant<int, CT_F32>());
    if (dtype == FNN_F16)
        return weight_dtype == FNN_F16 ? f(std::integral_constant<int, CT_F16>(), std::integral_constant<int, CT_F16>())
                                       : f(std::integral_constant<int, CT_F16>(), std::integral_constant<int, CT_F32>());
    return weight_dtype == FNN_BF16 ? f(std::integral_constant<int, CT_BF16>(), std::integral_constant<int, CT_BF16>())
                                    : f(std::integral_constant<int, CT_BF16>(), std::integral_constant<int, CT_F32>());
}

}  // namespace fnn
