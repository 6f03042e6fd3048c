// Layer norm over rows and its gradient (fnn_layer_norm, fnn_layer_norm_backward).
//
// Both are bound by memory: a row is read once, kept in registers as fp32 while its sums are formed (the variance from the
// centred values, so a mean far from zero costs no digits), and written once.
#include <type_traits>

#include "net_device.hpp"
#include "net_kernels.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

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

// y = (x - mean) rstd w + b.  A wave a row while its registers hold one (up to 2048 16-bit elements), so that rows need no barrier; weights are loaded once per
// workgroup, of which there are at most 2048.  24576 x 1024 bf16 (101 MB): 21.4 us, 4.7 TB/s of the 5.1 that a large copy reaches.  One row: 2.7 us, a launch.
template <int DT, int WT, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_kernel(NormArgs a) {
    constexpr int N = Elem<DT>::N, THREADS = norm_threads(LANES), ROWS = THREADS / LANES;
    typedef typename Elem<DT>::T T;
    typedef typename Elem<WT>::T W;
    __shared__ float slots[2][THREADS / 64];
    const int lane = threadIdx.x % LANES;
    const float d = (float)a.d;
    float w[CHUNKS][N], b[CHUNKS][N];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = (c * LANES + lane) * N, count = a.d - at;
#pragma unroll
        for (int e = 0; e < N; ++e) w[c][e] = 1.f, b[c][e] = 0.f;
        if (a.weight && count > 0) load_elems<WT, N>((const W*)a.weight + at, count, w[c]);
        if (a.bias && count > 0) load_elems<WT, N>((const W*)a.bias + at, count, b[c]);
    }
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.n; row += (int64_t)gridDim.x * ROWS) {
        const T* x = (const T*)a.x + row * a.x_stride;
        float v[CHUNKS][N];
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
            load_elems<DT, N>(x + at, a.d - at, v[c]);
#pragma unroll
            for (int e = 0; e < N; ++e) sum += v[c][e];
        }
        const float mean = row_sum<LANES>(sum, slots[0]) / d;  // divided, so that a row of one value has that value as its mean
        float square = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int count = a.d - (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[c][e] = e < count ? v[c][e] - mean : 0.f;
                square = __builtin_fmaf(v[c][e], v[c][e], square);
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<LANES>(square, slots[1]) / d + a.eps);
        T* y = (T*)a.y + row * a.y_stride;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) v[c][e] = __builtin_fmaf(v[c][e] * rstd, w[c][e], b[c][e]);
            store_elems<DT, N>(y + at, a.d - at, v[c]);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// With g = dy w, h = (x - mean) rstd:  dx = rstd (g - mean(g) - h mean(g h)),  dw = sum dy h,  db = sum dy.
// One pass over dy and x: dx of each row, and in registers the columns' sums over the workgroup's rows, which end as one row of
// `partial`; 768 workgroups at most, three a compute unit, so that these rows stay small beside the operands.  24576 x 1024 bf16 (151 MB): 30 us and 4 for the join
// of the sums, 4.4 TB/s in all; 6151 x 1021 fp32 (75 MB, rows on 4-byte boundaries) 18 and 4 us.
template <int DT, int WT, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_backward_kernel(NormBackArgs a) {
    constexpr int N = Elem<DT>::N, THREADS = norm_threads(LANES), ROWS = THREADS / LANES;
    typedef typename Elem<DT>::T T;
    typedef typename Elem<WT>::T W;
    __shared__ float slots[2][2 * (THREADS / 64)];
    const int lane = threadIdx.x % LANES;
    const float inv_d = 1.f / (float)a.d;
    const bool sums = a.partial != nullptr;
    float w[CHUNKS][N], dw[CHUNKS][N], db[CHUNKS][N];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = (c * LANES + lane) * N, count = a.d - at;
#pragma unroll
        for (int e = 0; e < N; ++e) w[c][e] = 1.f, dw[c][e] = 0.f, db[c][e] = 0.f;
        if (a.weight && count > 0) load_elems<WT, N>((const W*)a.weight + at, count, w[c]);
    }
    // A row is asked for while the one before it is worked on: with a workgroup's few rows in flight the time is the memory's latency otherwise
    // (24576 x 1024 bf16, cold: 49 us without, 40 with).  Where a thread has 32 elements of a row, or a workgroup 1024 threads, the registers for it are not there.
    constexpr bool AHEAD = CHUNKS * N <= 16 && LANES < 1024;
    uint4 next_dy[CHUNKS], next_x[CHUNKS];
    float next_mean = 0.f, next_rstd = 0.f;
    auto ask = [&](int64_t row) {
        if (row >= a.n) return;
        const T* dy = (const T*)a.dy + row * a.dy_stride;
        const T* x = (const T*)a.x + row * a.x_stride;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
            next_dy[c] = load_run<DT>(dy + at, a.d - at);
            next_x[c] = load_run<DT>(x + at, a.d - at);
        }
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
    };
    const int64_t rows_on = (int64_t)gridDim.x * ROWS;
    int turn = 0;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (AHEAD) ask(row);
    for (; row < a.n; row += rows_on, turn ^= 1) {
        if (!AHEAD) ask(row);
        const float mean = next_mean, rstd = next_rstd;
        float g[CHUNKS][N], h[CHUNKS][N];
        float sum_g = 0.f, sum_gh = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            T raw[N];
            __builtin_memcpy(raw, &next_dy[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) g[c][e] = (float)raw[e];
            __builtin_memcpy(raw, &next_x[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) h[c][e] = (float)raw[e];
        }
        if (AHEAD) ask(row + rows_on);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int count = a.d - (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                h[c][e] = e < count ? (h[c][e] - mean) * rstd : 0.f;
                dw[c][e] = __builtin_fmaf(g[c][e], h[c][e], dw[c][e]);
                db[c][e] += g[c][e];
                g[c][e] *= w[c][e];
                sum_g += g[c][e];
                sum_gh = __builtin_fmaf(g[c][e], h[c][e], sum_gh);
            }
        }
        if (!a.dx) continue;
        sum_g = wave_sum(sum_g);
        sum_gh = wave_sum(sum_gh);
        if constexpr (LANES > 64) {
            float* slot = slots[turn];
            if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = sum_g, slot[THREADS / 64 + (threadIdx.x >> 6)] = sum_gh;
            __syncthreads();
            sum_g = sum_gh = 0.f;
#pragma unroll
            for (int i = 0; i < LANES / 64; ++i) sum_g += slot[i], sum_gh += slot[THREADS / 64 + i];
        }
        const float mg = sum_g * inv_d, mgh = sum_gh * inv_d;
        T* dx = (T*)a.dx + row * a.dx_stride;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) g[c][e] = (g[c][e] - mg - h[c][e] * mgh) * rstd;
            store_elems<DT, N>(dx + at, a.d - at, g[c]);
        }
    }
    if (!sums) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.d;
    if constexpr (ROWS > 1) {  // the waves' sums are joined in LDS, in their order
        __shared__ float joined[ROWS - 1][64 * N];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float (&mine)[N] = which ? db[c] : dw[c];
                __syncthreads();
                if (threadIdx.x >= LANES) {
#pragma unroll
                    for (int e = 0; e < N; ++e) joined[threadIdx.x / LANES - 1][e * 64 + lane] = mine[e];
                }
                __syncthreads();
                if (threadIdx.x < LANES) {
                    const int at = (c * LANES + lane) * N;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
#pragma unroll
                        for (int r = 0; r < ROWS - 1; ++r) mine[e] += joined[r][e * 64 + lane];
                    }
                    store_elems<CT_F32, N>(out + (int64_t)which * a.d + at, a.d - at, mine);
                }
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
            store_elems<CT_F32, N>(out + at, a.d - at, dw[c]);
            store_elems<CT_F32, N>(out + a.d + at, a.d - at, db[c]);
        }
    }
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

constexpr int64_t NORM_GROUPS = 2048;

}  // namespace

hipError_t launch_layer_norm(const NormArgs& a, int dtype, int weight_dtype, hipStream_t s) {
    return with_types(dtype, weight_dtype, [&](auto dt, auto wt) {
        return with_shape<dt.value>(a.d, [&](auto lanes, auto chunks) {
            constexpr int threads = norm_threads(lanes.value), rows = threads / lanes.value;
            const int64_t groups = (a.n + rows - 1) / rows;
            return launch(TK_LAYER_NORM, layer_norm_kernel<dt.value, wt.value, lanes.value, chunks.value>,
                          dim3((unsigned)(groups < NORM_GROUPS ? groups : NORM_GROUPS)), dim3(threads), 0, s, a);
        });
    });
}

int64_t layer_norm_backward_groups(int64_t n, int32_t d) {
    const int64_t groups = (n + 3) / 4;
    return groups < 768 ? (groups < 1 ? 1 : groups) : 768;
}

hipError_t launch_layer_norm_backward(const NormBackArgs& a, int dtype, int weight_dtype, hipStream_t s) {
    const int64_t groups = layer_norm_backward_groups(a.n, a.d);
    return with_types(dtype, weight_dtype, [&](auto dt, auto wt) {
        const hipError_t e = with_shape<dt.value>(a.d, [&](auto lanes, auto chunks) {
            return launch(TK_LAYER_NORM_BACKWARD, layer_norm_backward_kernel<dt.value, wt.value, lanes.value, chunks.value>,
                          dim3((unsigned)groups), dim3(norm_threads(lanes.value)), 0, s, a);
        });
        if (e != hipSuccess || !a.partial) return e;
        return launch_column_sums(a.partial, groups, 2 * (int64_t)a.d, a.d, a.dweight, a.dbias, weight_dtype, TK_LAYER_NORM_BACKWARD, s);
    });
}

}  // namespace fnn
