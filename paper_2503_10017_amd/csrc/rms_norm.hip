// Root-mean-square norm of a sum over rows, with its result in the inputs' type, in 8 bits with scales, or both, and its gradient (fnn_rms_norm,
// fnn_rms_norm_backward).
//
// Both are bound by memory: a row is read once, kept in registers as fp32 while its sum of squares is formed, and written once.  A block of 128 elements lies in 16
// neighbouring lanes (fp32: 32), so its largest magnitude takes no LDS.
#include "e4m3_device.hpp"
#include "norm_shape.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// 1 / sqrt(mean square + eps) of a row whose sum of squares is too large or too small for fp32, or no number: summed again in units of its largest
// magnitude, and put together in 64 bits.  v is left in these units; `of_v` is what brings it to the norm.  Every thread of the row is here.
template <int LANES, int CHUNKS, int N>
__device__ float rare_rstd(float (&v)[CHUNKS][N], float total, int d, float eps, float* slot, float& of_v) {
    uint32_t bits = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) bits = larger(bits, top_of<false>(v[c]));
    bits = lanes_max<64>(bits);
    if constexpr (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = __uint_as_float(bits);
        __syncthreads();
        for (int w = 0; w < LANES / 64; ++w) bits = larger(bits, __float_as_uint(slot[w]));
        __syncthreads();
    }
    const float top = __uint_as_float(bits);
    int exponent = 0;
    if (top > 0.f && top < __builtin_inff()) {
        exponent = ilogbf(top);
        float square = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                v[c][e] = ldexpf(v[c][e], -exponent);
                square = __builtin_fmaf(v[c][e], v[c][e], square);
            }
        total = row_sum<LANES>(square, slot);
        if constexpr (LANES > 64) __syncthreads();
    }
    const double rstd = 1.0 / sqrt(ldexp((double)total / d, 2 * exponent) + eps);
    of_v = (float)ldexp(rstd, exponent);
    return (float)rstd;
}

// s = x + residual, r = 1 / sqrt(mean(s^2) + eps), y = s r w; the sum is rounded where it is stored, y is of the unrounded one.  Rows are divided as the layer
// norm's are: a wave a row while its registers hold one.  24576 x 1024 bf16 with a residual, the sum stored and the norm in 8 bits (177 MB): 33-35 us, what a copy
// takes (35-37 with loads that waited for each other); fp32 (328 MB) 61 us; one row: 3.1-3.6 us, a launch.  16-bit rows that end in a partial run of 16 bytes wait for its elements one after the other:
// 24576 x 1021 bf16 50 us (fp32 64).
template <int DT, int WT, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void rms_norm_kernel(RmsArgs a) {
    constexpr int N = Elem<DT>::N, THREADS = norm_threads(LANES), ROWS = THREADS / LANES, BLOCK_LANES = SCALED_BLOCK / N;
    typedef typename Elem<DT>::T T;
    typedef typename Elem<WT>::T W;
    __shared__ float slots[2][THREADS / 64];
    const int lane = threadIdx.x % LANES;
    float w[CHUNKS][N];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = (c * LANES + lane) * N, count = a.d - at;
#pragma unroll
        for (int e = 0; e < N; ++e) w[c][e] = 1.f;
        if (a.weight && count > 0) load_elems<WT, N>((const W*)a.weight + at, count, w[c]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES; row < a.n; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const T* x = (const T*)a.x + row * a.x_stride;
        // everything is asked for before anything is used, but for partial runs of 16 bytes (load_run)
        uint4 asked[CHUNKS], more[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
            asked[c] = load_run<DT>(x + at, a.d - at);
        }
        if (a.residual) {
            const T* residual = (const T*)a.residual + row * a.residual_stride;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c * LANES + lane) * N;
                more[c] = load_run<DT>(residual + at, a.d - at);
            }
        }
        float v[CHUNKS][N];
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            T raw[N];
            __builtin_memcpy(raw, &asked[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) v[c][e] = (float)raw[e];
        }
        if (a.residual) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                T raw[N];
                __builtin_memcpy(raw, &more[c], 16);
#pragma unroll
                for (int e = 0; e < N; ++e) v[c][e] += (float)raw[e];
            }
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) sum = __builtin_fmaf(v[c][e], v[c][e], sum);
        if (a.sum) {
            T* to = (T*)a.sum + row * a.sum_stride;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c * LANES + lane) * N;
                store_elems<DT, N>(to + at, a.d - at, v[c]);
            }
        }
        sum = row_sum<LANES>(sum, slots[turn]);
        // squares above fp32's range, or so small that they lose digits beside a small eps
        float rstd, of_v;
        if (sum < 0x1p126f && (sum > 0x1p-100f || a.eps > 0x1p-90f)) of_v = rstd = 1.f / sqrtf(sum / (float)a.d + a.eps);
        else rstd = rare_rstd<LANES>(v, sum, a.d, a.eps, slots[turn], of_v);
        // in this order: s r is at most sqrt(d) in size, while r w leaves fp32's range for weights and rows far from 1
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) v[c][e] = v[c][e] * of_v * w[c][e];
        if (a.y) {
            T* y = (T*)a.y + row * a.y_stride;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c * LANES + lane) * N;
                store_elems<DT, N>(y + at, a.d - at, v[c]);
            }
        }
        if (a.codes.data) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c * LANES + lane) * N, count = a.d - at;
                const Scale s = Scale::of<true>(block_top<BLOCK_LANES>(v[c]));
                if (count <= 0) continue;
                store_codes<N>(a.codes.data + row * a.codes.row + at, count, v[c], s);
                if (lane % BLOCK_LANES == 0) a.codes.scale[row * a.codes.scale_row + at / SCALED_BLOCK * a.codes.scale_block] = s.scale;
            }
        }
        if (lane == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// With g = dy w, h = s r:  dx = r (g - h mean(g h)) + dsum,  dw = sum dy h.  One pass over dy, s and dsum; in registers the columns' sums over the workgroup's
// rows, which end as one row of `partial`.  24576 x 1024 bf16 with dsum (201 MB): 36-41 us, 5.2 TB/s, and 4 to 4.7 to join the columns' sums; fp32 (403 MB) 74 and 4.1.  6151 x 1021 fp32, whose rows start on 4-byte
// boundaries (75 MB): 17 us, 4.4 TB/s, and 3.9; 6151 x 1024 16.5.  Partial runs of 16-bit types are waited for as above, and with them the row asked for ahead: 24576 x 1021 bf16 60 us.
template <int DT, int WT, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void rms_norm_backward_kernel(RmsBackArgs a) {
    constexpr int N = Elem<DT>::N, THREADS = norm_threads(LANES), ROWS = THREADS / LANES;
    typedef typename Elem<DT>::T T;
    typedef typename Elem<WT>::T W;
    __shared__ float slots[2][THREADS / 64];
    const int lane = threadIdx.x % LANES;
    const float inv_d = 1.f / (float)a.d;
    const bool sums = a.partial != nullptr;
    float w[CHUNKS][N], dw[CHUNKS][N];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int at = (c * LANES + lane) * N, count = a.d - at;
#pragma unroll
        for (int e = 0; e < N; ++e) w[c][e] = 1.f, dw[c][e] = 0.f;
        if (a.weight && count > 0) load_elems<WT, N>((const W*)a.weight + at, count, w[c]);
    }
    // A row is asked for while the one before it is worked on, where a thread has the registers for it.
    constexpr bool AHEAD = CHUNKS * N <= 16 && LANES < 1024;
    uint4 next_dy[CHUNKS], next_x[CHUNKS], next_more[CHUNKS];
    float next_rstd = 0.f;
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
        if (a.dsum && a.dx) {
            const T* more = (const T*)a.dsum + row * a.dsum_stride;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int at = (c * LANES + lane) * N;
                next_more[c] = load_run<DT>(more + at, a.d - at);
            }
        }
        next_rstd = a.rstd[row];
    };
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) next_more[c] = uint4{0u, 0u, 0u, 0u};
    const int64_t rows_on = (int64_t)gridDim.x * ROWS;
    int turn = 0;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (AHEAD) ask(row);
    for (; row < a.n; row += rows_on, turn ^= 1) {
        if (!AHEAD) ask(row);
        const float rstd = next_rstd;
        float g[CHUNKS][N], h[CHUNKS][N], more[CHUNKS][N];
        float sum_gh = 0.f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            T raw[N];
            __builtin_memcpy(raw, &next_dy[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) g[c][e] = (float)raw[e];
            __builtin_memcpy(raw, &next_x[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) h[c][e] = (float)raw[e] * rstd;
            __builtin_memcpy(raw, &next_more[c], 16);
#pragma unroll
            for (int e = 0; e < N; ++e) more[c][e] = (float)raw[e];
        }
        if (AHEAD) ask(row + rows_on);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int count = a.d - (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (e >= count) h[c][e] = 0.f;  // what an infinite or missing rstd makes of the zeros behind a row's end
                dw[c][e] = __builtin_fmaf(g[c][e], h[c][e], dw[c][e]);
                g[c][e] *= w[c][e];
                sum_gh = __builtin_fmaf(g[c][e], h[c][e], sum_gh);
            }
        }
        if (!a.dx) continue;
        const float along = row_sum<LANES>(sum_gh, slots[turn]) * inv_d;
        T* dx = (T*)a.dx + row * a.dx_stride;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) g[c][e] = __builtin_fmaf(__builtin_fmaf(-h[c][e], along, g[c][e]), rstd, more[c][e]);
            store_elems<DT, N>(dx + at, a.d - at, g[c]);
        }
    }
    if (!sums) return;
    float* out = a.partial + (int64_t)blockIdx.x * a.d;
    if constexpr (ROWS > 1) {  // the waves' sums are joined in LDS, in their order
        __shared__ float joined[ROWS - 1][64 * N];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            __syncthreads();
            if (threadIdx.x >= LANES) {
#pragma unroll
                for (int e = 0; e < N; ++e) joined[threadIdx.x / LANES - 1][e * 64 + lane] = dw[c][e];
            }
            __syncthreads();
            if (threadIdx.x < LANES) {
                const int at = (c * LANES + lane) * N;
#pragma unroll
                for (int e = 0; e < N; ++e) {
#pragma unroll
                    for (int r = 0; r < ROWS - 1; ++r) dw[c][e] += joined[r][e * 64 + lane];
                }
                store_elems<CT_F32, N>(out + at, a.d - at, dw[c]);
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = (c * LANES + lane) * N;
            store_elems<CT_F32, N>(out + at, a.d - at, dw[c]);
        }
    }
}

constexpr int64_t NORM_GROUPS = 2048;

}  // namespace

hipError_t launch_rms_norm(const RmsArgs& a, int dtype, int weight_dtype, hipStream_t s) {
    return with_types(dtype, weight_dtype, [&](auto dt, auto wt) {
        return with_shape<dt.value>(a.d, [&](auto lanes, auto chunks) {
            constexpr int threads = norm_threads(lanes.value), rows = threads / lanes.value;
            const int64_t groups = (a.n + rows - 1) / rows;
            return launch(TK_RMS_NORM, rms_norm_kernel<dt.value, wt.value, lanes.value, chunks.value>,
                          dim3((unsigned)(groups < NORM_GROUPS ? groups : NORM_GROUPS)), dim3(threads), 0, s, a);
        });
    });
}

int64_t rms_norm_backward_groups(int64_t n, int32_t d) { return layer_norm_backward_groups(n, d); }

hipError_t launch_rms_norm_backward(const RmsBackArgs& a, int dtype, int weight_dtype, hipStream_t s) {
    const int64_t groups = rms_norm_backward_groups(a.n, a.d);
    return with_types(dtype, weight_dtype, [&](auto dt, auto wt) {
        const hipError_t e = with_shape<dt.value>(a.d, [&](auto lanes, auto chunks) {
            return launch(TK_RMS_NORM_BACKWARD, rms_norm_backward_kernel<dt.value, wt.value, lanes.value, chunks.value>,
                          dim3((unsigned)groups), dim3(norm_threads(lanes.value)), 0, s, a);
        });
        if (e != hipSuccess || !a.partial) return e;
        return launch_column_sums(a.partial, groups, a.d, a.d, a.dweight, nullptr, weight_dtype, TK_RMS_NORM_BACKWARD, s);
    });
}

}  // namespace fnn
