// Matrices in 8 bits with a scale for each block of 128 (fnn_quantize), and what the gradient of a layer in 8 bits quantises on the way.
//
// A block's values are read once and kept in registers while their largest magnitude is found; scale = that / 448, code = e4m3(value / scale).  Bound by memory.
#include <type_traits>

#include "e4m3_device.hpp"
#include "net_kernels.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// Blocks of 128 along the rows: 16 bytes a lane, so 16 lanes (fp32: 32) a block.
template <int DT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* x, int64_t x_stride, int64_t n, int32_t d, uint32_t blocks, CodesOut out) {
    typedef typename Elem<DT>::T T;
    constexpr int N = Elem<DT>::N, LANES = SCALED_BLOCK / N, PER = 256 / LANES;
    const uint32_t item = blockIdx.x * PER + threadIdx.x / LANES, block = item % blocks;
    const int64_t row = item / blocks;
    const int lane = threadIdx.x % LANES, at = (int)block * SCALED_BLOCK + lane * N;
    const int count = row < n ? d - at : 0;
    float v[N];
    load_elems<DT, N>((const T*)x + (count > 0 ? row * x_stride + at : 0), count, v);
    const Scale s(block_top<LANES>(v));
    if (row >= n) return;
    if (count > 0) store_codes<N>(out.data + row * out.row + at, count, v, s);
    if (lane == 0) out.scale[row * out.scale_row + block * out.scale_block] = s.scale;
}

// A tile of 128 x 128 a workgroup of 256 threads, 64 values a thread: N neighbouring columns of R rows.  From it come, as wanted, codes by rows, codes
// across (the matrix transposed, its codes gathered in LDS so that 16 of a row leave together), with TILES one scale for the whole of it, and the columns' sums.  With
// SLOPE the values are dy * act'(pre).
template <int DT, bool TILES, bool SLOPE>
__global__ __launch_bounds__(256) void quantize_tile_kernel(QuantizeArgs a) {
    typedef typename Elem<DT>::T T;
    constexpr int N = Elem<DT>::N, LANES = SCALED_BLOCK / N, STRANDS = 256 / LANES, R = SCALED_BLOCK / STRANDS;
    __shared__ __attribute__((aligned(16))) char codes[SCALED_BLOCK * SCALED_BLOCK];
    __shared__ float joined[STRANDS][SCALED_BLOCK];
    const int run = threadIdx.x % LANES, strand = threadIdx.x / LANES;
    const uint32_t tiles_c = (uint32_t)scaled_blocks(a.d), tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x % tiles_c;
    const int64_t r0 = (int64_t)tile_r * SCALED_BLOCK + strand * R;
    const int c0 = (int)tile_c * SCALED_BLOCK, at = c0 + run * N, count = a.d - at;
    float v[R][N];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool there = r0 + i < a.n && count > 0;
        load_elems<DT, N>((const T*)a.x + (there ? (r0 + i) * a.x_stride + at : 0), there ? count : 0, v[i]);
    }
    if constexpr (SLOPE) {
        if (a.act != ACT_NONE) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const bool there = r0 + i < a.n && count > 0;
                float pre[N];
                load_elems<DT, N>((const T*)a.pre + (there ? (r0 + i) * a.pre_stride + at : 0), there ? count : 0, pre);
                times_slope<DT != CT_F32>(v[i], pre, a.act);
            }
        }
        if (a.partial) {
            float sum[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sum[e] = 0.f;
#pragma unroll
                for (int i = 0; i < R; ++i) sum[e] += v[i][e];
                joined[strand][e * LANES + run] = sum[e];
            }
            __syncthreads();
            if (threadIdx.x < SCALED_BLOCK) {
                const int column = c0 + (int)(threadIdx.x % LANES) * N + threadIdx.x / LANES;
                float total = 0.f;
#pragma unroll
                for (int s = 0; s < STRANDS; ++s) total += joined[s][threadIdx.x];
                if (column < a.d) a.partial[tile_r * (int64_t)a.d + column] = total;
            }
            __syncthreads();
        }
    }
    float whole = 0.f;
    if constexpr (TILES) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) top = __builtin_fmaxf(top, top_of<true>(v[i]));
        top = lanes_max<64>(top);
        if ((threadIdx.x & 63) == 0) joined[0][threadIdx.x >> 6] = top;
        __syncthreads();
        whole = __builtin_fmaxf(__builtin_fmaxf(joined[0][0], joined[0][1]), __builtin_fmaxf(joined[0][2], joined[0][3]));
        const Scale s(whole);
        if (threadIdx.x == 0) {
            if (a.rows.data) a.rows.scale[tile_r * a.rows.scale_row + tile_c * a.rows.scale_block] = s.scale;
            if (a.across.data) a.across.scale[tile_c * a.across.scale_row + tile_r * a.across.scale_block] = s.scale;
        }
    }
    if (a.rows.data) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const Scale s(TILES ? whole : block_top<LANES>(v[i]));
            if (r0 + i >= a.n) continue;
            if (count > 0) store_codes<N>(a.rows.data + (r0 + i) * a.rows.row + at, count, v[i], s);
            if (!TILES && run == 0) a.rows.scale[(r0 + i) * a.rows.scale_row + tile_c * a.rows.scale_block] = s.scale;
        }
    }
    if (!a.across.data) return;
    // a column's largest magnitude, over the strands
    float top[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        top[e] = whole;
        if constexpr (!TILES) {
            float column[R];
#pragma unroll
            for (int i = 0; i < R; ++i) column[i] = v[i][e];
            joined[strand][e * LANES + run] = top_of<true>(column);
        }
    }
    if constexpr (!TILES) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < N; ++e) {
            top[e] = joined[0][e * LANES + run];
#pragma unroll
            for (int s = 1; s < STRANDS; ++s) top[e] = __builtin_fmaxf(top[e], joined[s][e * LANES + run]);
        }
    }
    // Column c lies at 128 c, the 16-byte runs of its codes exchanged by the thread that had it, so that the writes of one instruction spread over LDS.
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const Scale s(top[e]);
        uint32_t raw[R / 4];
#pragma unroll
        for (int i = 0; i < R; i += 4) raw[i / 4] = four_codes(v[i][e], v[i + 1][e], v[i + 2][e], v[i + 3][e], s);
        const int first = strand * R, slot = ((first >> 4) ^ (run & 7)) * 16 + (first & 15);
        __builtin_memcpy(codes + (run * N + e) * SCALED_BLOCK + slot, raw, R);
        if (!TILES && strand == 0 && e < count) a.across.scale[(at + e) * a.across.scale_row + tile_r * a.across.scale_block] = s.scale;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int column = i * 32 + threadIdx.x / 8, piece = threadIdx.x % 8;
        const int64_t row = (int64_t)tile_r * SCALED_BLOCK + piece * 16;
        if (c0 + column >= a.d || row >= a.n) continue;
        const uint4 got = *reinterpret_cast<const uint4*>(codes + column * SCALED_BLOCK + ((piece ^ ((column / N) & 7)) << 4));
        uint8_t* to = a.across.data + (c0 + column) * a.across.row + row;
        if (row + 16 <= a.n) {
            __builtin_memcpy(to, &got, 16);
        } else {
            uint8_t raw[16];
            __builtin_memcpy(raw, &got, 16);
#pragma unroll
            for (int e = 0; e < 15; ++e)
                if (row + e < a.n) to[e] = raw[e];
        }
    }
}

// Codes transposed as they are: a tile of 128 x 128 bytes a workgroup, through LDS.
__global__ __launch_bounds__(256) void transpose_codes_kernel(const uint8_t* from, int64_t from_stride, int64_t n, int32_t d, uint8_t* to, int64_t to_stride) {
    __shared__ __attribute__((aligned(16))) uint8_t tile[SCALED_BLOCK][SCALED_BLOCK + 4];
    const uint32_t tiles_c = (uint32_t)scaled_blocks(d);
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * SCALED_BLOCK;
    const int c0 = (int)(blockIdx.x % tiles_c) * SCALED_BLOCK;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 32 + threadIdx.x / 8, column = threadIdx.x % 8 * 16;
        const uint4 got = r0 + row < n ? load_run<CT_E4M3>(from + (r0 + row) * from_stride + c0 + column, d - c0 - column) : uint4{0u, 0u, 0u, 0u};
        const uint32_t words[4] = {got.x, got.y, got.z, got.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<uint32_t*>(&tile[row][column + 4 * w]) = words[w];
    }
    __syncthreads();
    // a thread: 16 rows of four columns, read as words and turned
    const int column = threadIdx.x % 32 * 4, row = threadIdx.x / 32 * 16;
    uint32_t word[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) word[i] = *reinterpret_cast<const uint32_t*>(&tile[row + i][column]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c0 + column + e >= d) break;
        uint8_t out[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) out[i] = (uint8_t)(word[i] >> (8 * e));
        uint8_t* at = to + (int64_t)(c0 + column + e) * to_stride + r0 + row;
        if (r0 + row + 16 <= n) {
            __builtin_memcpy(at, out, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (r0 + row + i < n) at[i] = out[i];
        }
    }
}

template <typename F>
hipError_t with_type(int dtype, F f) {
    if (dtype == FNN_F32) return f(std::integral_constant<int, CT_F32>());
    if (dtype == FNN_F16) return f(std::integral_constant<int, CT_F16>());
    return f(std::integral_constant<int, CT_BF16>());
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int64_t x_stride, int64_t n, int32_t d, const CodesOut& out, int dtype, int kind, hipStream_t s) {
    if (n < 1 || d < 1) return hipSuccess;
    return with_type(dtype, [&](auto dt) {
        constexpr int per = 256 * Elem<dt.value>::N / SCALED_BLOCK;
        const int64_t blocks = scaled_blocks(d), groups = (n * blocks + per - 1) / per;
        if (n * blocks > (int64_t)UINT32_MAX - per) return hipErrorInvalidValue;  // blocks are counted in 32 bits: no memory holds so many
        return launch(kind, quantize_rows_kernel<dt.value>, dim3((unsigned)groups), dim3(256), 0, s, x, x_stride, n, d, (uint32_t)blocks, out);
    });
}

hipError_t launch_quantize_tiles(const QuantizeArgs& a, bool tiles, bool slope, int dtype, int kind, hipStream_t s) {
    if (a.n < 1 || a.d < 1) return hipSuccess;
    const int64_t count = scaled_blocks(a.n) * scaled_blocks(a.d);
    if (count > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)count);
    return with_type(dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        if (slope) return launch(kind, quantize_tile_kernel<DT, false, true>, grid, dim3(256), 0, s, a);
        if (tiles) return launch(kind, quantize_tile_kernel<DT, true, false>, grid, dim3(256), 0, s, a);
        return launch(kind, quantize_tile_kernel<DT, false, false>, grid, dim3(256), 0, s, a);
    });
}

hipError_t launch_transpose_codes(const void* from, int64_t from_stride, int64_t n, int32_t d, void* to, int64_t to_stride, int kind, hipStream_t s) {
    if (n < 1 || d < 1) return hipSuccess;
    const int64_t count = scaled_blocks(n) * scaled_blocks(d);
    if (count > INT32_MAX) return hipErrorInvalidValue;
    return launch(kind, transpose_codes_kernel, dim3((unsigned)count), dim3(256), 0, s, (const uint8_t*)from, from_stride, n, d, (uint8_t*)to, to_stride);
}

}  // namespace fnn
