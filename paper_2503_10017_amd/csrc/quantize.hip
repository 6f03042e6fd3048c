// Matrices in 8 bits with a scale for each block of 128 (fnn_quantize), and what the gradient of a layer in 8 bits quantises on the way.
//
// A block's values are read once and kept in registers while their largest magnitude is found; scale = that / 448, code = e4m3(value / scale).  Bound by memory.
#include <type_traits>

#include "e4m3_device.hpp"
#include "net_kernels.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// Blocks of 128 along the rows: 16 bytes a lane, so 16 lanes (fp32: 32) a block, and a block's largest takes no LDS.  24576 x 4096 bf16 (305 MB): 55-59 us, 5.2 to 5.5 TB/s.
template <int DT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const void* x, int64_t x_stride, int64_t n, int32_t d, uint32_t blocks, uint32_t first, CodesOut out) {
    typedef typename Elem<DT>::T T;
    constexpr int N = Elem<DT>::N, LANES = SCALED_BLOCK / N, PER = 256 / LANES;
    const uint32_t item = (first + blockIdx.x) * PER + threadIdx.x / LANES, block = item % blocks;
    const int64_t row = item / blocks;
    const int lane = threadIdx.x % LANES, at = (int)block * SCALED_BLOCK + lane * N;
    const int count = row < n ? d - at : 0;
    float v[N];
    load_elems<DT, N>((const T*)x + (count > 0 ? row * x_stride + at : 0), count, v);
    const Scale s = Scale::of<true>(block_top<LANES>(v));
    if (row >= n) return;
    if (count > 0) store_codes<N>(out.data + row * out.row + at, count, v, s);
    if (lane == 0) out.scale[row * out.scale_row + block * out.scale_block] = s.scale;
}

constexpr int TILE_THREADS = 512;

// join(x, y) over the wave's strands of rows, for each of the thread's N columns, left in LDS.
template <int N, typename V, typename Join>
__device__ __forceinline__ void over_strands(V (&x)[N], V (*parts)[SCALED_BLOCK], Join join) {
    constexpr int LANES = SCALED_BLOCK / N;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto bits = [](V v) { return __builtin_bit_cast(uint32_t, v); };
    auto value = [](uint32_t v) { return __builtin_bit_cast(V, v); };
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (LANES == 16) {
            const auto a = __builtin_amdgcn_permlane16_swap(bits(x[e]), bits(x[e]), false, false);
            x[e] = join(value(a[0]), value(a[1]));
        }
        const auto b = __builtin_amdgcn_permlane32_swap(bits(x[e]), bits(x[e]), false, false);
        x[e] = join(value(b[0]), value(b[1]));
    }
    if (lane < LANES) __builtin_memcpy(&parts[wave][lane * N], x, sizeof(x));
}
// ... and over the waves, of one column.
template <typename V, typename Join>
__device__ __forceinline__ V over_waves(const V (*parts)[SCALED_BLOCK], int column, Join join) {
    V total = parts[0][column];
#pragma unroll
    for (int w = 1; w < TILE_THREADS / 64; ++w) total = join(total, parts[w][column]);
    return total;
}
__device__ __forceinline__ float plus(float x, float y) { return x + y; }

struct TileRoom {
    __attribute__((aligned(16))) char codes[SCALED_BLOCK * SCALED_BLOCK];
    float sums[TILE_THREADS / 64][SCALED_BLOCK];
    uint32_t tops[TILE_THREADS / 64][SCALED_BLOCK];
    float scale[SCALED_BLOCK], over[SCALED_BLOCK];
};

// A tile of 128 x 128 a workgroup, 32 values a thread: N neighbouring columns of R rows.  From it come, as wanted, codes by rows, codes across (the matrix transposed, its codes gathered in
// LDS so that 16 of a row leave together), with TILES one scale for the whole of it, and the columns' sums.  With SLOPE the values are dy * act'(pre).  A column's scale is formed by one
// thread, not by the 16 that use it, and the joins over rows share the workgroup's three meetings.  Inside a matrix the time is the bytes': 12288 x 1024 fp16 across (38 MB) 9.4 us, 24576 x 4096 bf16
// (305 MB) in tiles 57 and across 56 us, fp32 (503 MB) 90 and 98.  A tile at an edge takes longer, and a launch of few generations of workgroups as long as those do: 12289 x 1024 10.9 us, and
// 12289 x 1016 12.0, whose rows are asked for under a branch each; 12289 x 1021 14.0, whose partial runs are read element by element and waited for one after the other.
template <int DT, bool TILES, bool SLOPE>
__device__ __forceinline__ void quantize_tile(const QuantizeArgs& a, uint32_t tile, TileRoom& room) {
    typedef typename Elem<DT>::T T;
    constexpr int N = Elem<DT>::N, LANES = SCALED_BLOCK / N, R = SCALED_BLOCK * SCALED_BLOCK / TILE_THREADS / N;
    const int run = threadIdx.x % LANES, strand = threadIdx.x / LANES;
    const uint32_t tiles_c = (uint32_t)scaled_blocks(a.d), tile_r = tile / tiles_c, tile_c = tile % tiles_c;
    const int64_t r0 = (int64_t)tile_r * SCALED_BLOCK + strand * R;
    const int c0 = (int)tile_c * SCALED_BLOCK, at = c0 + run * N, count = a.d - at;
    // Everything is asked for before anything is used, but for partial runs of 16 bytes (load_run).
    const bool inside = (int64_t)(tile_r + 1) * SCALED_BLOCK <= a.n && a.d - c0 >= SCALED_BLOCK;
    auto ask = [&](uint4 (&to)[R], const void* base, int64_t stride) {
        const T* from = (const T*)base + r0 * stride + at;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (inside) __builtin_memcpy(&to[i], from + i * stride, 16);
            else to[i] = load_run<DT>(from + i * stride, r0 + i < a.n ? count : 0);
        }
    };
    auto values = [&](float (&to)[N], const uint4& of) {
        T raw[N];
        __builtin_memcpy(raw, &of, 16);
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = (float)raw[e];
    };
    uint4 asked[R], pre[R];
    ask(asked, a.x, a.x_stride);
    if (SLOPE && a.act != ACT_NONE) ask(pre, a.pre, a.pre_stride);
    float v[R][N];
#pragma unroll
    for (int i = 0; i < R; ++i) values(v[i], asked[i]);
    if constexpr (SLOPE) {
        if (a.act != ACT_NONE) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                float p[N];
                values(p, pre[i]);
                times_slope<DT != CT_F32>(v[i], p, a.act);
            }
        }
        if (a.partial) {
            float sum[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sum[e] = 0.f;
#pragma unroll
                for (int i = 0; i < R; ++i) sum[e] += v[i][e];
            }
            over_strands<N>(sum, room.sums, plus);
        }
    }
    uint32_t whole = 0;
    if constexpr (TILES) {
#pragma unroll
        for (int i = 0; i < R; ++i) whole = larger(whole, top_of<true>(v[i]));
        whole = lanes_max<64>(whole);
        if ((threadIdx.x & 63) == 0) room.tops[0][threadIdx.x >> 6] = whole;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TILE_THREADS / 64; ++w) whole = larger(whole, room.tops[0][w]);
        const float scale = Scale::of<false>(whole).scale;
        if (threadIdx.x == 0) {
            if (a.rows.data) a.rows.scale[tile_r * a.rows.scale_row + tile_c * a.rows.scale_block] = scale;
            if (a.across.data) a.across.scale[tile_c * a.across.scale_row + tile_r * a.across.scale_block] = scale;
        }
    } else {
        if (a.across.data) {
            uint32_t top[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float column[R];
#pragma unroll
                for (int i = 0; i < R; ++i) column[i] = v[i][e];
                top[e] = top_of<false>(column);
                if (__any(top[e] >= INFINITE)) top[e] = top_of<true>(column);  // what is not finite is rare, and does not enter the scale
            }
            over_strands<N>(top, room.tops, larger);
        }
        __syncthreads();
    }
    auto encode = [&](auto divided) {  // see four_codes
        constexpr bool DIVIDED = decltype(divided)::value;
        // two waves join the columns' largest and two their sums, the others begin with the rows
        if (!TILES && a.across.data && threadIdx.x < SCALED_BLOCK) {
            const Scale s = Scale::of<DIVIDED>(over_waves(room.tops, threadIdx.x, larger));
            room.scale[threadIdx.x] = s.scale;
            room.over[threadIdx.x] = s.over;
            if (c0 + threadIdx.x < a.d) a.across.scale[(c0 + threadIdx.x) * a.across.scale_row + tile_r * a.across.scale_block] = s.scale;
        }
        if constexpr (SLOPE) {
            const int column = threadIdx.x - SCALED_BLOCK;
            if (a.partial && column >= 0 && column < SCALED_BLOCK && c0 + column < a.d) a.partial[tile_r * (int64_t)a.d + c0 + column] = over_waves(room.sums, column, plus);
        }
        if (a.rows.data) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const Scale s = Scale::of<DIVIDED>(TILES ? whole : block_top<LANES>(v[i]));
                if (r0 + i >= a.n) continue;
                if (count > 0) store_codes<N, DIVIDED>(a.rows.data + (r0 + i) * a.rows.row + at, count, v[i], s);
                if (!TILES && run == 0) a.rows.scale[(r0 + i) * a.rows.scale_row + tile_c * a.rows.scale_block] = s.scale;
            }
        }
        if (!a.across.data) return;
        Scale s = Scale::of<DIVIDED>(whole);
        if (!TILES) __syncthreads();
        // Column c lies at 128 c, the 16-byte runs of its codes exchanged by the thread that had it, so that the writes of one instruction spread over LDS.
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (!TILES) s = Scale::kept<DIVIDED>(room.scale[run * N + e], room.over[run * N + e]);
            uint32_t raw[R / 4];
#pragma unroll
            for (int i = 0; i < R; i += 4) raw[i / 4] = four_codes<DIVIDED>(v[i][e], v[i + 1][e], v[i + 2][e], v[i + 3][e], s);
            const int first = strand * R, slot = ((first >> 4) ^ (run & 7)) * 16 + (first & 15);
            __builtin_memcpy(room.codes + (run * N + e) * SCALED_BLOCK + slot, raw, R);
        }
    };
    if (SLOPE && DT != CT_F32 && a.act >= ACT_GELU) encode(std::false_type());
    else encode(std::true_type());
    if (!a.across.data) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 1024 / TILE_THREADS; ++i) {
        const int column = i * (TILE_THREADS / 8) + threadIdx.x / 8, piece = threadIdx.x % 8;
        const int64_t row = (int64_t)tile_r * SCALED_BLOCK + piece * 16;
        if (c0 + column >= a.d || row >= a.n) continue;
        const uint4 got = *reinterpret_cast<const uint4*>(room.codes + column * SCALED_BLOCK + ((piece ^ ((column / N) & 7)) << 4));
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

template <int DT, bool TILES>
__global__ __launch_bounds__(TILE_THREADS) void quantize_tile_kernel(QuantizeArgs a, uint32_t first) {
    __shared__ TileRoom room;
    quantize_tile<DT, TILES, false>(a, first + blockIdx.x, room);
}

// Codes transposed as they are: a tile of 128 x 64 bytes a workgroup, through LDS.
__device__ __forceinline__ void transpose_tile(const TransposeArgs& a, uint32_t tile, char* room) {
    constexpr int PITCH = 64 + 4;
    const uint32_t tiles_c = (uint32_t)((a.d + 63) / 64);
    const int64_t r0 = (int64_t)(tile / tiles_c) * 128;
    const int c0 = (int)(tile % tiles_c) * 64;
    {
        const int row = threadIdx.x / 4, column = threadIdx.x % 4 * 16;
        const uint4 got = r0 + row < a.n ? load_run<CT_E4M3>(a.from + (r0 + row) * a.from_stride + c0 + column, a.d - c0 - column) : uint4{0u, 0u, 0u, 0u};
        const uint32_t words[4] = {got.x, got.y, got.z, got.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<uint32_t*>(room + row * PITCH + column + 4 * w) = words[w];
    }
    __syncthreads();
    const int column = threadIdx.x / 8, row = threadIdx.x % 8 * 16;
    if (c0 + column >= a.d) return;
    uint8_t out[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) out[i] = room[(row + i) * PITCH + column];
    uint8_t* at = a.to + (int64_t)(c0 + column) * a.to_stride + r0 + row;
    if (r0 + row + 16 <= a.n) {
        __builtin_memcpy(at, out, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (r0 + row + i < a.n) at[i] = out[i];
    }
}

// What the products of a gradient take, in one launch: q by rows and across with its columns' sums, x across, w transposed; as many of these as are wanted.  12288 x 1024 -> 4096 bf16 with GELU
// (347 MB): 80 us, 67 at a copy's rate; the vector units are busy three quarters of the time, with the slope (18 instructions a value) and two sets of codes.  (104 us with loads that waited for each
// other and scales formed by every thread; workgroups of 80 registers instead of 92, so that three fit a compute unit: 5 % longer, they spill.)
template <int DT>
__global__ __launch_bounds__(TILE_THREADS) void gradient_operands_kernel(GradientOperands a) {
    __shared__ TileRoom room;
    const uint32_t tile = a.first + blockIdx.x;
    if (tile < a.tiles_q) quantize_tile<DT, false, true>(a.q, tile, room);
    else if (tile < a.tiles_q + a.tiles_x) quantize_tile<DT, false, false>(a.x, tile - a.tiles_q, room);
    else transpose_tile(a.w, tile - a.tiles_q - a.tiles_x, room.codes);
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
        return in_launches(groups, 256, [&](uint32_t first, dim3 grid) {
            return launch(kind, quantize_rows_kernel<dt.value>, grid, dim3(256), 0, s, x, x_stride, n, d, (uint32_t)blocks, first, out);
        });
    });
}

hipError_t launch_quantize_tiles(const QuantizeArgs& a, bool tiles, int dtype, int kind, hipStream_t s) {
    if (a.n < 1 || a.d < 1) return hipSuccess;
    const int64_t count = scaled_blocks(a.n) * scaled_blocks(a.d);
    if (count > INT32_MAX) return hipErrorInvalidValue;
    return with_type(dtype, [&](auto dt) {
        return in_launches(count, TILE_THREADS, [&](uint32_t first, dim3 grid) {
            return launch(kind, tiles ? quantize_tile_kernel<dt.value, true> : quantize_tile_kernel<dt.value, false>, grid, dim3(TILE_THREADS), 0, s, a, first);
        });
    });
}

hipError_t launch_gradient_operands(GradientOperands a, int dtype, int kind, hipStream_t s) {
    const int64_t q = a.q.x ? scaled_blocks(a.q.n) * scaled_blocks(a.q.d) : 0, x = a.x.x ? scaled_blocks(a.x.n) * scaled_blocks(a.x.d) : 0;
    const int64_t w = a.w.from ? (a.w.n + 127) / 128 * ((a.w.d + 63) / 64) : 0, count = q + x + w;
    if (count > INT32_MAX) return hipErrorInvalidValue;
    if (count == 0) return hipSuccess;
    a.tiles_q = (uint32_t)q;
    a.tiles_x = (uint32_t)x;
    return with_type(dtype, [&](auto dt) {
        return in_launches(count, TILE_THREADS, [&](uint32_t first, dim3 grid) {
            a.first = first;
            return launch(kind, gradient_operands_kernel<dt.value>, grid, dim3(TILE_THREADS), 0, s, a);
        });
    });
}

}  // namespace fnn
