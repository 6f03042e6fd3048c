// Linear layers with their epilogue, and what their gradients need beside matrix products (fnn_linear, fnn_linear_backward).
#include <algorithm>
#include <type_traits>

#include "gemm.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// Whether a product is a pass over b with all of a in registers: up to 16 rows always; up to 64 while a, which every workgroup reads whole, is small.
// (Microseconds, this way and in tiles: 24 x 4096 -> 1024 11.2 and 11.5, 32 x 4096 -> 1024 12.7 and 11.4, 64 x 1024 -> 4096 7.4 and 12.2.)
bool few_rows(int64_t m, int64_t k) { return m <= 16 || (m <= 64 && m * k <= 98304); }
constexpr int FEW_WAVES = 8;

// Few rows of a: the time is that of reading b once.  A workgroup takes 16 rows of b, its waves share k between them, and every
// lane asks for all of its runs of four turns before it multiplies the first; a (its rows are few) comes out of the L2.  The shares are
// joined in LDS in the order of the waves.  1 x 1024 -> 4096 bf16: 4.4 us, 1.9 TB/s of 8.4 MB; a launch that does nothing is about 3.5 of it.
template <int DT, int BLOCKS>
__global__ __launch_bounds__(FEW_WAVES * 64) void few_rows_kernel(GemmArgs a) {
    typedef typename Elem<DT>::T E;
    constexpr int N = Elem<DT>::N, STEP = 4 * N, TURNS = 4;
    __shared__ f32x4 shares[FEW_WAVES][BLOCKS][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const E* row_b = (const E*)a.b + min(n0 + r, (int64_t)a.n - 1) * a.ldb;
    const E* row_a[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) row_a[i] = (const E*)a.a + min((int64_t)(16 * i + r), a.m - 1) * a.lda;
    f32x4 acc[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) acc[i] = (f32x4)(0.f);
    for (int64_t k = (int64_t)wave * STEP; k < a.k; k += FEW_WAVES * STEP * TURNS) {
        uint4 fb[TURNS], fa[TURNS][BLOCKS];
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t at = k + t * FEW_WAVES * STEP + q * N;
            const int count = (int)min((int64_t)a.k - at, (int64_t)N);
            fb[t] = load_run<DT>(row_b + at, count);
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) fa[t][i] = load_run<DT>(row_a[i] + at, count);
        }
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) acc[i] = mma16<DT>(fb[t], fa[t][i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) shares[wave][i][lane] = acc[i];
    __syncthreads();
    // 8 consecutive results a thread: row 16 i + r of a, columns 8 g .. + 7 of the 16
    const int i = threadIdx.x >> 5, g = (threadIdx.x >> 4) & 1;
    if (i >= BLOCKS) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) {
        const f32x4 lo = shares[w][i][(2 * g) * 16 + r], hi = shares[w][i][(2 * g + 1) * 16 + r];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += lo[e], v[4 + e] += hi[e];
    }
    const int64_t m = 16 * i + r, n = n0 + 8 * g;
    if (m < a.m && n < a.n) finish_run<DT>(a, m, (int)n, (int)(a.n - n), v);
}

// p = dy * act'(pre), and the columns' sums of it for the bias: 32 threads across, 16 bytes each, 8 rows at a time, one strip of rows a workgroup.  p is rounded
// to the operands' type, as both products take it; the sums are of the unrounded values.  Bound by memory: 12288 x 4096 bf16 (302 MB) with GELU 56 us,
// 5.4 TB/s.  It is a pass of its own because both products read p, one of them across its rows: formed in each, the slope would be worked out again for every tile that reads it.
template <int DT>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a, int64_t strip) {
    typedef typename Elem<DT>::T E;
    constexpr int N = Elem<DT>::N;
    __shared__ float joined[7][32 * N];
    const int place = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int at = ((int)blockIdx.x * 32 + place) * N, count = a.n - at;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    if (count > 0) {
        const int64_t end = min(a.m, (blockIdx.y + 1) * strip);
        auto take = [&](const uint4& raw_dy, const uint4& raw_pre, int64_t m) {
            E y[N], x[N];
            __builtin_memcpy(y, &raw_dy, 16);
            __builtin_memcpy(x, &raw_pre, 16);
            float p[N], v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) p[e] = (float)y[e], v[e] = (float)x[e];
            times_slope<DT != CT_F32>(p, v, a.act);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += p[e];
            if (a.p) store_elems<DT>((E*)a.p + m * a.p_stride + at, N, p);  // what lies behind dy's last element is 0
        };
        const bool slope = a.act != ACT_NONE;
        const E* dy = (const E*)a.dy + at;
        const E* pre = (const E*)a.pre + at;
        int64_t m = blockIdx.y * strip + strand;
        for (; m + 8 < end; m += 16) {  // two rows are asked for at once
            const uint4 y0 = load_run<DT>(dy + m * a.dy_stride, count), y1 = load_run<DT>(dy + (m + 8) * a.dy_stride, count);
            uint4 x0 = {0u, 0u, 0u, 0u}, x1 = x0;
            if (slope) x0 = load_run<DT>(pre + m * a.pre_stride, count), x1 = load_run<DT>(pre + (m + 8) * a.pre_stride, count);
            take(y0, x0, m);
            take(y1, x1, m + 8);
        }
        if (m < end) {
            uint4 x0 = {0u, 0u, 0u, 0u};
            if (slope) x0 = load_run<DT>(pre + m * a.pre_stride, count);
            take(load_run<DT>(dy + m * a.dy_stride, count), x0, m);
        }
    }
    if (!a.partial) return;
    if (strand) {
#pragma unroll
        for (int e = 0; e < N; ++e) joined[strand - 1][e * 32 + place] = sum[e];
    }
    __syncthreads();
    if (strand || count <= 0) return;
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
        for (int s = 0; s < 7; ++s) sum[e] += joined[s][e * 32 + place];
    store_elems<CT_F32, N>(a.partial + blockIdx.y * (int64_t)a.n + at, count, sum);
}

// The sums of columns over the shares that other launches left: 32 columns a workgroup, 32 threads over the shares of each, added in one fixed order, so that a
// gradient has the same bits every time.  768 shares of 2048 columns (6.3 MB): 4.5 us, of which 3.5 are a launch.
template <int WT>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* partial, int64_t groups, int64_t width, int64_t first, void* out, void* more) {
    typedef typename Elem<WT>::T W;
    __shared__ float part[32][33];
    const int strand = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    float sum = 0.f;
    if (column < width) {
#pragma unroll 8
        for (int64_t g = strand; g < groups; g += 32) sum += partial[g * width + column];
    }
    part[strand][threadIdx.x & 31] = sum;
    __syncthreads();
    if (strand == 0 && column < width) {
        for (int i = 1; i < 32; ++i) sum += part[i][threadIdx.x];
        W* to = (W*)(column < first ? out : more);
        if (to) to[column < first ? column : column - first] = (W)sum;
    }
}

// The tile (256 x 256, a workgroup of eight waves a compute unit; or 128 x 128, two or three of four waves) and the number of shares that a product is
// split into, from its sizes alone.
struct Plan {
    int tile, splits;
};
constexpr int64_t round_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
Plan plan_of(int64_t m, int64_t n, int64_t k, int dtype) {
    const int64_t big = round_to(m, 256) / 256 * (round_to(n, 256) / 256), small = round_to(m, 128) / 128 * (round_to(n, 128) / 128);
    const int64_t step = dtype == FNN_F32 ? 16 : 64, steps = (k + step - 1) / step;
    auto most = [&](int64_t tiles, int64_t wanted, int64_t least_steps, int64_t limit) {
        const int64_t splits = std::min(std::min(wanted / std::max(tiles, (int64_t)1), steps / least_steps), limit);
        return std::max(splits, (int64_t)1);
    };
    // The large tiles need less of the operands' traffic per product, and win where they, or up to four long shares of each, keep 160 compute units busy
    // (12288 x 1024 -> 1024: 34 us in 192 large tiles, 36 in 768 small ones; 4096 x 12288 -> 1024: 112 us in 64 large ones of four shares, 117 in 256 small ones of two).
    if (dtype != FNN_F32) {
        const int64_t shares = most(big, 256, 16, 4);
        if (big * shares >= 160) return {256, (int)shares};
    }
    // fp32 products are slow enough that two workgroups a compute unit pay for their shares; 16-bit ones are not (768 x 1024 -> 4096: 15 us in 192 tiles, 25 in 384).
    return {128, (int)most(small, dtype == FNN_F32 ? 512 : 256, 8, 32)};
}
size_t partial_bytes(int64_t m, int64_t n, const Plan& p) {
    return p.splits > 1 ? (size_t)p.splits * round_to(m, p.tile) * round_to(n, p.tile) * sizeof(float) : 0;
}

// Rows on 16-byte boundaries, zeros behind their ends: a thread writes 16 bytes, read from wherever they are.  Bound by memory and, below some MB, the launch:
// 6001 x 1023 bf16 (25 MB) 8.5 us.
template <int DT>
__global__ __launch_bounds__(256) void copy_rows_kernel(const void* from, int64_t from_stride, int64_t rows, int64_t width, void* to, int64_t stride) {
    typedef typename Elem<DT>::T E;
    constexpr int N = Elem<DT>::N;
    const int64_t runs = stride / N, at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / runs;
    if (row >= rows) return;
    const int64_t e = (at - row * runs) * N;
    reinterpret_cast<uint4*>(to)[at] = load_run<DT>((const E*)from + row * from_stride + e, (int)min(width - e, (int64_t)N));
}

// Whether an operand's runs of 16 bytes lie on 16-byte boundaries, a tile's offsets fit 32 bits and k ends with a run.
bool direct(const void* data, int64_t stride, int64_t rows, int64_t k, int dtype, int layout) {
    const int es = dtype == FNN_F32 ? 4 : 2;
    return ((uintptr_t)data & 15) == 0 && (rows < 2 || stride * es % 16 == 0) && stride < ((int64_t)1 << 31) / (256 * es) &&
           (layout == COLUMNS || k * es % 16 == 0);
}

template <int DT, int LA, int LB>
hipError_t run_gemm(GemmArgs a, bool is_direct, const Plan& p, int kind, hipStream_t s) {
    a.tiles_m = (int)(round_to(a.m, p.tile) / p.tile);
    a.tiles_n = (int)(round_to(a.n, p.tile) / p.tile);
    a.splits = p.splits;
    if ((int64_t)a.tiles_m * a.tiles_n * a.splits > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)((int64_t)a.tiles_m * a.tiles_n * a.splits));
    hipError_t e;
    if (DT != CT_F32 && p.tile == 256) {
        if constexpr (DT != CT_F32)
            e = is_direct ? launch(kind, gemm_kernel<DT, 256, 256, 2, 4, 128, 2, LA, LB, true>, grid, dim3(512), 0, s, a)
                          : launch(kind, gemm_kernel<DT, 256, 256, 2, 4, 128, 2, LA, LB, false>, grid, dim3(512), 0, s, a);
    } else {
        constexpr int SB = DT == CT_F32 ? 64 : 128, STAGES = DT == CT_F32 ? 3 : 2;
        e = is_direct ? launch(kind, gemm_kernel<DT, 128, 128, 2, 2, SB, STAGES, LA, LB, true>, grid, dim3(256), 0, s, a)
                      : launch(kind, gemm_kernel<DT, 128, 128, 2, 2, SB, STAGES, LA, LB, false>, grid, dim3(256), 0, s, a);
    }
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t pitch = (int64_t)a.tiles_n * p.tile, share = pitch * a.tiles_m * p.tile, runs = (int64_t)((a.n + 7) / 8) * a.m;
    return launch(kind, gemm_join_kernel<DT>, dim3((unsigned)((runs + 255) / 256)), dim3(256), 0, s, a, pitch, share);
}

template <int DT>
hipError_t run_few_rows(const GemmArgs& a, int kind, hipStream_t s) {
    const dim3 grid((unsigned)((a.n + 15) / 16)), block(FEW_WAVES * 64);
    if (a.m <= 16) return launch(kind, few_rows_kernel<DT, 1>, grid, block, 0, s, a);
    if (a.m <= 32) return launch(kind, few_rows_kernel<DT, 2>, grid, block, 0, s, a);
    return launch(kind, few_rows_kernel<DT, 4>, grid, block, 0, s, a);
}

template <typename F>
hipError_t with_type(int dtype, F f) {
    if (dtype == FNN_F32) return f(std::integral_constant<int, CT_F32>());
    if (dtype == FNN_F16) return f(std::integral_constant<int, CT_F16>());
    return f(std::integral_constant<int, CT_BF16>());
}

}  // namespace

// Microseconds with operands as they are (through registers) and copied, copies included.  Forward, bf16: 12288 x 1023 -> 4095 168 and 124, 12288 x 1001 -> 1001
// 49 and 50, 6001 x 777 -> 1001 30 and 33; fp32: 6001 x 1023 -> 4095 463 and 439, 1531 x 777 -> 1001 44 and 49.  Gradients, whose products read an operand
// across its rows, bf16: 12288 x 1023 -> 4095 733 and 345, 600 x 777 -> 1001 60 and 45, 200 x 501 -> 501 54 and 37, 8 x 1021 -> 4095 41 and 39, 16 x 101 -> 101 24 and
// 27; fp32: 6001 x 777 -> 1001 305 and 271, 1531 x 777 -> 1001 100 and 100, 300 x 777 -> 1001 58 and 60.
bool copies_pay(int64_t m, int64_t n, int64_t k, int64_t width, int dtype, bool backward) {
    if (!backward && few_rows(m, k)) return false;  // that pass takes rows at any address (16 x 20001 -> 40003 fp16: 960 us, 1080 with copies, and no 1.6 GB for them)
    const double least = !backward ? 1.2e10 : dtype == FNN_F32 ? 2e9 : 3e7;
    return width * (dtype == FNN_F32 ? 4 : 2) % 16 != 0 && (double)m * n * k >= least;
}

hipError_t launch_copy_rows(const void* from, int64_t from_stride, int64_t rows, int64_t width, void* to, int64_t stride, int dtype, int kind, hipStream_t s) {
    return with_type(dtype, [&](auto dt) {
        const int64_t runs = rows * (stride / Elem<dt.value>::N);
        return launch(kind, copy_rows_kernel<dt.value>, dim3((unsigned)((runs + 255) / 256)), dim3(256), 0, s, from, from_stride, rows, width, to, stride);
    });
}

size_t gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, int layout_a, int layout_b) {
    if (m < 1 || n < 1) return 0;
    if (layout_a == ROWS && layout_b == ROWS && few_rows(m, k)) return 0;
    return partial_bytes(m, n, plan_of(m, n, k, dtype));
}

hipError_t launch_gemm(GemmArgs a, int dtype, int layout_a, int layout_b, int kind, hipStream_t s) {
    if (a.m < 1 || a.n < 1) return hipSuccess;
    return with_type(dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        if (layout_a == ROWS && layout_b == ROWS && few_rows(a.m, a.k)) return run_few_rows<DT>(a, kind, s);
        const Plan p = plan_of(a.m, a.n, a.k, dtype);
        const bool d = direct(a.a, a.lda, layout_a == ROWS ? a.m : a.k, a.k_a, dtype, layout_a) && direct(a.b, a.ldb, layout_b == ROWS ? a.n : a.k, a.k_b, dtype, layout_b);
        if (layout_a == ROWS && layout_b == ROWS) return run_gemm<DT, ROWS, ROWS>(a, d, p, kind, s);
        if (layout_a == ROWS) return run_gemm<DT, ROWS, COLUMNS>(a, d, p, kind, s);
        return run_gemm<DT, COLUMNS, COLUMNS>(a, d, p, kind, s);
    });
}

int64_t slope_strips(int64_t m, int64_t n) {
    const int64_t across = (n + 255) / 256, wanted = 2048 / (across < 1 ? 1 : across), most = (m + 15) / 16;
    const int64_t strips = wanted < most ? wanted : most;
    return strips < 1 ? 1 : strips;
}

hipError_t launch_slope(const SlopeArgs& a, int dtype, hipStream_t s) {
    const int64_t strips = slope_strips(a.m, a.n), strip = (a.m + strips - 1) / strips;
    return with_type(dtype, [&](auto dt) {
        constexpr int per = 32 * Elem<dt.value>::N;
        return launch(TK_LINEAR_BACKWARD, slope_kernel<dt.value>, dim3((unsigned)((a.n + per - 1) / per), (unsigned)strips), dim3(256), 0, s, a, strip);
    });
}

hipError_t launch_column_sums(const float* partial, int64_t groups, int64_t width, int64_t first, void* out, void* more, int dtype, int kind, hipStream_t s) {
    return with_type(dtype, [&](auto dt) {
        return launch(kind, column_sums_kernel<dt.value>, dim3((unsigned)((width + 31) / 32)), dim3(1024), 0, s, partial, groups, width, first, out, more);
    });
}

}  // namespace fnn
