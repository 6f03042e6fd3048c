// Linear layers with their epilogue, and what their gradients need beside matrix products (fnn_linear, fnn_linear_backward).
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
// lane asks for all of its runs of four turns before it multiplies the first; a (its rows are few) comes out of the L2.
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

// p = dy * act'(pre): 256 columns a workgroup (two types: 8 elements a thread), 8 rows at a time, strip after strip of rows.
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
        for (int64_t m = blockIdx.y * strip + strand; m < end; m += 8) {
            float p[N];
            load_elems<DT>((const E*)a.dy + m * a.dy_stride + at, count, p);
            if (a.act != ACT_NONE) {
                float x[N];
                load_elems<DT>((const E*)a.pre + m * a.pre_stride + at, count, x);
                times_slope<DT != CT_F32>(p, x, a.act);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += p[e];
            if (a.p) store_elems<DT>((E*)a.p + m * a.p_stride + at, count, p);
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

// 32 columns a workgroup, 32 threads over the shares of each.
template <int WT>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* partial, int64_t groups, int64_t width, int64_t first, void* out, void* more) {
    typedef typename Elem<WT>::T W;
    __shared__ float part[32][33];
    const int strand = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
    float sum = 0.f;
    if (column < width)
        for (int64_t g = strand; g < groups; g += 32) sum += partial[g * width + column];
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
    const bool whole = dtype != FNN_F32 && big >= 160;
    const int64_t tiles = whole ? big : small, wanted = dtype == FNN_F32 ? 512 : 256, step = dtype == FNN_F32 ? 16 : 64;
    const int64_t steps = (k + step - 1) / step;
    int64_t splits = wanted / (tiles > 0 ? tiles : 1);
    if (splits > steps / 8) splits = steps / 8;
    if (splits > 32) splits = 32;
    return {whole ? 256 : 128, splits < 1 ? 1 : (int)splits};
}
size_t partial_bytes(int64_t m, int64_t n, const Plan& p) {
    return p.splits > 1 ? (size_t)p.splits * round_to(m, p.tile) * round_to(n, p.tile) * sizeof(float) : 0;
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
        const bool d = direct(a.a, a.lda, layout_a == ROWS ? a.m : a.k, a.k, dtype, layout_a) && direct(a.b, a.ldb, layout_b == ROWS ? a.n : a.k, a.k, dtype, layout_b);
        if (layout_a == ROWS && layout_b == ROWS) return run_gemm<DT, ROWS, ROWS>(a, d, p, kind, s);
        if (layout_a == ROWS) return run_gemm<DT, ROWS, COLUMNS>(a, d, p, kind, s);
        return run_gemm<DT, COLUMNS, COLUMNS>(a, d, p, kind, s);
    });
}

int64_t slope_strips(int64_t m, int64_t n) {
    const int64_t across = (n + 255) / 256, wanted = 1024 / (across < 1 ? 1 : across), most = (m + 31) / 32;
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
