// The matrix product behind the linear layers: C[m][n] = sum over k of A(m, k) B(n, k), fp32 sums, on tiles that workgroups stage in LDS.
#pragma once
#include "net_device.hpp"
#include "net_kernels.hpp"

namespace fnn {

// How an operand lies in memory: its rows run along k, or its rows are the k's and run along m (n).
enum : int { ROWS = 0, COLUMNS = 1 };

// Who works on what: neighbouring workgroups are dealt to the 8 XCDs in turn, so each XCD is given a run of tiles of its own, in blocks
// of 8 tiles of rows by as many tiles of columns as it takes, which share their operands in its L2.
struct TileAt {
    int m, n, split;
};
__device__ __forceinline__ TileAt tile_at(const GemmArgs& a) {
    const int per = a.tiles_m * a.tiles_n, total = per * a.splits, id = blockIdx.x;
    const int xcd = id & 7, q = total >> 3, r = total & 7;
    const int mine = xcd * q + min(xcd, r) + (id >> 3);
    TileAt t;
    t.split = mine / per;
    const int i = mine - t.split * per;
    const int block = i / (8 * a.tiles_n), first = block * 8, tall = min(8, a.tiles_m - first);
    const int j = i - block * 8 * a.tiles_n;
    t.m = first + j % tall;
    t.n = j / tall;
    return t;
}

// One operand's tile of T rows (columns) and one step of k (SB bytes of a row), in LDS.  ROWS: [T][SB]; COLUMNS: [k][T].  LDS serves 256 bytes at a
// time, so the 16-byte runs of a row are exchanged such that what one instruction reads together lies in different columns of 256
// bytes: 16 rows at one run (ROWS), 4 rows at 4 runs (COLUMNS of 16 bits, transposing reads), rows k and k + 4 at 128 bytes (COLUMNS of 32 bits).
template <int DT, int T, int SB, int THREADS, int LAYOUT>
struct Operand {
    typedef typename Elem<DT>::T E;
    static constexpr int ES = sizeof(E), N = Elem<DT>::N, STEP = SB / ES, BYTES = T * SB;
    static constexpr int RUNS = BYTES / 16, PER_THREAD = RUNS / THREADS;
    static constexpr int ROW_RUNS = LAYOUT == ROWS ? SB / 16 : T * ES / 16;  // 16-byte runs in a row of the tile
    static_assert(RUNS % THREADS == 0 && THREADS % ROW_RUNS == 0, "every thread's runs are at one place of their rows");
    static constexpr int ROWS_APART = THREADS / ROW_RUNS;
    static __device__ __forceinline__ int exchanged(int row) { return LAYOUT == ROWS ? (SB == 64 ? row >> 2 & 3 : row >> 1 & 7) : ES == 2 ? (row & 3) << 2 : (row >> 2 & 1) << 3; }

    const E* base;      // ROWS: the tile's first row, at the first k of the split; COLUMNS: the first k's row, at the tile's first column
    int64_t stride;     // elements
    int have;           // rows (columns) of the tile that exist
    uint32_t offset;    // this thread's first run, in bytes from base
    uint32_t apart;     // and how far its next one is
    int col;            // element at which its runs start within the row

    __device__ __forceinline__ void begin(const void* data, int64_t stride_, int64_t first, int64_t total, int64_t k0) {
        stride = stride_;
        const int row = threadIdx.x / ROW_RUNS, run = (threadIdx.x % ROW_RUNS) ^ exchanged(row);
        static_assert(ROWS_APART % (LAYOUT == ROWS ? 16 : ES == 2 ? 4 : 8) == 0, "the exchange is the same for all of a thread's runs");
        col = run * N;
        have = (int)min((int64_t)T, total - first);
        base = (const E*)data + (LAYOUT == ROWS ? first * stride + k0 : k0 * stride + first);
        offset = (uint32_t)((row * stride + col) * ES);
        apart = (uint32_t)(ROWS_APART * stride * ES);
    }

    // Direct loads to LDS through a buffer that ends with the operand, so that what lies behind it arrives as zero: rows past the last, and
    // (ROWS) runs past the end of k, whose lanes ask for what lies behind.  `left`: k's from `base` on.
    __device__ __forceinline__ void stage(char* lds, int left) const {
        const int64_t rows = LAYOUT == ROWS ? have : min(left, STEP), width = LAYOUT == ROWS ? left : have;
        const uint32_t bytes = (uint32_t)((((rows - 1) * stride + width) * ES + 3) & ~(int64_t)3);
        const i32x4 buffer = buffer_of(base, bytes);
        const bool there = col < (LAYOUT == ROWS ? left : have);
        const uint32_t to = lds_address(lds) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) load_to_lds(buffer, there ? offset + i * apart : 0xFFFFFFF0u, to + i * THREADS * 16);
    }
    // The same for any alignment and any number of k's, through registers.
    __device__ __forceinline__ void fetch(uint4 (&held)[PER_THREAD], int left) const {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int row = threadIdx.x / ROW_RUNS + i * ROWS_APART;
            const int rows = LAYOUT == ROWS ? have : min(left, STEP), width = LAYOUT == ROWS ? left : have;
            held[i] = row < rows ? load_run<DT>(base + row * stride + col, width - col) : uint4{0u, 0u, 0u, 0u};
        }
    }
    __device__ __forceinline__ void put(char* lds, const uint4 (&held)[PER_THREAD]) const {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) *reinterpret_cast<uint4*>(lds + (i * THREADS + threadIdx.x) * 16) = held[i];
    }
    __device__ __forceinline__ void advance() { base += LAYOUT == ROWS ? (int64_t)STEP : STEP * stride; }

    // A matrix instruction's operand: rows 32 block .. + 31, the kk-th 32 bytes of the step's k's.
    static __device__ __forceinline__ uint4 fragment(const char* lds, int block, int kk, int lane) {
        const int c = lane & 31, h = lane >> 5;
        if constexpr (LAYOUT == ROWS) {
            return *reinterpret_cast<const uint4*>(lds + block * (32 * SB) + c * SB + (((2 * kk + h) ^ exchanged(c)) << 4));
        } else if constexpr (ES == 2) {
            const int t = lane & 15, row = 16 * kk + 8 * h + (t >> 2);
            const int run = (4 * block + 2 * ((lane >> 4) & 1) + ((t >> 1) & 1)) ^ ((t >> 2) << 2);
            const char* at = lds + row * (T * ES) + run * 16 + (t & 1) * 8;
            const uint2 lo = read_transposed(at), hi = read_transposed(at + 4 * T * ES);
            return {lo.x, lo.y, hi.x, hi.y};
        } else {
            const char* at = lds + (8 * kk + 4 * h) * (T * ES) + (((8 * block + (c >> 2)) ^ (h << 3)) << 4) + (c & 3) * 4;
            uint4 v;
            v.x = *reinterpret_cast<const uint32_t*>(at);
            v.y = *reinterpret_cast<const uint32_t*>(at + T * ES);
            v.z = *reinterpret_cast<const uint32_t*>(at + 2 * T * ES);
            v.w = *reinterpret_cast<const uint32_t*>(at + 3 * T * ES);
            return v;
        }
    }
};

// Eight consecutive elements, as stored: `count` of them exist.
template <int DT>
struct Eight {
    static constexpr int N = Elem<DT>::N;
    uint4 raw[8 / N];
    __device__ __forceinline__ void load(const void* data, int64_t at, int count) {
#pragma unroll
        for (int p = 0; p < 8 / N; ++p) raw[p] = load_run<DT>((const typename Elem<DT>::T*)data + at + p * N, count - p * N);
    }
    __device__ __forceinline__ float operator[](int e) const {
        typename Elem<DT>::T x[N];
        __builtin_memcpy(x, &raw[e / N], 16);
        return (float)x[e % N];
    }
};
template <int DT>
__device__ __forceinline__ void store_eight(void* data, int64_t at, int count, const float (&v)[8]) {
    constexpr int N = Elem<DT>::N;
#pragma unroll
    for (int p = 0; p < 8 / N; ++p) {
        if (count <= p * N) return;
        float w[N];
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = v[p * N + e];
        store_elems<DT>((typename Elem<DT>::T*)data + at + p * N, count - p * N, w);
    }
}

// Eight consecutive results of row m, from column n on (`count` of them exist): bias, activation, residual.
template <int DT>
__device__ __forceinline__ void finish_run(const GemmArgs& a, int64_t m, int n, int count, float (&v)[8], const Eight<DT>& bias, const Eight<DT>& residual) {
    if (a.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += bias[e];
    }
    if (a.pre) store_eight<DT>(a.pre, m * a.ldp + n, count, v);
    activate<DT != CT_F32>(v, a.act);
    if (a.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += residual[e];
    }
    store_eight<DT>(a.y, m * a.ldy + n, count, v);
}
// The same where what it takes is not there yet.
template <int DT>
__device__ __forceinline__ void finish_run(const GemmArgs& a, int64_t m, int n, int count, float (&v)[8]) {
    Eight<DT> bias = {}, residual = {};
    if (a.bias) bias.load(a.bias, n, count);
    if (a.residual) residual.load(a.residual, m * a.ldr + n, count);
    finish_run<DT>(a, m, n, count, v, bias, residual);
}

// A workgroup's tile of TM x TN results, a wave's 128 x 64 or 64 x 64 of it in registers.  Per 128-byte step of k a tile of 256 x 256 stages 64 KB and has 64 products
// a wave, two of whose operands come from LDS for every eight (large) or four (small) products; results leave through LDS, with the epilogue on the way.  What
// bounds it: large products the matrix instructions at the power limit and the loads that do not quite hide behind them (4096 x 4096 -> 4096 fp16 115 us,
// 1195 TFLOP/s, 87 % of the library's rate there; 12288 x 1024 -> 4096 with GELU 127 us, 810 TFLOP/s, some 20 us of them GELU); those of fewer
// tiles than compute units the latency of a step.  fp32 1531 x 777 -> 1001: 43 us for 2.4 GFLOP, the latency of loads through registers.
// Measured and slower or no faster: four stages of 64 bytes, loads spread between the products, operands asked for in the order of k rotated from tile to
// tile, two half-workgroups taking turns at loads and products, tiles of 256 x 128.
template <int DT, int TM, int TN, int WAVES_M, int WAVES_N, int SB, int STAGES, int LA, int LB, bool DIRECT>
__global__ __launch_bounds__(WAVES_M* WAVES_N * 64, 512 / (WAVES_M * WAVES_N * 64)) void gemm_kernel(GemmArgs a) {
    constexpr int THREADS = WAVES_M * WAVES_N * 64, BM = TM / WAVES_M / 32, BN = TN / WAVES_N / 32, PARTS = SB / 32;
    using OpA = Operand<DT, TM, SB, THREADS, LA>;
    using OpB = Operand<DT, TN, SB, THREADS, LB>;
    __shared__ __attribute__((aligned(16))) char stages[STAGES][OpA::BYTES + OpB::BYTES];
    const TileAt tile = tile_at(a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WAVES_M, wn = wave / WAVES_M;
    const int steps = (a.k + OpA::STEP - 1) / OpA::STEP;
    const int s0 = (int)((int64_t)steps * tile.split / a.splits), s1 = (int)((int64_t)steps * (tile.split + 1) / a.splits);
    const int64_t m0 = (int64_t)tile.m * TM;
    const int n0 = tile.n * TN;
    OpA opa;
    OpB opb;
    opa.begin(a.a, a.lda, m0, a.m, (int64_t)s0 * OpA::STEP);
    opb.begin(a.b, a.ldb, n0, a.n, (int64_t)s0 * OpA::STEP);
    int done = s0 * OpA::STEP;
    const int n = n0 + wn * 64 + 8 * (lane & 7);  // the first of the eight columns that this lane finishes
    Eight<DT> bias = {};
    if (a.bias && a.splits == 1) bias.load(a.bias, n, a.n - n);

    f32x16 acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = (f32x16)(0.f);

    uint4 held_a[DIRECT ? 1 : OpA::PER_THREAD], held_b[DIRECT ? 1 : OpB::PER_THREAD];
    auto get = [&](char* to) {
        if constexpr (DIRECT) {
            opa.stage(to, (LA == ROWS ? a.k_a : a.k) - done);
            opb.stage(to + OpA::BYTES, (LB == ROWS ? a.k_b : a.k) - done);
        } else {
            opa.fetch(held_a, a.k - done);
            opb.fetch(held_b, a.k - done);
        }
        opa.advance();
        opb.advance();
        done += OpA::STEP;
    };
    auto put = [&](char* to) {
        if constexpr (!DIRECT) {
            opa.put(to, held_a);
            opb.put(to + OpA::BYTES, held_b);
        }
    };
    uint4 fa[2][BM], fb[2][BN];
    auto read = [&](const char* from, int kk) {
#pragma unroll
        for (int j = 0; j < BN; ++j) fb[kk & 1][j] = OpB::fragment(from + OpA::BYTES, wn * BN + j, kk, lane);
#pragma unroll
        for (int i = 0; i < BM; ++i) fa[kk & 1][i] = OpA::fragment(from, wm * BM + i, kk, lane);
    };
    // the first part's operands have been read; each next part's are while one is multiplied
    auto multiply = [&](const char* from) {
#pragma unroll
        for (int kk = 0; kk < PARTS; ++kk) {
            if (kk + 1 < PARTS) read(from, kk + 1);
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) acc[i][j] = mma32<DT>(fb[kk & 1][j], fa[kk & 1][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // A step: what was asked for STAGES - 1 steps ago has arrived, in every wave; the stage that everyone has left is filled; this one is multiplied.
    constexpr int LOADS = OpA::PER_THREAD + OpB::PER_THREAD;
    auto step = [&](int stage, int s) {
        const int later = s1 - 1 - s;  // steps whose loads may still be under way
        if (STAGES >= 3 && later >= 1) lds_loads_left<LOADS>();
        else lds_loads_left<0>();
        meet();
        read(stages[stage], 0);
        if (s + STAGES - 1 < s1) get(stages[(stage + STAGES - 1) % STAGES]);
        multiply(stages[stage]);
    };
    if constexpr (DIRECT) {
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (s0 + i < s1) get(stages[i]);
        for (int s = s0; s < s1; s += STAGES) {
#pragma unroll
            for (int i = 0; i < STAGES; ++i)
                if (s + i < s1) step(i, s + i);
        }
    } else {
        // one step ahead: stage s mod 2
        if (s0 < s1) {
            get(nullptr);
            put(stages[0]);
        }
        for (int s = s0; s < s1; ++s) {
            __syncthreads();
            const bool more = s + 1 < s1;
            read(stages[(s - s0) & 1], 0);
            if (more) get(nullptr);
            multiply(stages[(s - s0) & 1]);
            if (more) put(stages[(s - s0 + 1) & 1]);
        }
    }

    // The results go through LDS, 32 rows of a wave at a time, so that 8 lanes have 64 consecutive columns of a row: whole lines of y, residual and
    // pre instead of 32-byte pieces of 32 rows.  As in the tiles, the runs of a row are exchanged by its number.  Loads are waited for in
    // the order of all accesses, stores among them, so the bias is there before the first store and each 32 rows' residual before
    // those of the rows before it (bias loaded where it is added: 12 us longer on a tile of 256 x 256).
    __syncthreads();
    static_assert(BN == 2 && WAVES_M * WAVES_N * 8192 <= sizeof(stages), "a wave's 32 rows have 64 columns and 8 KB");
    char* mine = &stages[0][0] + wave * 8192;
    const int c = lane & 31, h = lane >> 5;
    const bool whole = a.splits == 1;
    auto row_of = [&](int i, int part) { return m0 + (wm * BM + i) * 32 + 8 * part + (lane >> 3); };
    Eight<DT> residual[2][4] = {};
    auto fetch_residual = [&](int i) {
        if (!a.residual || !whole) return;
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            const int64_t m = row_of(i, part);
            if (m < a.m) residual[i & 1][part].load(a.residual, m * a.ldr + n, a.n - n);
        }
    };
    fetch_residual(0);
#pragma unroll
    for (int i = 0; i < BM; ++i) {
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(mine + c * 256 + (((8 * j + 2 * g + h) ^ (c & 15)) << 4)) =
                    f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        __builtin_amdgcn_wave_barrier();
        if (i + 1 < BM) fetch_residual(i + 1);
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            const int row = 8 * part + (lane >> 3);
            const int64_t m = row_of(i, part);
            float v[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + row * 256 + (((2 * (lane & 7) + e) ^ (row & 15)) << 4));
                v[4 * e] = x[0], v[4 * e + 1] = x[1], v[4 * e + 2] = x[2], v[4 * e + 3] = x[3];
            }
            if (m >= a.m || n >= a.n) continue;
            if (whole) {
                finish_run<DT>(a, m, n, a.n - n, v, bias, residual[i & 1][part]);
            } else {
                // shares lie in whole tiles, so they need no edge
                float* to = a.partial + (((int64_t)tile.split * a.tiles_m * TM + m) * a.tiles_n * TN + n);
                reinterpret_cast<f32x4*>(to)[0] = f32x4{v[0], v[1], v[2], v[3]};
                reinterpret_cast<f32x4*>(to)[1] = f32x4{v[4], v[5], v[6], v[7]};
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The shares of a split product, added up in the order of k, so that the result does not depend on which workgroup ended first; the epilogue is here then.  Bound
// by memory: 1024 x 4096 in four shares (67 MB written by the product, still in the caches) 12 us.
template <int DT>
__global__ __launch_bounds__(256) void gemm_join_kernel(GemmArgs a, int64_t pitch, int64_t share) {
    const int64_t runs = (a.n + 7) / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= runs * a.m) return;
    const int64_t m = at / runs;
    const int n = (int)(at - m * runs) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; ++s) {
        const f32x4* from = reinterpret_cast<const f32x4*>(a.partial + s * share + m * pitch + n);
        const f32x4 lo = from[0], hi = from[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += lo[e], v[4 + e] += hi[e];
    }
    finish_run<DT>(a, m, n, a.n - n, v);
}

}  // namespace fnn
