// The matrix product behind the linear layers: C[m][n] = sum over k of A(m, k) B(n, k), fp32 sums, on tiles that workgroups stage in LDS.
#pragma once
#include "net_device.hpp"
#include "net_kernels.hpp"

namespace fnn {

// How an operand lies in memory: its rows run along k, or its rows are the k's and run along m (n).
enum : int { ROWS = 0, COLUMNS = 1 };

constexpr int STEP_BYTES = 64;  // of every row of a tile, per step: 32 elements of 16 bits, 16 of 32
constexpr int STAGES = 3;

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

// One operand's tile of T rows (columns) and one step of k, in LDS.  ROWS: [T][64 bytes]; COLUMNS: [k][T].  LDS serves 256 bytes at a time, so
// the 16-byte runs of a row are exchanged such that what one instruction reads together lies in different columns of 256 bytes: 16 rows
// at one run (ROWS), 4 rows at 4 runs (COLUMNS of 16 bits, transposing reads), rows k and k + 4 at 128 bytes (COLUMNS of 32 bits).
template <int DT, int T, int THREADS, int LAYOUT>
struct Operand {
    typedef typename Elem<DT>::T E;
    static constexpr int ES = sizeof(E), N = Elem<DT>::N, STEP = STEP_BYTES / ES;
    static constexpr int RUNS = T * 4, PER_THREAD = RUNS / THREADS;
    static constexpr int ROW_RUNS = LAYOUT == ROWS ? 4 : T * ES / 16;  // 16-byte runs in a row of the tile
    static_assert(RUNS % THREADS == 0 && THREADS % ROW_RUNS == 0, "every thread's runs are at one place of their rows");
    static constexpr int ROWS_APART = THREADS / ROW_RUNS;
    static __device__ __forceinline__ int exchanged(int row) { return LAYOUT == ROWS ? (row >> 2 & 3) : ES == 2 ? (row & 3) << 2 : (row >> 2 & 1) << 3; }

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

    // A matrix instruction's operand: rows 32 block .. + 31, the kk-th half of the step's k's.
    static __device__ __forceinline__ uint4 fragment(const char* lds, int block, int kk, int lane) {
        const int c = lane & 31, h = lane >> 5;
        if constexpr (LAYOUT == ROWS) {
            return *reinterpret_cast<const uint4*>(lds + block * (32 * STEP_BYTES) + c * STEP_BYTES + (((2 * kk + h) ^ (c >> 2 & 3)) << 4));
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

// Eight consecutive results of row m, from column n on (`count` of them exist): bias, activation, residual; or, of a split product, the share.
template <int DT>
__device__ __forceinline__ void finish_run(const GemmArgs& a, int64_t m, int n, int count, float (&v)[8]) {
    typedef typename Elem<DT>::T E;
    constexpr int N = Elem<DT>::N;
#pragma unroll
    for (int part = 0; part < 8 / N; ++part) {
        const int at = n + part * N, here = count - part * N;
        float w[N];
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = v[part * N + e];
        if (here <= 0) return;
        if (a.bias) {
            float b[N];
            load_elems<DT>((const E*)a.bias + at, here, b);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] += b[e];
        }
        if (a.pre) store_elems<DT>((E*)a.pre + m * a.ldp + at, here, w);
        activate<DT != CT_F32>(w, a.act);
        if (a.residual) {
            float r[N];
            load_elems<DT>((const E*)a.residual + m * a.ldr + at, here, r);
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] += r[e];
        }
        store_elems<DT>((E*)a.y + m * a.ldy + at, here, w);
    }
}

template <int DT, int TM, int TN, int WAVES_M, int WAVES_N, int LA, int LB, bool DIRECT>
__global__ __launch_bounds__(WAVES_M* WAVES_N * 64, 2) void gemm_kernel(GemmArgs a) {
    constexpr int THREADS = WAVES_M * WAVES_N * 64, BM = TM / WAVES_M / 32, BN = TN / WAVES_N / 32;
    using OpA = Operand<DT, TM, THREADS, LA>;
    using OpB = Operand<DT, TN, THREADS, LB>;
    __shared__ __attribute__((aligned(16))) char stages[STAGES][(TM + TN) * STEP_BYTES];
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
    int left = a.k - s0 * OpA::STEP;

    f32x16 acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = (f32x16)(0.f);

    uint4 held_a[DIRECT ? 1 : OpA::PER_THREAD], held_b[DIRECT ? 1 : OpB::PER_THREAD];
    auto get = [&](char* to) {
        if constexpr (DIRECT) {
            opa.stage(to, left);
            opb.stage(to + TM * STEP_BYTES, left);
        } else {
            opa.fetch(held_a, left);
            opb.fetch(held_b, left);
        }
        opa.advance();
        opb.advance();
        left -= OpA::STEP;
    };
    auto put = [&](char* to) {
        if constexpr (!DIRECT) {
            opa.put(to, held_a);
            opb.put(to + TM * STEP_BYTES, held_b);
        }
    };
    uint4 fa[2][BM], fb[2][BN];
    auto read = [&](const char* from, int kk) {
#pragma unroll
        for (int j = 0; j < BN; ++j) fb[kk][j] = OpB::fragment(from + TM * STEP_BYTES, wn * BN + j, kk, lane);
#pragma unroll
        for (int i = 0; i < BM; ++i) fa[kk][i] = OpA::fragment(from, wm * BM + i, kk, lane);
    };
    // the first half's operands have been read; the second's are while the first half is multiplied
    auto multiply = [&](const char* from) {
        read(from, 1);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) acc[i][j] = mma32<DT>(fb[kk][j], fa[kk][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // A step: what was asked for two steps ago has arrived, in every wave; the stage that everyone has left is filled; this one is multiplied.
    auto step = [&](int stage, int s) {
        char* now = stages[stage];
        char* next = stages[(stage + 2) % STAGES];
        if (s + 1 < s1) lds_loads_left<OpA::PER_THREAD + OpB::PER_THREAD>();
        else lds_loads_left<0>();
        meet();
        read(now, 0);
        if (s + 2 < s1) get(next);
        multiply(now);
    };
    if constexpr (DIRECT) {
        if (s0 < s1) get(stages[0]);
        if (s0 + 1 < s1) get(stages[1]);
        for (int s = s0; s < s1; s += 3) {
            step(0, s);
            if (s + 1 < s1) step(1, s + 1);
            if (s + 2 < s1) step(2, s + 2);
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
    // pre instead of 32-byte pieces of 32 rows.  As in the tiles, the runs of a row are exchanged by its number.
    __syncthreads();
    static_assert(BN == 2 && 4 * 8192 <= sizeof(stages), "a wave's 32 rows have 64 columns and 8 KB");
    char* mine = &stages[0][0] + wave * 8192;
    const int c = lane & 31, h = lane >> 5, n = n0 + wn * 64 + 8 * (lane & 7);
#pragma unroll
    for (int i = 0; i < BM; ++i) {
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(mine + c * 256 + (((8 * j + 2 * g + h) ^ (c & 15)) << 4)) =
                    f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            const int row = 8 * part + (lane >> 3);
            const int64_t m = m0 + (wm * BM + i) * 32 + row;
            float v[8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + row * 256 + (((2 * (lane & 7) + e) ^ (row & 15)) << 4));
                v[4 * e] = x[0], v[4 * e + 1] = x[1], v[4 * e + 2] = x[2], v[4 * e + 3] = x[3];
            }
            if (m >= a.m || n >= a.n) continue;
            if (a.splits > 1) {
                // shares lie in whole tiles, so they need no edge
                float* to = a.partial + (((int64_t)tile.split * a.tiles_m * TM + m) * a.tiles_n * TN + n);
                reinterpret_cast<f32x4*>(to)[0] = f32x4{v[0], v[1], v[2], v[3]};
                reinterpret_cast<f32x4*>(to)[1] = f32x4{v[4], v[5], v[6], v[7]};
            } else {
                finish_run<DT>(a, m, n, a.n - n, v);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The shares of a split product, added up in the order of k.
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
