// Matrix products of operands in 8 bits with a scale for each block of 128, behind fnn_linear_e4m3 and its gradient.
//
// C[m][n] = sum over the blocks b of k of scale_a(m, b) scale_b(n, b) sum over b of A(m, k) B(n, k): a step of the loop is one block, whose products are summed
// by the matrix instructions from zero and then added, times the two scales, to the fp32 sums in registers.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "e4m3_device.hpp"
#include "gemm.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// A lane's 32 codes of one row of a block, as two runs of 16.
struct Codes {
    uint4 run[2];
};

// Eight codes as bf16, which has every value of e4m3.
__device__ __forceinline__ uint4 widened(uint32_t low, uint32_t high) {
    typedef __bf16 two __attribute__((ext_vector_type(2)));
    uint4 v;
    v.x = __builtin_bit_cast(uint32_t, (two)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.f, false));
    v.y = __builtin_bit_cast(uint32_t, (two)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.f, true));
    v.z = __builtin_bit_cast(uint32_t, (two)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.f, false));
    v.w = __builtin_bit_cast(uint32_t, (two)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.f, true));
    return v;
}

// The products of 16 rows of a and 16 of b over one block of 128: lane (r = lane & 15, q = lane >> 4) holds 32 of the codes of row r, the same ones of both operands;
// result v belongs to row 4 q + v of a and row r of b.
//
// For 16-bit results by the instruction for 8 bits (4.8 PFLOP/s on this card, twice the 16-bit ones).  It sums eight products at a time after cutting each at 2^-13 of the power of two
// of the largest among them, and the sixteen sums in fp32: 1.4e-5 of the result's size on normal values, where the result's own rounding is 2^-12 (fp16) or 2^-9 (bf16)
// and that of its operands 2^-4.  fp32 results take the codes widened to bf16, whose products are exact and summed in fp32, at half the rate.
template <bool WIDE>
__device__ __forceinline__ f32x4 block_product(const Codes& a, const Codes& b) {
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) {
        f32x4 t = zero;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            t = mma16<CT_BF16>(widened(a.run[h].x, a.run[h].y), widened(b.run[h].x, b.run[h].y), t);
            t = mma16<CT_BF16>(widened(a.run[h].z, a.run[h].w), widened(b.run[h].z, b.run[h].w), t);
        }
        return t;
    } else {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, a), __builtin_bit_cast(i32x8, b), zero, 0, 0, 0, 0, 0, 0);
    }
}

// ---- few rows ----

// Whether a product is a pass over b with all of a in registers: up to 16 rows always, up to 32 while a, which every workgroup reads whole, is small.  (Microseconds, this way and in
// tiles: 32 x 1024 -> 4096 4.2 and 6.0, 48 x 1024 -> 4096 5.5 and 6.0, 48 x 512 -> 8192 7.0 and 4.7, 24 x 4096 -> 1024 7.5 and 8.6.)
bool few_rows(int64_t m, int64_t k) { return m <= 16 || (m <= 32 && m * k <= 98304); }
constexpr int FEW_WAVES = 8;

// Few rows of a: the time is that of reading b once.  A workgroup takes 16 rows of b, its waves share the blocks of k between them, and a lane asks for all of
// its runs of TURNS blocks before it multiplies the first, but for the partial run of a row whose length is no multiple of 16, whose codes come one by one (load_run).  The shares are joined in LDS in
// the order of the waves.  1 x 1024 -> 4096 bf16 (4.2 MB): 4.1 us, with GELU 4.2-4.9, most of it a launch and one latency of memory; 1 x 1023 -> 4096 5.2.
template <int DT, int BLOCKS>
__global__ __launch_bounds__(FEW_WAVES * 64) void few_rows_e4m3_kernel(ScaledGemmArgs s, uint32_t first_group) {
    constexpr int TURNS = 2;
    __shared__ f32x4 shares[FEW_WAVES][BLOCKS][64];
    const GemmArgs& a = s.g;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)(first_group + blockIdx.x) * 16;
    const uint8_t* row_b = (const uint8_t*)a.b + min(n0 + r, (int64_t)a.n - 1) * a.ldb;
    const uint8_t* row_a[BLOCKS];
    const float* scale_a[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
        const int64_t row = min((int64_t)(16 * i + r), a.m - 1);
        row_a[i] = (const uint8_t*)a.a + row * a.lda;
        scale_a[i] = s.scale_a + (row >> s.shift_a) * s.sa_row;
    }
    const float* scale_b[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) scale_b[v] = s.scale_b + (min(n0 + 4 * q + v, (int64_t)a.n - 1) >> s.shift_b) * s.sb_row;
    f32x4 acc[BLOCKS];
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) acc[i] = (f32x4)(0.f);
    const int blocks = (int)scaled_blocks(a.k);
    for (int first = wave; first < blocks; first += FEW_WAVES * TURNS) {
        Codes fb[TURNS], fa[TURNS][BLOCKS];
        float sa[TURNS][BLOCKS], sb[TURNS][4];
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int block = first + t * FEW_WAVES;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t at = (int64_t)block * SCALED_BLOCK + (4 * h + q) * 16;
                const int count = (int)min((int64_t)a.k - at, (int64_t)16);
                fb[t].run[h] = load_run<CT_E4M3>(row_b + at, count);
#pragma unroll
                for (int i = 0; i < BLOCKS; ++i) fa[t][i].run[h] = load_run<CT_E4M3>(row_a[i] + at, count);
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) sb[t][v] = block < blocks ? scale_b[v][block * s.sb_block] : 0.f;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) sa[t][i] = block < blocks ? scale_a[i][block * s.sa_block] : 0.f;
        }
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) {
                const f32x4 product = block_product<DT == CT_F32>(fb[t], fa[t][i]);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][v] = __builtin_fmaf(product[v], sa[t][i] * sb[t][v], acc[i][v]);
            }
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

// ---- tiles ----

// finish_run of fewer than eight results, one after the other: there is one such place in a row at most, and in line they would be most of the kernel's code.  Each result waits for its bias, its residual
// and the store before it, which shows in large tiles: 24576 x 1024 -> 4095 bf16 194 us, with bias and residual 332, where 4096 columns take 122 and 200; 1531 x 777 -> 1007 fp32 with residual 16.9, 1008 13.0.
template <int DT>
__device__ __forceinline__ void finish_few(const GemmArgs& a, int64_t m, int n, int count, float (&v)[8]) {
    typedef typename Elem<DT>::T E;
#pragma unroll 1
    for (int e = 0; e < count; ++e) {
        float x[1] = {v[0]};
#pragma unroll
        for (int i = 0; i < 7; ++i) v[i] = v[i + 1];
        if (a.bias) x[0] += (float)((const E*)a.bias)[n + e];
        if (a.pre) ((E*)a.pre)[m * a.ldp + n + e] = (E)x[0];
        activate<DT != CT_F32>(x, a.act);
        if (a.residual) x[0] += (float)((const E*)a.residual)[m * a.ldr + n + e];
        ((E*)a.y)[m * a.ldy + n + e] = (E)x[0];
    }
}

// A mask of the first `count` bytes of a word.
__device__ __forceinline__ uint32_t first_bytes(int count) { return count >= 4 ? 0xFFFFFFFFu : count <= 0 ? 0u : (1u << (8 * count)) - 1u; }

// Clears a row of a step in LDS from its `left`-th code on.
__device__ __forceinline__ void clear_behind(char* row, int exchanged, int left) {
#pragma unroll 1
    for (int run = left / 16; run < SCALED_BLOCK / 16; ++run) {
        uint4* at = reinterpret_cast<uint4*>(row + ((run ^ exchanged) << 4));
        const int count = left - run * 16;
        uint4 codes = *at;
        codes.x &= first_bytes(count);
        codes.y &= first_bytes(count - 4);
        codes.z &= first_bytes(count - 8);
        codes.w &= first_bytes(count - 12);
        *at = codes;
    }
}

// f(0), f(1), .. f(N - 1), the numbers as types.
template <int N, typename F>
__device__ __forceinline__ void ask_pieces(F f) {
    if constexpr (N > 0) {
        ask_pieces<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// A workgroup has one tile of TM x TN results after the other, a wave (TM / WAVES_M) x (TN / WAVES_N) of it in registers.  A step's codes and scales are staged by direct loads to LDS
// through buffers that end with the operand, two stages in turn.  The steps of all its tiles are one sequence: before a wave's last products of a step the next step has arrived and the
// waves meet, then it reads that step's first operands beside these products and asks for the step after, of the next tile where this one ends; so neither the meeting nor a tile's end stops
// the products for long.  SHARED: a wave's columns have one scale a step (weights in tiles).
//
// What bounds it is the issue of instructions, and power: a wave issues one in four cycles, and 32 products a step come with 128 multiply-adds of their results, 24 reads of LDS and 18 loads.  At
// 24576 x 4096 -> 6144 bf16 an instruction is issued in 69 to 74 % of the slots, the matrix cores are busy 53 % of the cycles and LDS 24 %, without conflicts, at 2.0 of 2.6 GHz.  Tiles of 256 x 256 take
// 1.6 us a step with two waves a SIMD (2.7 PFLOP/s on 256 compute units), 6 us a tile's end, 12 with GELU.  24576 x 4096 -> 6144 520 to 550 us one call after the other (2.3 PFLOP/s; a library
// product with one scale for everything 2.93), 540 to 630 with the card idle before it; 24576 x 1024 -> 4096 122, with GELU 156 to 165 (170 to 190); fp32 results, in tiles of 128, 1148 and 234.  Tiles of
// 128 x 128 for bf16: 708 and, with GELU, 197; products of 32 x 32 x 64 instead of 16 x 16 x 128: 2 to 5 % longer; one workgroup a tile, with scales loaded where they are used: 3261 (first form),
// staged 591, as one sequence of steps 531 to 566.
template <int DT, int TM, int TN, int WAVES_M, int WAVES_N, bool SHARED, bool DIRECT>
__global__ __launch_bounds__(WAVES_M* WAVES_N * 64, 512 / (WAVES_M * WAVES_N * 64)) void gemm_e4m3_kernel(ScaledGemmArgs s) {
    constexpr int THREADS = WAVES_M * WAVES_N * 64, BM = TM / WAVES_M / 16, BN = TN / WAVES_N / 16, SCALES = (TM + TN) / THREADS;
    constexpr bool WIDE = DT == CT_F32;
    using Op = Operand<CT_E4M3, TM, SCALED_BLOCK, THREADS, ROWS>;
    static_assert(TM == TN && (TM + TN) % THREADS == 0 && TM % 128 == 0, "both operands' tiles are alike, and 64 scales are of one of them");
    static_assert(BM % 2 == 0 && 2 * Op::PER_THREAD <= BN * (BM - 1), "everything is asked for before the last rows' products");
    struct Stage {
        char a[Op::BYTES], b[Op::BYTES];
        float scale[TM + TN];
    };
    __shared__ __attribute__((aligned(128))) Stage stages[2];
    const GemmArgs& a = s.g;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WAVES_M, wn = wave / WAVES_M, r = lane & 15, q = lane >> 4;
    const uint32_t lds = lds_address((const char*)&stages[0]);
    const int a0 = wm * (TM / WAVES_M), b0 = wn * (TN / WAVES_N);  // the wave's first row and column
    const int steps = max((int)scaled_blocks(a.k), 1), total = a.tiles_m * a.tiles_n * a.splits;  // without k one step of zeros
    auto first_step = [&](int split) { return (int)((uint32_t)(steps * split) / (uint32_t)a.splits); };  // at most 2^24 steps and 32 shares

    // What is asked for next: a step's codes and scales, through buffers that move along k and end with the operand.  (Every instruction of the loop counts: a wave has one in four
    // cycles, and 32 products a step.)  A wave brings 64 scales of one operand, or several times as many, one a lane; of a tile of rows they are one.
    Op opa, opb;  // where a thread's runs are; with their bases, what goes through registers
    i32x4 buffer_a = buffer_of(a.a, 0), buffer_b = buffer_of(a.b, 0), buffer_scale[SCALES];
    uint32_t scale_offset[SCALES];
    int64_t scale_by[SCALES];         // bytes from a step's scales to the next one's
    const float* lane_scale[SCALES];  // through registers a lane's scale; NULL for a row that is not there
    int ask_id = blockIdx.x, ask_steps = 0, left = 0;  // the tile, how many of its steps, and of k (0: nothing is left)
    opa.begin(a.a, a.lda, 0, a.m, 0);
    opb.begin(a.b, a.ldb, 0, a.n, 0);
#pragma unroll
    for (int i = 0; i < SCALES; ++i) {
        const bool of_a = i * THREADS + wave * 64 < TM;
        scale_offset[i] = (of_a ? s.shift_a : s.shift_b) ? 0u : (uint32_t)(lane * (of_a ? s.sa_row : s.sb_row) * 4);
        scale_by[i] = (of_a ? s.sa_block : s.sb_block) * 4;
        buffer_scale[i] = buffer_of(s.scale_a, 0);
    }
    uint32_t offset_a[Op::PER_THREAD], offset_b[Op::PER_THREAD];
#pragma unroll
    for (int i = 0; i < Op::PER_THREAD; ++i) {
        offset_a[i] = opa.offset + i * opa.apart;
        offset_b[i] = opb.offset + i * opb.apart;
    }
    auto begin = [&] {
        const TileAt t = tile_at(a, ask_id);
        const int s0 = first_step(t.split);
        const int64_t k0 = (int64_t)s0 * SCALED_BLOCK;
        ask_steps = first_step(t.split + 1) - s0;
        left = (int)(a.k - k0);
        opa.move(a.a, (int64_t)t.m * TM, a.m, k0);
        opb.move(a.b, (int64_t)t.n * TN, a.n, k0);
        const bool some = left > 0;  // without k nothing is
        buffer_a = buffer_of(opa.base, some ? (uint32_t)((opa.have - 1) * (int)a.lda + left + 3) & ~3u : 0u);
        buffer_b = buffer_of(opb.base, some ? (uint32_t)((opb.have - 1) * (int)a.ldb + left + 3) & ~3u : 0u);
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            const int at = i * THREADS + wave * 64;  // the first of the stage's scales that this wave brings
            const bool of_a = at < TM;
            const int shift = of_a ? s.shift_a : s.shift_b;
            const int64_t first = of_a ? (int64_t)t.m * TM + at : (int64_t)t.n * TN + at - TM, have = (of_a ? a.m : (int64_t)a.n) - first;
            const int64_t row = of_a ? s.sa_row : s.sb_row, block = of_a ? s.sa_block : s.sb_block;
            const float* from = (of_a ? s.scale_a : s.scale_b) + (have > 0 ? (first >> shift) * row : 0) + s0 * block;
            if constexpr (DIRECT) buffer_scale[i] = buffer_of(from, some && have > 0 ? (uint32_t)(shift ? 4 : (min(have, (int64_t)64) - 1) * row * 4 + 4) : 0u);
            else lane_scale[i] = lane < have ? from + (shift ? 0 : lane * row) : nullptr;
        }
    };
    auto moved = [](i32x4& buffer, int64_t by) {
        const uint64_t at = (((uint64_t)(uint32_t)buffer[1] << 32) | (uint32_t)buffer[0]) + by;
        buffer[0] = (int)(uint32_t)at;
        buffer[1] = (int)(uint32_t)(at >> 32);
    };
    auto ask_on = [&] {
        if (--ask_steps > 0) {
            moved(buffer_a, SCALED_BLOCK);
            moved(buffer_b, SCALED_BLOCK);
            buffer_a[2] -= SCALED_BLOCK;
            buffer_b[2] -= SCALED_BLOCK;
            left -= SCALED_BLOCK;
            if constexpr (!DIRECT) {
                opa.advance();
                opb.advance();
            }
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {
                if constexpr (DIRECT) moved(buffer_scale[i], scale_by[i]);
                else if (lane_scale[i]) lane_scale[i] += scale_by[i] / 4;
            }
        } else if (ask_id + (int)gridDim.x < total) {
            ask_id += gridDim.x;
            begin();
        } else {
            left = buffer_a[2] = buffer_b[2] = 0;
#pragma unroll
            for (int i = 0; i < SCALES; ++i) buffer_scale[i][2] = 0;
        }
    };
    // It is asked for in pieces between the products.
    constexpr int PIECES = 2 * Op::PER_THREAD;
    uint4 held_a[DIRECT ? 1 : Op::PER_THREAD], held_b[DIRECT ? 1 : Op::PER_THREAD];
    float held_scale[SCALES];
    uint32_t place = lds + wave * 1024;  // of this wave's first piece in the stage that is asked for
    auto ask_scales = [&] {
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            if constexpr (DIRECT) {
                const uint32_t to = place - wave * 768;
                if (i == 0) load_word_to_lds<2 * Op::BYTES>(buffer_scale[i], scale_offset[i], to);
                else load_word_to_lds<2 * Op::BYTES + THREADS * 4>(buffer_scale[i], scale_offset[i], to);
            } else {
                held_scale[i] = left > 0 && lane_scale[i] ? *lane_scale[i] : 0.f;
            }
        }
    };
    auto ask_piece = [&](auto piece) {
        constexpr int i = decltype(piece)::value;
        if constexpr (DIRECT) {
            if constexpr (i < Op::PER_THREAD) load_to_lds<Op::BYTES + i * THREADS * 16>(buffer_b, offset_b[i], place);
            else load_to_lds<(i - Op::PER_THREAD) * THREADS * 16>(buffer_a, offset_a[i - Op::PER_THREAD], place);
        } else if constexpr (i == 0) {
            opa.fetch(held_a, left);
            opb.fetch(held_b, left);
        }
    };
    // What was asked for is in its stage, and everyone has left the other one, which is asked for next.  What lies behind k in a row is not zero: it is cleared before anything is read.
    // Stores of a tile's results that were begun after what arrives here was asked for are not waited for: loads and stores end in the order in which they began.
    int behind = 0;
    auto arrive = [&](int into, auto after_stores) {
        Stage& to = stages[into];
        if constexpr (!DIRECT) {
            opa.put(to.a, held_a);
            opb.put(to.b, held_b);
#pragma unroll
            for (int i = 0; i < SCALES; ++i) to.scale[i * THREADS + threadIdx.x] = held_scale[i];
        }
        if (!DIRECT || !decltype(after_stores)::value || behind == 0) lds_loads_arrived();
        else if (behind == 2 * BM) lds_loads_left<2 * BM>();
        else lds_loads_left<4 * BM>();
        meet();
        if (DIRECT && left > 0 && left < SCALED_BLOCK) {
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {
                const int row = i * THREADS + threadIdx.x;
                clear_behind(row < TM ? to.a + row * SCALED_BLOCK : to.b + (row - TM) * SCALED_BLOCK, Op::exchanged(row & 15), left);
            }
            __syncthreads();
        }
        place = lds + wave * 1024 + (into ? 0 : (uint32_t)sizeof(Stage));
    };

    // A step's operands in registers: all columns of the wave, 16 rows and the next 16.  A lane's places in the stage that is read.
    Codes fb[BN], fa[2];
    float sa[2], sb[SHARED ? 1 : BN][4];
    const char* at_a = stages[0].a + (a0 + r) * SCALED_BLOCK + ((q ^ Op::exchanged(r)) << 4);
    const char* at_b = stages[0].b + (b0 + r) * SCALED_BLOCK + ((q ^ Op::exchanged(r)) << 4);
    const char* at_scale_a = (const char*)&stages[0].scale[a0 + r];
    const char* at_scale_b = (const char*)&stages[0].scale[TM + b0 + (SHARED ? 0 : 4 * q)];
    int other = (int)((4 ^ Op::exchanged(r) ^ q) - (q ^ Op::exchanged(r))) * 16;  // from a lane's first run of a row to its second, four on before the exchange
    auto read = [&](const char* at) {
        Codes c;
        c.run[0] = *reinterpret_cast<const uint4*>(at);
        c.run[1] = *reinterpret_cast<const uint4*>(at + other);
        return c;
    };
    auto read_rows = [&](int i) {
        fa[i & 1] = read(at_a + 16 * SCALED_BLOCK * i);
        sa[i & 1] = *reinterpret_cast<const float*>(at_scale_a + 64 * i);
    };
    auto read_columns = [&](int j) { fb[j] = read(at_b + 16 * SCALED_BLOCK * j); };
    auto read_scales = [&] {
        if constexpr (SHARED) {
            sb[0][0] = *reinterpret_cast<const float*>(at_scale_b);
        } else {
#pragma unroll
            for (int j = 0; j < BN; ++j) {
                const f32x4 four = *reinterpret_cast<const f32x4*>(at_scale_b + 64 * j);
#pragma unroll
                for (int v = 0; v < 4; ++v) sb[j][v] = four[v];
            }
        }
    };
    auto turn = [&](int stage) {
        const int by = stage ? (int)sizeof(Stage) : -(int)sizeof(Stage);
        at_a += by;
        at_b += by;
        at_scale_a += by;
        at_scale_b += by;
    };

    int stage = 0;
    begin();
    ask_scales();
    ask_pieces<PIECES>(ask_piece);
    arrive(0, std::false_type());
    ask_on();
    ask_scales();
    if constexpr (DIRECT) ask_pieces<PIECES>(ask_piece);
    else ask_piece(std::integral_constant<int, 0>());

    for (int id = blockIdx.x; id < total; id += gridDim.x) {
        const TileAt tile = tile_at(a, id);
        f32x4 acc[BM][BN];
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[i][j] = (f32x4)(0.f);
        read_rows(0);
#pragma unroll
        for (int j = 0; j < BN; ++j) read_columns(j);
        read_scales();
        // 16 rows of a after the other against all of the wave's columns.  A product is scaled and added while the third after it is formed.
        constexpr int LAG = 3;
        auto one_step = [&](auto first) {
            f32x4 t[LAG + 1];
            float factor[2];
            auto add = [&](int p) {
                const int i = p / BN, j = p % BN;
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(t[p % (LAG + 1)][v], SHARED ? factor[i & 1] : factor[i & 1] * sb[j][v], acc[i][j][v]);
                asm volatile("" : "+v"(acc[i][j]));  // here, and not where the sums are next used, which is behind a branch
            };
            ask_pieces<BM * BN>([&](auto product) {
                constexpr int at = decltype(product)::value, i = at / BN, j = at % BN;
                if constexpr (i == BM - 1 && j == 0) {
                    arrive(stage ^ 1, first);
                    ask_on();
                    ask_scales();
                    if constexpr (!DIRECT) ask_piece(std::integral_constant<int, 0>());
                    turn(stage ^ 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
                t[at % (LAG + 1)] = block_product<WIDE>(fb[j], fa[i & 1]);
                if constexpr (j == 0) read_rows(i + 1 < BM ? i + 1 : 0);
                if constexpr (i == BM - 1) read_columns(j);
                if constexpr (DIRECT && !decltype(first)::value && at < PIECES) ask_piece(product);
                if constexpr (at >= LAG) add(at - LAG);
                if constexpr (j == LAG - 1) factor[i & 1] = SHARED ? sa[i & 1] * sb[0][0] : sa[i & 1];
                if constexpr (!WIDE) __builtin_amdgcn_sched_barrier(0);
            });
#pragma unroll
            for (int p = BM * BN - LAG; p < BM * BN; ++p) add(p);
            read_scales();
            stage ^= 1;
        };
        // What follows a tile's first step is asked for before the results of the tile before are stored.
        one_step(std::true_type());
        for (int step = first_step(tile.split + 1) - first_step(tile.split); --step > 0;) one_step(std::false_type());
        if constexpr (DIRECT) ask_pieces<PIECES>(ask_piece);

        // Of 16 rows and 64 columns a lane has four columns each in four places of one row.  Exchanged with the lane 16 away they are eight each in two places, 32 columns apart, and with the lane
        // 8 away eight columns each of two rows, 8 apart: eight lanes have a row's 64 columns, whole lines of 16-bit results.
        static_assert(BN == 4, "64 columns a wave");
        const bool whole = a.splits == 1;
        int of = lane;
        asm volatile("" : "+v"(of));  // what follows from it is formed here, not before the loop and kept
        const int64_t m0 = (int64_t)tile.m * TM + a0 + (of & 7);
        const int n = tile.n * TN + b0 + 32 * ((of >> 3) & 1) + 16 * ((of >> 4) & 1) + 8 * (of >> 5);  // the first of the eight columns
        // A run of the residual is unpacked, and so waited for, where it is loaded, since each is under a branch of its own: with bias and residual 24576 x 1024 -> 4096 bf16 takes 200 us instead of 122
        // (39 of the difference are the residual's bytes), 24576 x 4096 -> 1024 142 instead of 124 with the bias.
        Eight<DT> bias = {}, residual[2][2] = {};
        auto fetch_residual = [&](int i) {
            if (!a.residual || !whole || a.n - n < 8) return;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t m = m0 + 16 * i + 8 * h;
                if (m < a.m) residual[i & 1][h].load(a.residual, m * a.ldr + n, 8);
            }
        };
        if (a.bias && whole && a.n - n >= 8) bias.load(a.bias, n, 8);
        fetch_residual(0);
#pragma unroll
        for (int i = 0; i < BM; ++i) {
            if (i + 1 < BM) fetch_residual(i + 1);
            float v[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][2 * h][e]), __float_as_uint(acc[i][2 * h + 1][e]), false, false);
                    v[h][e] = __uint_as_float(both[0]);
                    v[h][4 + e] = __uint_as_float(both[1]);
                }
#pragma unroll
            for (int e = 0; e < 8; ++e) {  // lanes 8 to 15 of 16 give the first rows' half for the last rows' of lanes 0 to 7
                const uint32_t x = __float_as_uint(v[0][e]), y = __float_as_uint(v[1][e]);
                v[0][e] = __uint_as_float(__builtin_amdgcn_update_dpp(x, y, 0x128, 0xF, 0xC, false));  // row_ror:8
                v[1][e] = __uint_as_float(__builtin_amdgcn_update_dpp(y, x, 0x128, 0xF, 0x3, false));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t m = m0 + 16 * i + 8 * h;
                if (m >= a.m || n >= a.n) continue;
                if (whole) {
                    if (n + 8 <= a.n) finish_run<DT>(a, m, n, 8, v[h], bias, residual[i & 1][h]);
                    else finish_few<DT>(a, m, n, a.n - n, v[h]);
                } else {
                    // shares lie in whole tiles, so they need no edge
                    float* to = a.partial + (((int64_t)tile.split * a.tiles_m * TM + m) * a.tiles_n * TN + n);
                    reinterpret_cast<f32x4*>(to)[0] = f32x4{v[h][0], v[h][1], v[h][2], v[h][3]};
                    reinterpret_cast<f32x4*>(to)[1] = f32x4{v[h][4], v[h][5], v[h][6], v[h][7]};
                }
            }
        }
        // at least one store of 16 bytes for each run of eight results, two of shares and where `pre` is kept
        behind = (int64_t)(tile.m + 1) * TM > a.m || a.n - tile.n * TN < TN ? 0 : whole && !a.pre ? 2 * BM : 4 * BM;
    }
    lds_loads_arrived();  // what was asked for last ends before its place is given away
}

// Small products: tiles of 64 x 64, a wave 32 x 32 of one, and a ring of stages, since the time is the latency of the loads and not what they bring: STAGES - 1 steps are under way while one is
// multiplied.  Every wave has five loads a step (waves 2 and 3 bring the scales that 0 and 1 do), behind the last step of zeros, so that it can wait by their number.  1531 x 777 -> 1001 with fp32
// results and residual, 384 tiles: 14.0-14.5 us with the card idle before it; with fp16 results and no residual 9.6-10.5.
constexpr int SMALL = 64;
struct SmallStage {
    char a[SMALL * SCALED_BLOCK], b[SMALL * SCALED_BLOCK];
    float scale[2 * SMALL];
};
template <int DT, bool SHARED, int STAGES>
__device__ __forceinline__ void gemm_small_e4m3(const ScaledGemmArgs& s, int id, SmallStage* stages) {
    constexpr bool WIDE = DT == CT_F32;
    constexpr int BM = 2, BN = 2;
    using Op = Operand<CT_E4M3, SMALL, SCALED_BLOCK, 256, ROWS>;
    typedef SmallStage Stage;
    static_assert(Op::PER_THREAD == 2 && Op::BYTES == sizeof(Stage::a), "five loads a step");
    const GemmArgs& a = s.g;
    const TileAt tile = tile_at(a, id);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4, a0 = (wave & 1) * 32, b0 = (wave >> 1) * 32;
    const int steps = (int)scaled_blocks(a.k);
    const int s0 = (int)((uint32_t)(steps * tile.split) / (uint32_t)a.splits), s1 = (int)((uint32_t)(steps * (tile.split + 1)) / (uint32_t)a.splits);
    const int64_t m0 = (int64_t)tile.m * SMALL, k0 = (int64_t)s0 * SCALED_BLOCK;
    const int n0 = tile.n * SMALL;
    Op opa, opb;
    opa.begin(a.a, a.lda, m0, a.m, k0);
    opb.begin(a.b, a.ldb, n0, a.n, k0);
    const bool of_a = (wave & 1) == 0;
    const int shift = of_a ? s.shift_a : s.shift_b;
    const int64_t first = of_a ? m0 : n0, last = (of_a ? a.m : (int64_t)a.n) - 1, row = of_a ? s.sa_row : s.sb_row, block = of_a ? s.sa_block : s.sb_block;
    const float* scale = (of_a ? s.scale_a : s.scale_b) + (first >> shift) * row + s0 * block;
    const uint32_t scale_offset = shift ? 0u : (uint32_t)(lane * row * 4), scale_bytes = (uint32_t)(shift ? 4 : (min(last - first, (int64_t)63) * row + 1) * 4);
    int left = (int)(a.k - k0), asked = s0;
    const uint32_t lds = lds_address((const char*)&stages[0]);
    auto ask = [&](int stage) {
        const bool some = asked < s1;
        const uint32_t place = lds + stage * (uint32_t)sizeof(Stage);
        const i32x4 from_a = buffer_of(opa.base, some ? (uint32_t)((opa.have - 1) * (int)a.lda + left + 3) & ~3u : 0u);
        const i32x4 from_b = buffer_of(opb.base, some ? (uint32_t)((opb.have - 1) * (int)a.ldb + left + 3) & ~3u : 0u);
        load_to_lds<0>(from_a, opa.offset, place + wave * 1024);
        load_to_lds<4096>(from_a, opa.offset + opa.apart, place + wave * 1024);
        load_to_lds<Op::BYTES>(from_b, opb.offset, place + wave * 1024);
        load_to_lds<Op::BYTES + 4096>(from_b, opb.offset + opb.apart, place + wave * 1024);
        load_word_to_lds<2 * Op::BYTES>(buffer_of(scale, some ? scale_bytes : 0u), scale_offset, place + (wave & 1) * 256);
        opa.advance();
        opb.advance();
        scale += block;
        left -= SCALED_BLOCK;
        ++asked;
    };
    f32x4 acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = (f32x4)(0.f);
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) ask(i);
    const bool whole = a.splits == 1;
    const int n = n0 + b0 + 16 * (q & 1) + 8 * (q >> 1);  // the first of the eight columns that this lane finishes
    int stage = 0;
    for (int step = s0; step < s1; ++step, stage = stage + 1 == STAGES ? 0 : stage + 1) {
        lds_loads_left<5 * (STAGES - 2)>();
        meet();
        Stage& here = stages[stage];
        const int k_left = a.k - step * SCALED_BLOCK;
        if (k_left < SCALED_BLOCK) {  // what lies behind k in a row is not zero
            if (threadIdx.x < 2 * SMALL) clear_behind(here.a + threadIdx.x * SCALED_BLOCK, Op::exchanged(threadIdx.x & 15), k_left);
            __syncthreads();
        }
        ask(stage == 0 ? STAGES - 1 : stage - 1);
        Codes fa[BM], fb[BN];
        float sa[BM], sb[BN][4];
        auto read = [&](const char* from) {
            Codes c;
#pragma unroll
            for (int h = 0; h < 2; ++h) c.run[h] = *reinterpret_cast<const uint4*>(from + r * SCALED_BLOCK + (((4 * h + q) ^ Op::exchanged(r)) << 4));
            return c;
        };
#pragma unroll
        for (int i = 0; i < BM; ++i) fa[i] = read(here.a + (a0 + 16 * i) * SCALED_BLOCK), sa[i] = here.scale[a0 + 16 * i + r];
#pragma unroll
        for (int j = 0; j < BN; ++j) {
            fb[j] = read(here.b + (b0 + 16 * j) * SCALED_BLOCK);
            const f32x4 four = *reinterpret_cast<const f32x4*>(&here.scale[SMALL + b0 + 16 * j + 4 * q]);
#pragma unroll
            for (int v = 0; v < 4; ++v) sb[j][v] = SHARED ? four[0] : four[v];
        }
        f32x4 t[BM][BN];
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) t[i][j] = block_product<WIDE>(fb[j], fa[i]);
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(t[i][j][v], sa[i] * sb[j][v], acc[i][j][v]);
    }
    lds_loads_arrived();  // what was asked for last ends before its place is given away
#pragma unroll
    for (int i = 0; i < BM; ++i) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][0][e]), __float_as_uint(acc[i][1][e]), false, false);
            v[e] = __uint_as_float(both[0]);
            v[4 + e] = __uint_as_float(both[1]);
        }
        const int64_t m = m0 + a0 + 16 * i + r;
        if (m >= a.m || n >= a.n) continue;
        if (!whole) {
            float* to = a.partial + (((int64_t)tile.split * a.tiles_m * SMALL + m) * a.tiles_n * SMALL + n);
            reinterpret_cast<f32x4*>(to)[0] = f32x4{v[0], v[1], v[2], v[3]};
            reinterpret_cast<f32x4*>(to)[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else if (n + 8 <= a.n) {
            finish_run<DT>(a, m, n, 8, v);
        } else {
            finish_few<DT>(a, m, n, a.n - n, v);
        }
    }
}

template <int DT, bool SHARED, int STAGES>
__global__ __launch_bounds__(256) void gemm_small_e4m3_kernel(ScaledGemmArgs s) {
    __shared__ __attribute__((aligned(128))) SmallStage stages[STAGES];
    gemm_small_e4m3<DT, SHARED, STAGES>(s, blockIdx.x, stages);
}

// The sums of the columns of partial ([groups][columns]), beside other work of their launch.
struct ColumnSums {
    const float* partial;
    void* to;
    int64_t groups, columns;
    unsigned workgroups() const { return to ? (unsigned)((columns + 31) / 32) : 0u; }
};
// 32 columns, in the order of column_sums_kernel: 32 strands of groups, then the strands one after the other; a thread has four strands.
template <int DT>
__device__ __forceinline__ void sum_columns(const ColumnSums& p, int id, float (*parts)[33]) {
    const int lane = threadIdx.x & 31, first = threadIdx.x >> 5;
    const int64_t column = (int64_t)id * 32 + lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float sum = 0.f;
        if (column < p.columns)
#pragma unroll 4
            for (int64_t g = first + 8 * i; g < p.groups; g += 32) sum += p.partial[g * p.columns + column];
        parts[first + 8 * i][lane] = sum;
    }
    __syncthreads();
    if (first == 0 && column < p.columns) {
        float sum = parts[0][lane];
        for (int i = 1; i < 32; ++i) sum += parts[i][lane];
        ((typename Elem<DT>::T*)p.to)[column] = (typename Elem<DT>::T)sum;
    }
}
// The two products of a small gradient and the sums of its columns in one launch, since each by itself leaves compute units idle: the tiles of the first, those of the second, then 32 columns a
// workgroup.  (1531 x 777 -> 1001 fp16: 14.7 us for 10.5, 9.1 and 3.7 in launches of their own.)
struct SmallGradient {
    ScaledGemmArgs of[2];
    int32_t first, tiles;  // of the first product and of both
    ColumnSums sums;
};
template <int DT>
__global__ __launch_bounds__(256) void gradient_small_e4m3_kernel(SmallGradient p) {
    constexpr int STAGES = 3;  // so that a compute unit has room for three workgroups: four stages and two of them take 18.2 us at the size above
    __shared__ __attribute__((aligned(128))) SmallStage stages[STAGES];
    const int id = blockIdx.x;
    if (id >= p.tiles) return sum_columns<DT>(p.sums, id - p.tiles, (float(*)[33])stages);
    const int which = id >= p.first;
    gemm_small_e4m3<DT, false, STAGES>(p.of[which], id - (which ? p.first : 0), stages);
}

// The tile and the shares of k of a product, from its sizes alone: those that take the least time by a count of what they do.  A card holds 256 workgroups with a tile of 256 x 256, 512 with
// smaller ones, and a step takes less where there are 256 of them at most.  Microseconds, fitted to 14000 timings of 1500 products of 17 to 24576 rows: what is chosen takes 1.4 % longer than the
// best of all tiles and shares on average, 45 % at most.  (By numbers of tiles alone, as for gemm_kernel: 36 % on average.)
struct Plan {
    int tile, splits;
};
constexpr int64_t round_to(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
struct TileCosts {
    int tile;
    double each, step_alone, step;  // a tile, a step with at most 256 workgroups and with more
};
Plan plan_of(int64_t m, int64_t n, int64_t k, int dtype) {
    constexpr TileCosts halves[3] = {{SMALL, 2.0, 0.35, 0.66}, {128, 2.9, 0.94, 1.1}, {256, 5.8, 1.66, 1.66}}, floats[2] = {{SMALL, 2.1, 0.45, 0.74}, {128, 2.7, 1.3, 1.4}};
    constexpr int shares_of[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    const int64_t steps = std::max(scaled_blocks(k), (int64_t)1);
    Plan best = {SMALL, 1};
    double least = HUGE_VAL;
    for (int t = 0; t < (dtype == FNN_F32 ? 2 : 3); ++t) {
        const TileCosts& c = dtype == FNN_F32 ? floats[t] : halves[t];
        const int64_t tiles = round_to(m, c.tile) / c.tile * (round_to(n, c.tile) / c.tile), slots = c.tile == 256 ? 256 : 512;
        for (const int splits : shares_of) {
            if (splits > 1 && (steps / splits < 2 || tiles * splits > 1100)) break;
            const int64_t shares = tiles * splits, rest = shares % slots;
            const double per = (double)steps / splits, few = c.each + per * c.step_alone, many = c.each + per * c.step;
            double time;
            if (c.tile == SMALL) time = std::max(1.0, shares / 512.0) * (shares <= 256 ? few : many);  // not one after the other in a workgroup
            else time = (double)(shares / slots) * many + (rest == 0 ? 0.0 : rest <= 256 ? few : many);
            if (splits > 1) time += 2.5 + 0.26 * splits + (double)splits * m * n * 4 / 3.9e6;
            if (time < least) {
                least = time;
                best = {c.tile, splits};
            }
        }
    }
    return best;
}

// Whether an operand's rows start on 16-byte boundaries.
bool on_runs(const void* data, int64_t stride, int64_t rows) { return ((uintptr_t)data & 15) == 0 && (rows < 2 || stride % 16 == 0); }
// Whether they do, and the offsets of a tile's codes and of 64 rows' scales fit 32 bits.
bool direct(const void* data, int64_t stride, int64_t rows, int64_t scale_row) {
    return on_runs(data, stride, rows) && stride < ((int64_t)1 << 31) / 256 && scale_row < ((int64_t)1 << 31) / 256;
}

// gemm_join_kernel with the columns' sums in its first workgroups.  1024 x 4096 in four shares and 4096 columns of 96 groups: 15.5 us for 12.8 and 4.9 in launches of their own; with
// the sums in the last workgroups 17.7.
template <int DT>
__global__ __launch_bounds__(256) void join_and_sum_kernel(GemmArgs a, int64_t pitch, int64_t share, unsigned first, ColumnSums sums) {
    __shared__ float parts[32][33];
    if (blockIdx.x >= first) gemm_join<DT>(a, pitch, share, blockIdx.x - first);
    else sum_columns<DT>(sums, blockIdx.x, parts);
}

// (The numbers that go with the launches name what ran to a trace: a tile's side, 129 for what goes through registers, 65 for a small gradient, 16 or 32 for few rows.)
template <int DT, bool SHARED>
hipError_t run_tiles(ScaledGemmArgs a, bool is_direct, Plan p, const ColumnSums& sums, int kind, hipStream_t s) {
    GemmArgs& g = a.g;
    if (!is_direct) p.tile = 128;  // what goes through registers; the workspace has room for its shares, too
    g.tiles_m = (int)(round_to(g.m, p.tile) / p.tile);
    g.tiles_n = (int)(round_to(g.n, p.tile) / p.tile);
    g.splits = p.splits;
    const int64_t count = (int64_t)g.tiles_m * g.tiles_n * g.splits;
    if (count > INT32_MAX) return hipErrorInvalidValue;
    hipError_t e;
    // of the larger tiles as many workgroups as the card's 256 compute units hold
    const dim3 few((unsigned)std::min(count, (int64_t)256)), more((unsigned)std::min(count, (int64_t)512));
    if (p.tile == SMALL) {
        e = launch_detail(kind, SMALL, gemm_small_e4m3_kernel<DT, SHARED, 4>, dim3((unsigned)count), dim3(256), 0, s, a);
    } else if (DT != CT_F32 && p.tile == 256) {
        if constexpr (DT != CT_F32) e = launch_detail(kind, 256, gemm_e4m3_kernel<DT, 256, 256, 2, 4, SHARED, true>, few, dim3(512), 0, s, a);
    } else {
        e = is_direct ? launch_detail(kind, 128, gemm_e4m3_kernel<DT, 128, 128, 2, 2, SHARED, true>, more, dim3(256), 0, s, a)
                      : launch_detail(kind, 129, gemm_e4m3_kernel<DT, 128, 128, 2, 2, SHARED, false>, more, dim3(256), 0, s, a);
    }
    if (e != hipSuccess || g.splits == 1) return e;
    const int64_t pitch = (int64_t)g.tiles_n * p.tile, share = pitch * g.tiles_m * p.tile, runs = (int64_t)((g.n + 7) / 8) * g.m;
    const unsigned joins = (unsigned)((runs + 255) / 256);
    if (sums.to) return launch(kind, join_and_sum_kernel<DT>, dim3(joins + sums.workgroups()), dim3(256), 0, s, g, pitch, share, sums.workgroups(), sums);
    return launch(kind, gemm_join_kernel<DT>, dim3(joins), dim3(256), 0, s, g, pitch, share);
}

// Rows on 16-byte boundaries, zeros behind their ends, of one operand or of both: a thread writes 16 bytes, read from wherever they are.
struct CopyCodes {
    const uint8_t* from[2];
    uint8_t* to[2];
    int64_t from_stride[2], rows[2];
    int64_t stride;
    int32_t width;
};
__global__ __launch_bounds__(256) void copy_codes_kernel(CopyCodes a, uint32_t first_group) {
    const int64_t runs = a.stride / 16, at = (int64_t)(first_group + blockIdx.x) * 256 + threadIdx.x, row = at / runs;
    const int e = (int)(at - row * runs) * 16, which = row >= a.rows[0];
    const int64_t of = which ? row - a.rows[0] : row;
    if (of >= a.rows[which]) return;
    *reinterpret_cast<uint4*>(a.to[which] + of * a.stride + e) = load_run<CT_E4M3>(a.from[which] + of * a.from_stride[which] + e, a.width - e);
}

// Copies of operands whose rows do not start on 16-byte boundaries, in the room that the workspace has for them where k is no multiple of 16.  (Microseconds through registers and
// copied, bf16: 24576 x 1023 -> 4096 321 and 148, 1531 x 777 -> 1001 23.8 and 14.9, 64 x 1001 -> 4096 21.7 and 12.8.)
hipError_t copy_operands(GemmArgs& g, char* room, int kind, hipStream_t s) {
    CopyCodes c = {};
    c.stride = round_to(g.k, 16);
    c.width = g.k;
    const bool copy[2] = {!on_runs(g.a, g.lda, g.m), !on_runs(g.b, g.ldb, g.n)};
    int64_t rows = 0;
    for (int i = 0; i < 2; ++i) {
        const int64_t n = i ? (int64_t)g.n : g.m;
        c.from[i] = (const uint8_t*)(i ? g.b : g.a);
        c.from_stride[i] = i ? g.ldb : g.lda;
        c.to[i] = (uint8_t*)room + (i ? round_to(g.m * c.stride, 256) : 0);
        if (!copy[i]) continue;
        c.rows[i] = n;
        rows += n;
        (i ? g.b : g.a) = c.to[i];
        (i ? g.ldb : g.lda) = c.stride;
    }
    if (rows == 0) return hipSuccess;
    const int64_t groups = (rows * (c.stride / 16) + 255) / 256;
    if (groups > INT32_MAX) return hipErrorInvalidValue;  // 8 TB
    return in_launches(groups, 256, [&](uint32_t first, dim3 grid) { return launch(kind, copy_codes_kernel, grid, dim3(256), 0, s, c, first); });
}

template <int DT>
hipError_t run_few_rows(const ScaledGemmArgs& a, int kind, hipStream_t s) {
    constexpr int THREADS = FEW_WAVES * 64;
    return in_launches(((int64_t)a.g.n + 15) / 16, THREADS, [&](uint32_t first, dim3 grid) {
        return a.g.m <= 16 ? launch_detail(kind, 16, few_rows_e4m3_kernel<DT, 1>, grid, dim3(THREADS), 0, s, a, first)
                           : launch_detail(kind, 32, few_rows_e4m3_kernel<DT, 2>, grid, dim3(THREADS), 0, s, a, first);
    });
}

template <typename F>
hipError_t with_type(int dtype, F f) {
    if (dtype == FNN_F32) return f(std::integral_constant<int, CT_F32>());
    if (dtype == FNN_F16) return f(std::integral_constant<int, CT_F16>());
    return f(std::integral_constant<int, CT_BF16>());
}

}  // namespace

size_t scaled_gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, bool copies) {
    if (m < 1 || n < 1 || few_rows(m, k)) return 0;
    const Plan p = plan_of(m, n, k, dtype);
    const int64_t tile = std::max(p.tile, 128), stride = round_to(k, 16);
    const size_t partial = p.splits > 1 ? (size_t)p.splits * round_to(m, tile) * round_to(n, tile) * sizeof(float) : 0;
    return copies && k % 16 ? (size_t)round_to(partial, 256) + (size_t)round_to(m * stride, 256) + (size_t)round_to(n * stride, 256) : partial;
}

namespace {

// sums: taken along where the product's shares are joined, and otherwise before it.
hipError_t run_product(ScaledGemmArgs a, int dtype, bool copies, const ColumnSums& sums, int kind, hipStream_t s) {
    GemmArgs& g = a.g;
    const bool some = g.m > 0 && g.n > 0, few = some && few_rows(g.m, g.k);
    const Plan p = some && !few ? plan_of(g.m, g.n, g.k, dtype) : Plan{SMALL, 1};
    if (sums.to && p.splits == 1) {
        const hipError_t e = launch_column_sums(sums.partial, sums.groups, sums.columns, sums.columns, sums.to, nullptr, dtype, kind, s);
        if (e != hipSuccess) return e;
    }
    if (!some) return hipSuccess;
    return with_type(dtype, [&](auto dt) {
        constexpr int DT = dt.value;
        if (few) return run_few_rows<DT>(a, kind, s);
        if (copies && g.k % 16) {
            const hipError_t e = copy_operands(g, (char*)g.partial + round_to((int64_t)scaled_gemm_workspace(g.m, g.n, g.k, dtype, false), 256), kind, s);
            if (e != hipSuccess) return e;
        }
        const bool d = direct(g.a, g.lda, g.m, a.sa_row) && direct(g.b, g.ldb, g.n, a.sb_row);
        return a.shift_b ? run_tiles<DT, true>(a, d, p, sums, kind, s) : run_tiles<DT, false>(a, d, p, sums, kind, s);
    });
}

}  // namespace

hipError_t launch_scaled_gemm(const ScaledGemmArgs& a, int dtype, int kind, hipStream_t s) { return run_product(a, dtype, true, ColumnSums{}, kind, s); }

hipError_t launch_scaled_gradient(const ScaledGemmArgs& dx, const ScaledGemmArgs& dw, const float* partial, int64_t groups, int64_t columns, void* sums, int dtype, int kind, hipStream_t s) {
    const ScaledGemmArgs* of[2] = {&dx, &dw};
    const ColumnSums columns_sums = {partial, sums, groups, columns};
    int64_t tiles[2];
    bool small = true;
    for (int i = 0; i < 2 && small; ++i) {
        const GemmArgs& g = of[i]->g;
        small = g.m > 0 && g.n > 0 && g.k > 0 && !few_rows(g.m, g.k);
        if (!small) break;
        const Plan p = plan_of(g.m, g.n, g.k, dtype);
        small = p.tile == SMALL && p.splits == 1 && direct(g.a, g.lda, g.m, of[i]->sa_row) && direct(g.b, g.ldb, g.n, of[i]->sb_row);
        tiles[i] = round_to(g.m, SMALL) / SMALL * (round_to(g.n, SMALL) / SMALL);
    }
    if (small) {
        SmallGradient p;
        for (int i = 0; i < 2; ++i) {
            p.of[i] = *of[i];
            GemmArgs& g = p.of[i].g;
            g.tiles_m = (int)(round_to(g.m, SMALL) / SMALL);
            g.tiles_n = (int)(round_to(g.n, SMALL) / SMALL);
            g.splits = 1;
        }
        p.first = (int32_t)tiles[0];
        p.tiles = (int32_t)(tiles[0] + tiles[1]);
        p.sums = columns_sums;
        const dim3 grid((unsigned)p.tiles + columns_sums.workgroups());
        return with_type(dtype, [&](auto dt) { return launch_detail(kind, SMALL + 1, gradient_small_e4m3_kernel<dt.value>, grid, dim3(256), 0, s, p); });
    }
    const hipError_t e = run_product(dx, dtype, false, ColumnSums{}, kind, s);
    return e == hipSuccess ? run_product(dw, dtype, false, columns_sums, kind, s) : e;
}

}  // namespace fnn
