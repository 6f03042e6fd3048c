// The gradient of attention (fnn_attention_backward), without a score matrix in memory: with p = exp(scale q k^T - lse) formed again and
// delta = sum_e dout out,  ds = p (dout v^T - delta),  dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout.
//
// Two passes, so that every sum is one workgroup's own and its order fixed: rows by rows for dq (which also leaves delta behind), then
// keys by keys for dk and dv.  Seven products where five would do if the first pass could add into dk and dv; atomics would, in an order of their own.
// As in the forward pass the lane owns a row (a key) of the scores and the next product's operand is what the last one left in its registers; the
// tiles that are read along and across their rows lie in LDS once, for both.
#include <algorithm>
#include <type_traits>

#include "attention_device.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// fp16 weights are formed 2^14 times too large (at most 2^14) for dv: those of long rows, 1 / 16384 and less, would lose bits below the
// type's normal range.  The factor leaves with the result.
template <int DT>
constexpr int WEIGHT_SHIFT = DT == CT_F16 ? 14 : 0;

// ds is of any size: p, down to 0, times what dout and v are.  In fp16 it is rounded as ds times a power of two (`by`) of its row (dq) or key (dk), chosen such that the largest so
// far is between 1 and 2^15: nothing overflows, and half of the type's last step is 2^-25 of that largest or less.  As with the maximum of a softmax, what
// has been summed is rescaled in the rare case that the largest leaves that range; it starts again at 2^8.  bf16 has fp32's range and needs none of it.
// The largest costs 5 % of the two passes and the branch, which the products wait for, 6 % (6 x 2048 causal rows, 12 heads of 64: 242 and 268 us without and with it; 4 x 2048,
// 16 heads on 8 of 128: 532 and 587).  Looked at once for 64 keys with both blocks' ds held back, it is slower: the registers are not there.
template <int DT>
struct Digits {
    static constexpr bool USED = DT == CT_F16;
    static constexpr int LEAST = -40, MOST = 64;  // of by's exponent: |ds| <= 2^40 in fp16; smaller ones than 2^-64 are far below what a result shows
    float by = 1.f, largest = 0.f;

    // `ds`: 16 of the lane's row (key), the other half's lane has 16 more.  DB blocks of results so far.
    template <int DB>
    __device__ __forceinline__ void fit(f32x16& ds, f32x16 (&sums)[DB]) {
        if constexpr (!USED) return;
        float most = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) most = __builtin_fmaxf(most, __builtin_fabsf(ds[x]));
        largest = __builtin_fmaxf(largest, across_halves_max(most));
        const bool out = largest > 32768.f || (largest < 1.f && largest > 0.f);
        if (__builtin_expect(__ballot(out) != 0, 0)) {
            const int now = exponent(by), wanted = now + 8 - exponent(largest);
            const int step = out ? min(max(wanted, LEAST), MOST) - now : 0;
            const float factor = __uint_as_float((uint32_t)(127 + step) << 23);
            by *= factor;
            largest *= factor;
#pragma unroll
            for (int x = 0; x < 16; ++x) ds[x] *= factor;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x) sums[i][x] *= factor;
        }
    }
    static __device__ __forceinline__ int exponent(float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; }
};

// dq, and what the second pass takes of each row: a wave has 32 rows and runs over tiles of 64 keys, which its workgroup's four waves share.  Three products a tile.
// 12 sequences of up to 2048 rows, 12 heads of 64, bf16: 116 us, bound by the latency from product to exponential to product, of which a SIMD's two
// waves hide part: the matrix cores are busy 34 % of the cycles, the vector units 42 %.
template <int DT, int DB, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(AttentionBackArgs a) {
    constexpr int KEYS = 64, ROWS = 128;
    using Tile = HeadTile<DT, DB, KEYS>;
    typedef typename Elem<DT>::T E;
    __shared__ __attribute__((aligned(16))) char stages[2][2 * Tile::BYTES];
    __shared__ int any_not_finite;
    const AttentionArgs& f = a.forward;
    int group, tile;
    deal(f.row_tiles, f.causal, group, tile);
    const Sequence s = find_sequence<ROWS>(f, tile);
    if (s.index < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = s.lq * f.share, first = s.tile * ROWS, mine = first + wave * 32, r = mine + (lane & 31);
    const int tiles = (seen_by(f, s, min(first + ROWS, rows) - 1) + KEYS - 1) / KEYS;

    uint4 q[2 * DB], dout[2 * DB];
    float delta = 0.f, lse = -__builtin_inff();
    {
        uint4 out[2 * DB];
        load_row<DT, DB>(f.q, f.q_row, f.q_head, f, s, group, r, rows, lane, q);
        load_row<DT, DB>(a.dout, a.dout_row, a.dout_head, f, s, group, r, rows, lane, dout);
        load_row<DT, DB>(f.out, f.out_row, f.out_head, f, s, group, r, rows, lane, out);
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            E x[8], y[8];
            __builtin_memcpy(x, &dout[i], 16);
            __builtin_memcpy(y, &out[i], 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)x[e], (float)y[e], delta);
        }
        delta = across_halves_sum(delta);
        if (r < rows) lse = f.lse[flat_row(f, s, group, r)];
    }
    // a row that sees no key: plus infinity makes its weights 0; one that sees keys of no weight alone has minus infinity there, and no weights
    const int seen = seen_by(f, s, min(r, rows - 1));
    float base = r < rows && seen > 0 ? lse * LOG2E : __builtin_inff();
    const float c = f.scale * LOG2E;
    // lse and what it is compared with are off by up to five roundings: where those are whole units of the exponent, too much is taken off rather than too
    // little, so that no weight passes 1 by far, let alone overflows (below, by 2^1.25 at most)
    if (__builtin_fabsf(base) > 4194304.f && __builtin_fabsf(base) < __builtin_inff()) base += __builtin_fabsf(base) * 0x1p-21f;
    if (r < rows && lane < 32) {
        const int64_t at = flat_row(f, s, group, r);
        a.stats[at] = base - (float)WEIGHT_SHIFT<DT>;
        a.stats[at + (int64_t)f.tq * f.heads] = -delta;
    }
    if (!a.dq) return;
    const int least_seen = mine < rows ? seen_by(f, s, mine) : 0, most_seen = mine < rows ? seen_by(f, s, min(mine + 32, rows) - 1) : 0;
    f32x16 dq[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dq[i] = (f32x16)(0.f);
    Digits<DT> digits;

    const E* k = (const E*)f.k + s.k0 * f.k_row + group * f.k_head;
    const E* v = (const E*)f.v + s.k0 * f.v_row + group * f.v_head;
    auto stage = [&](char* to, int t) {
        const int key = t * KEYS, there = min(KEYS, s.lk - key);
        Tile::template stage<256, DIRECT>(to, k + key * f.k_row, f.k_row, there, f.d, threadIdx.x);
        Tile::template stage<256, DIRECT>(to + Tile::BYTES, v + key * f.v_row, f.v_row, there, f.d, threadIdx.x);
    };
    if (threadIdx.x == 0) any_not_finite = 0;
    if (tiles) stage(stages[0], 0);
    const int unseen = first_unseen<KEYS>(s, seen_by(f, s, first));  // by one of the workgroup's rows: the same for all its waves
    for (int t = 0, turn = 0; t < tiles; ++t, turn ^= 1) {
        char* keys = stages[turn];
        lds_loads_arrived();
        __syncthreads();
        if (t + 1 < tiles) stage(stages[turn ^ 1], t + 1);
        const int key = t * KEYS;
        // Keys that only some rows see: a weight of 0 would not keep an infinity or NaN out, so they are cleared, and rows that see them are spoiled at the end.
        if (t >= unseen) {
            const bool of_keys = Tile::template clear_not_finite<256>(keys, threadIdx.x), of_values = Tile::template clear_not_finite<256>(keys + Tile::BYTES, threadIdx.x);
            if (of_keys || of_values) any_not_finite = 1;
            __syncthreads();
        }
        if (key >= most_seen) continue;
#pragma unroll
        for (int kb = 0; kb < KEYS / 32; ++kb) {
            f32x16 p = (f32x16)(0.f), ds = (f32x16)(0.f);
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) {
                p = mma32<DT>(Tile::along(keys, kb, i, lane), q[i], p);
                ds = mma32<DT>(Tile::along(keys + Tile::BYTES, kb, i, lane), dout[i], ds);
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) p[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x], c, -base));
            if (key + KEYS > least_seen) {
                const int left = seen - key - 4 * (lane >> 5);
#pragma unroll
                for (int x = 0; x < 16; ++x) p[x] = 32 * kb + tile_row(x, 0) < left ? p[x] : 0.f;
            }
            const float less = delta * digits.by;
#pragma unroll
            for (int x = 0; x < 16; ++x) ds[x] = p[x] * (digits.USED ? __builtin_fmaf(ds[x], digits.by, -less) : ds[x] - delta);
            digits.fit(ds, dq);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 g = round_half<DT>(ds, half);
#pragma unroll
                for (int i = 0; i < DB; ++i) dq[i] = mma32<DT>(Tile::across(keys, i, 2 * kb + half, lane), g, dq[i]);
            }
        }
    }
    float scale = f.scale / digits.by;
    if (__builtin_expect(tiles && any_not_finite, 0)) {
        for (int j = unseen * KEYS; j < min(tiles * KEYS, s.lk); ++j) {
            const bool bad = not_finite(k + j * f.k_row, f.d, lane) || not_finite(v + j * f.v_row, f.d, lane);
            if (bad && j < seen) scale = __builtin_nanf("");
        }
    }
    if (r >= rows) return;
    const int token = token_of(f, r), head = group * f.share + (r - token * f.share);
    E* to = (E*)a.dq + (s.q0 + token) * a.dq_row + head * a.dq_head;
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        float x[2][8];
        rows_of_eight(dq[i], x);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int at = 32 * i + 16 * p + 8 * (lane >> 5);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[p][e] *= scale;
            if (at < f.d) store_elems<DT>(to + at, f.d - at, x[p]);
        }
    }
}

// dk and dv: a wave has 32 keys and runs over tiles of 64 rows, 32 of long vectors (of all the heads that share the key head), which its workgroup's four waves share.
// Four products a tile: 168 us on the sequences above, bound as the first pass is (matrix cores 30 %, vector units 33 %).  At more than 96 elements 48 bytes a lane (fp16: 92) are
// in scratch memory.
template <int DT, int DB, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_dkv_kernel(AttentionBackArgs a) {
    constexpr int KEYS = 128, ROWS = DB <= 2 ? 64 : 32;
    constexpr bool KEYS_IN_LDS = DB > 2;  // long vectors: dk, dv, k and v together are more registers than two waves a SIMD have, so k is read again and again
    using Tile = HeadTile<DT, DB, ROWS>;
    using KeyTile = HeadTile<DT, DB, KEYS>;
    typedef typename Elem<DT>::T E;
    // a stage: the rows' q, their dout, and two numbers for each (room for a wave's 64 lanes of both)
    constexpr int STAGE = 2 * Tile::BYTES + 2 * 64 * 4, STAGES = DIRECT && !KEYS_IN_LDS ? 3 : 2;
    __shared__ __attribute__((aligned(16))) char stages[STAGES][STAGE];
    __shared__ __attribute__((aligned(16))) char key_tile[KEYS_IN_LDS ? KeyTile::BYTES : 16];
    __shared__ int any_not_finite;
    const AttentionArgs& f = a.forward;
    int group, tile;
    deal(a.key_tiles, false, group, tile);
    const Sequence s = find_sequence<KEYS, true>(f, tile);
    if (s.index < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = s.lq * f.share, first = s.tile * KEYS, mine = first + wave * 32, key = mine + (lane & 31);
    // the first row that sees key j
    auto sees = [&](int j) { return f.causal ? (int)min((int64_t)rows, max((int64_t)0, (int64_t)f.share * ((int64_t)j - s.lk + s.lq))) : 0; };
    const int from_row = sees(key), wave_first = sees(mine), wave_all = sees(min(mine + 32, s.lk) - 1);

    uint4 k[KEYS_IN_LDS ? 1 : 2 * DB], v[2 * DB];
    if constexpr (KEYS_IN_LDS)
        KeyTile::template stage<256, false>(key_tile, (const E*)f.k + (s.k0 + (int64_t)first) * f.k_row + group * f.k_head, f.k_row, s.lk - first, f.d, threadIdx.x);
    {
        const E* at_k = (const E*)f.k + (s.k0 + (int64_t)key) * f.k_row + group * f.k_head;
        const E* at_v = (const E*)f.v + (s.k0 + (int64_t)key) * f.v_row + group * f.v_head;
#pragma unroll
        for (int i = 0; i < 2 * DB; ++i) {
            const int at = 16 * i + 8 * (lane >> 5), count = key < s.lk ? f.d - at : 0;
            if constexpr (!KEYS_IN_LDS) k[i] = load_run<DT>(at_k + at, count);
            v[i] = load_run<DT>(at_v + at, count);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) dk[i] = dv[i] = (f32x16)(0.f);
    const float c = f.scale * LOG2E, unshift = 1.f / (float)(1 << WEIGHT_SHIFT<DT>);
    Digits<DT> digits;

    // The rows of a tile are share heads of ROWS / share tokens each where share divides ROWS: then a thread's place in the tile says how far
    // its row lies from the tile's first.  Otherwise its rows are found one by one.
    const bool even = ROWS % f.share == 0;
    constexpr int PER_THREAD = ROWS * Tile::RUNS / 256, LOADS = 2 * PER_THREAD + 1;  // a stage's loads of a wave
    static_assert(PER_THREAD > 0 && ROWS * Tile::RUNS % 256 == 0, "every thread has as many runs");
    const float* stats_of = a.stats + (wave & 1) * (int64_t)f.tq * f.heads;
    auto stage = [&](char* to, int row0) {
        const int token0 = token_of(f, row0);
        const E* of_q = (const E*)f.q + (s.q0 + token0) * f.q_row + group * f.share * f.q_head;
        const E* of_dout = (const E*)a.dout + (s.q0 + token0) * a.dout_row + group * f.share * a.dout_head;
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / Tile::RUNS, run = (at % Tile::RUNS) ^ Tile::exchanged(row), r = row0 + row;
            const int token = even ? token_of(f, row) : token_of(f, r) - token0, head = even ? row - token * f.share : r - (token0 + token) * f.share;
            if constexpr (DIRECT) {
                const bool there = r < rows && run * 8 < f.d;
                const uint32_t q_at = (uint32_t)(token * (int)f.q_row + head * (int)f.q_head + run * 8) * 2;
                const uint32_t dout_at = (uint32_t)(token * (int)a.dout_row + head * (int)a.dout_head + run * 8) * 2;
                const uint32_t lds = lds_address(to) + (i * 256 + wave * 64) * 16;
                load_to_lds(buffer_of(of_q, 0x80000000u), there ? q_at : 0xFFFFFFF0u, lds);
                load_to_lds(buffer_of(of_dout, 0x80000000u), there ? dout_at : 0xFFFFFFF0u, lds + Tile::BYTES);
            } else {
                const int count = r < rows ? f.d - run * 8 : 0;
                *reinterpret_cast<uint4*>(to + at * 16) = load_run<DT>(of_q + token * f.q_row + head * f.q_head + run * 8, count);
                *reinterpret_cast<uint4*>(to + Tile::BYTES + at * 16) = load_run<DT>(of_dout + token * a.dout_row + head * a.dout_head + run * 8, count);
            }
        }
        // The two numbers of each row, the first from even waves, the second from odd ones (twice, so that all waves wait for as many loads).  Rows that
        // there are not get 0 and so a weight of 1, and have a q and dout of 0.
        const int r = row0 + lane, token = token_of(f, r), head = group * f.share + (r - token * f.share);
        const bool there = lane < ROWS && r < rows;
        if constexpr (DIRECT) {
            const uint32_t offset = (uint32_t)((token - token0) * f.heads + head) * 4;
            load_word_to_lds(buffer_of(stats_of + (s.q0 + (int64_t)token0) * f.heads, 0x80000000u), there ? offset : 0xFFFFFFF0u, lds_address(to) + 2 * Tile::BYTES + (wave & 1) * 256);
        } else {
            reinterpret_cast<float*>(to + 2 * Tile::BYTES)[(wave & 1) * 64 + lane] = there ? stats_of[(s.q0 + (int64_t)token) * f.heads + head] : 0.f;
        }
    };
    const int start = sees(first) / ROWS * ROWS, all_see = sees(min(first + KEYS, s.lk) - 1);  // rows from all_see on see all of the workgroup's keys
    if (threadIdx.x == 0) any_not_finite = 0;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (start + i * ROWS < rows) stage(stages[i], start + i * ROWS);
    int turn = 0;
    for (int row = start; row < rows; row += ROWS, turn = turn + 1 == STAGES ? 0 : turn + 1) {
        char* now = stages[turn];
        if (STAGES == 3 && row + ROWS < rows) lds_loads_left<LOADS>();
        else lds_loads_arrived();
        __syncthreads();
        if (row + (STAGES - 1) * ROWS < rows) stage(stages[turn == 0 ? STAGES - 1 : turn - 1], row + (STAGES - 1) * ROWS);
        // Rows that do not see all keys: as in the first pass, what is no number in them is cleared, and spoils the keys that they see at the end
        // (causal sequences of up to 2048: 107 to 110 us; longer ones less).
        if (row < all_see) {
            const bool of_q = Tile::template clear_not_finite<256>(now, threadIdx.x), of_dout = Tile::template clear_not_finite<256>(now + Tile::BYTES, threadIdx.x);
            bool bad = of_q || of_dout;
            if (threadIdx.x < ROWS) {
                float& delta = reinterpret_cast<float*>(now + 2 * Tile::BYTES)[64 + threadIdx.x];
                if (!(__builtin_fabsf(delta) < __builtin_inff())) delta = 0.f, bad = true;
            }
            if (bad) any_not_finite = 1;
            __syncthreads();
        }
        if (row + ROWS <= wave_first || mine >= s.lk) continue;
#pragma unroll
        for (int block = 0; block < ROWS / 32; ++block) {
            const float* stats = reinterpret_cast<const float*>(now + 2 * Tile::BYTES) + 32 * block + 4 * (lane >> 5);
            f32x16 p = (f32x16)(0.f), ds;
#pragma unroll
            for (int x = 0; x < 16; ++x) ds[x] = stats[64 + tile_row(x, 0)];  // dout v^T - delta: the product starts there
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) {
                p = mma32<DT>(Tile::along(now, block, i, lane), KEYS_IN_LDS ? KeyTile::along(key_tile, wave, i, lane) : k[KEYS_IN_LDS ? 0 : i], p);
                ds = mma32<DT>(Tile::along(now + Tile::BYTES, block, i, lane), v[i], ds);
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) p[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x], c, -stats[tile_row(x, 0)]));
            const float by = unshift * digits.by;
            if (row + 32 * block < wave_all) {
                const int least = from_row - row - 32 * block - 4 * (lane >> 5);
#pragma unroll
                for (int x = 0; x < 16; ++x) p[x] = tile_row(x, 0) >= least ? p[x] : 0.f;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) ds[x] = digits.USED ? p[x] * (ds[x] * by) : p[x] * ds[x];
            digits.fit(ds, dk);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 w = round_half<DT>(p, half), g = round_half<DT>(ds, half);
#pragma unroll
                for (int i = 0; i < DB; ++i) {
                    dv[i] = mma32<DT>(Tile::across(now + Tile::BYTES, i, 2 * block + half, lane), w, dv[i]);
                    dk[i] = mma32<DT>(Tile::across(now, i, 2 * block + half, lane), g, dk[i]);
                }
            }
        }
    }
    float spoiled[2] = {1.f, 1.f};  // dk, dv
    if (__builtin_expect(start < rows && any_not_finite, 0)) {
        for (int r = start; r < min((all_see + ROWS - 1) / ROWS * ROWS, rows); ++r) {
            const int token = token_of(f, r), head = group * f.share + (r - token * f.share);
            const bool bad = not_finite((const E*)f.q + (s.q0 + token) * f.q_row + head * f.q_head, f.d, lane) ||
                             not_finite((const E*)a.dout + (s.q0 + token) * a.dout_row + head * a.dout_head, f.d, lane);
            const float delta = a.stats[flat_row(f, s, group, r) + (int64_t)f.tq * f.heads];
            if (r < from_row) continue;
            if (bad) spoiled[1] = __builtin_nanf("");
            if (bad || !(__builtin_fabsf(delta) < __builtin_inff())) spoiled[0] = __builtin_nanf("");
        }
    }
    if (key >= s.lk) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!(which ? a.dv : a.dk)) continue;
        E* to = which ? (E*)a.dv + (s.k0 + (int64_t)key) * a.dv_row + group * a.dv_head : (E*)a.dk + (s.k0 + (int64_t)key) * a.dk_row + group * a.dk_head;
        const float scale = (which ? unshift : f.scale / digits.by) * spoiled[which];
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            float x[2][8];
            rows_of_eight(which ? dv[i] : dk[i], x);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int at = 32 * i + 16 * p + 8 * (lane >> 5);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[p][e] *= scale;
                if (at < f.d) store_elems<DT>(to + at, f.d - at, x[p]);
            }
        }
    }
}

template <int DT, int DB>
hipError_t run(const AttentionBackArgs& a, hipStream_t s) {
    if (a.forward.tq > 0) {
        const hipError_t e = launch(TK_ATTENTION_BACKWARD, a.forward.direct ? attention_dq_kernel<DT, DB, true> : attention_dq_kernel<DT, DB, false>,
                                    dim3((unsigned)(a.forward.row_tiles * a.forward.groups)), dim3(256), 0, s, a);
        if (e != hipSuccess) return e;
    }
    if (a.forward.tk < 1 || (!a.dk && !a.dv)) return hipSuccess;
    return launch(TK_ATTENTION_BACKWARD, a.direct_rows ? attention_dkv_kernel<DT, DB, true> : attention_dkv_kernel<DT, DB, false>,
                  dim3((unsigned)(a.key_tiles * a.forward.groups)), dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_attention_backward(AttentionBackArgs a, int dtype, hipStream_t s) {
    // at most so many tiles, whatever the sequences' lengths
    const int64_t rows = (int64_t)a.forward.tq * a.forward.share, keys = a.forward.tk;
    a.forward.row_tiles = (int)std::min(rows, (rows + 127) / 128 + a.forward.batch - 1);
    a.key_tiles = (int)std::min(keys, (keys + 127) / 128 + a.forward.batch - 1);
    const int blocks = (a.forward.d + 31) / 32;
    auto with_type = [&](auto dt) {
        constexpr int DT = dt.value;
        switch (blocks) {
            case 1: return run<DT, 1>(a, s);
            case 2: return run<DT, 2>(a, s);
            case 3: return run<DT, 3>(a, s);
            default: return run<DT, 4>(a, s);
        }
    };
    return dtype == FNN_F16 ? with_type(std::integral_constant<int, CT_F16>()) : with_type(std::integral_constant<int, CT_BF16>());
}

}  // namespace fnn
