// Attention over packed sequences (fnn_attention): out = softmax(scale q k^T) v, one pass over the keys with a running maximum
// and sum, the scores never leaving registers.
//
// Scores are formed as k q^T, so a lane owns one query (row) and 16 keys of each 32 x 32 block: the softmax needs one exchange between two lanes,
// and the weights, rounded to the operands' type, are the second product's operand as they lie -- v^T is read from LDS by
// transposing reads in the same order of keys.  The result is out^T, again one row per lane, so rescaling it is a plain multiplication.
#include <type_traits>

#include "attention_device.hpp"
#include "trace.hpp"

namespace fnn {

namespace {

// Weights are formed 2^7 times too large in fp16, at most 2^15: those of many keys far below the largest, which may weigh as much together, would lose bits below
// the type's normal range.  The factor leaves with the sum.
template <int DT>
constexpr float WEIGHT_LIFT = DT == CT_F16 ? 7.f : 0.f;
// lse from the largest score and the sum of lifted weights; no key: minus infinity
template <int DT>
__device__ __forceinline__ float lse_of(float top, float sum, float scale) {
    return top * scale + logf(DT == CT_F16 ? sum * 0x1p-7f : sum);
}
// What the weights of keys whose largest score is `top` are multiplied by beside others whose largest is `most`: 0 for no keys.
__device__ __forceinline__ float weight_beside(float top, float most, float c) {
    return top > -__builtin_inff() ? __builtin_amdgcn_exp2f((top - most) * c) : 0.f;
}

// One wave's 32 rows, a row per lane of either half.
template <int DT, int DB, int KEYS>
struct Rows {
    using Tile = HeadTile<DT, DB, KEYS>;
    typedef typename Elem<DT>::T E;
    static constexpr int KB = KEYS / 32;
    uint4 q[2 * DB];
    f32x16 out[DB];
    float top, sum;  // of the keys so far: a score that none exceeds by 8 / c, and (this half's share of) the sum of exp2(c (score - top) + WEIGHT_LIFT)

    __device__ __forceinline__ void begin(const AttentionArgs& a, const Sequence& s, int group, int row, int rows, int lane) {
        load_row<DT, DB>(a.q, a.q_row, a.q_head, a, s, group, row + (lane & 31), rows, lane, q);
#pragma unroll
        for (int i = 0; i < DB; ++i) out[i] = (f32x16)(0.f);
        top = -__builtin_inff();
        sum = 0.f;
    }

    // KEYS more keys, the first of which is number `key`; `seen`: how many of the sequence's keys each row sees.  mask (the same in every
    // lane): some row may not see all of these.  Only the masking itself is branched over: two copies of all of it kept two copies of `out` in registers.
    __device__ __forceinline__ void keys(const char* k, const char* v, float c, int key, int seen, bool mask, int lane) {
        f32x16 score[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) score[kb] = (f32x16)(0.f);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 2 * DB; ++i) {
                const uint4 f = Tile::along(k, kb, i, lane);
                score[kb] = mma32<DT>(f, q[i], score[kb]);
            }
        __builtin_amdgcn_sched_barrier(0);
        float most = -__builtin_inff();
        if (mask) {
            const int left = seen - key - 4 * (lane >> 5);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) score[kb][r] = 32 * kb + tile_row(r, 0) < left ? score[kb][r] : -__builtin_inff();
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, score[kb][r]);
        most = across_halves_max(most);
        // What is so far is rescaled only where some row's maximum rises by a factor of 2^8 and more: weights may as well reach 256.
        if (__ballot((most - top) * c > 8.f)) {
            most = __builtin_fmaxf(most, top);
            const float keep = weight_beside(top, most, c);
            top = most;
            sum *= keep;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) out[i][r] *= keep;
        }
        // exp2(c score - c top), for rows that have seen no key yet of anything finite in top's place: their weights are 0.  c top is rounded, which all weights of a row
        // have in common; where it is so large that this is a factor to notice (2^31: one that overflows), the difference comes first.
        const float shown = top > -__builtin_inff() ? top : 0.f;
        float base = shown * c - WEIGHT_LIFT<DT>;
        if (__ballot(__builtin_fabsf(base) > 1024.f)) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) score[kb][r] -= shown;
            base = -WEIGHT_LIFT<DT>;
        }
        // summed up before they are rounded: lse has fp32's precision
        float more = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                score[kb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[kb][r], c, -base));
                more += score[kb][r];
            }
        sum += more;
        __builtin_amdgcn_sched_barrier(0);
        // the weights are at most 2^8, lifted, and rounded to the values' type, as the matrix instructions take them; their sum is of the unrounded ones
#pragma unroll
        for (int t = 0; t < 2 * KB; ++t) {
            const uint4 p = round_half<DT>(score[t >> 1], t & 1);
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const uint4 f = Tile::across(v, i, t, lane);
                out[i] = mma32<DT>(f, p, out[i]);
            }
        }
    }

    // A causal tile that some rows see only a part of is multiplied with its values' infinities and NaN cleared, since a weight of 0 would not keep them
    // out; here the rows that see them get them.  No call without such values comes here.
    __device__ __forceinline__ void add_not_finite(const E* v, int64_t stride, int d, int key, int end, int seen, int lane) {
#pragma unroll 1
        for (int j = key; j < end; ++j) {
            const E* of_key = v + j * stride;
            if (!not_finite(of_key, d, lane)) continue;
#pragma unroll
            for (int i = 0; i < DB; ++i) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int e = 32 * i + tile_row(r, lane >> 5);
                    const float x = e < d ? (float)of_key[e] : 0.f;
                    const bool bad = !(__builtin_fabsf(x) < __builtin_inff());
                    out[i][r] += bad && j < seen ? x : 0.f;
                    if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
};

// Results of one row: element runs of 8 (`at` from 0, `count` of them exist).
template <int DT>
__device__ __forceinline__ void put_run(const AttentionArgs& a, const Sequence& s, int group, int r, int at, const float (&v)[8]) {
    typedef typename Elem<DT>::T E;
    const int token = token_of(a, r), head = group * a.share + (r - token * a.share);
    store_elems<DT>((E*)a.out + (s.q0 + token) * a.out_row + head * a.out_head + at, a.d - at, v);
}

constexpr int MOST_SPLITS = 64, MOST_KEYS = 1 << 30;

// Shares of a split call: [split][rows] of {the largest score, the sum}, then, from the next 16 bytes on, [split][rows][d rounded up to 8].
__host__ __device__ __forceinline__ int64_t stats_floats(int64_t shares) { return (shares * 2 + 3) & ~(int64_t)3; }
__device__ __forceinline__ float* share_stats(const AttentionArgs& a, int split, int64_t row) {
    return a.partial + ((int64_t)split * a.tq * a.heads + row) * 2;
}
__device__ __forceinline__ float* share_row(const AttentionArgs& a, int split, int64_t row) {
    return a.partial + stats_floats((int64_t)a.splits * a.tq * a.heads) + ((int64_t)split * a.tq * a.heads + row) * a.d_pad;
}

// The sum of a share whose row sees keys, each with a score of minus infinity: they weigh nothing beside others, but are no softmax by themselves.  The share of
// no keys has a sum of 0.
constexpr float NO_WEIGHT = -1.f;

// `part`: the first of the keys that `w` is of; `any`: whether there are some.
template <int DT, int DB, int KEYS>
__device__ __forceinline__ void finish_rows(const AttentionArgs& a, const Sequence& s, int group, int row, int rows, int part, bool any, const Rows<DT, DB, KEYS>& w, int lane) {
    const int c = lane & 31, h = lane >> 5;
    const int r = row + c;
    const float total = across_halves_sum(w.sum);
    const bool sees = any && seen_by(a, s, min(r, rows - 1)) > part;
    float scale = 1.f;
    if (a.splits == 1) scale = total > 0.f ? 1.f / total : sees ? __builtin_nanf("") : 0.f;  // a row that sees no key is 0
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        float v[2][8];
        rows_of_eight(w.out[i], v);
        if (r >= rows) continue;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int at = 32 * i + 16 * p + 8 * h;
            if (at >= a.d) continue;
            if (a.splits == 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] *= scale;
                put_run<DT>(a, s, group, r, at, v[p]);
            } else if (any) {  // the share of no keys is told by its statistics alone
                float* to = share_row(a, blockIdx.y, flat_row(a, s, group, r)) + at;
                reinterpret_cast<f32x4*>(to)[0] = f32x4{v[p][0], v[p][1], v[p][2], v[p][3]};
                reinterpret_cast<f32x4*>(to)[1] = f32x4{v[p][4], v[p][5], v[p][6], v[p][7]};
            }
        }
    }
    if (r >= rows || h) return;
    if (a.splits > 1) {
        float* to = share_stats(a, blockIdx.y, flat_row(a, s, group, r));
        to[0] = w.top;
        to[1] = sees && total == 0.f ? NO_WEIGHT : total;
    } else if (a.lse) {
        a.lse[flat_row(a, s, group, r)] = lse_of<DT>(w.top, total, a.scale);
    }
}

// The tiles of keys that this workgroup's part (blockIdx.y) of a split call has: as many parts as there are whole ones of part_tiles, so that
// sequences of different lengths are cut into pieces of one size; the parts beyond have none.
__device__ __forceinline__ void part_of(const AttentionArgs& a, int tiles, int& t0, int& t1) {
    const int part = blockIdx.y, parts = min(max((tiles + a.part_tiles - 1) / a.part_tiles, 1), a.splits);
    t0 = part < parts ? (int)((int64_t)tiles * part / parts) : 0;
    t1 = part < parts ? (int)((int64_t)tiles * (part + 1) / parts) : 0;
}

// Many rows: a workgroup's four waves have 32 rows each and share tiles of 64 keys.  32 sequences of 768 rows and keys, 16 heads of 64, bf16: 123 us, 630 TFLOP/s; packed
// causal rows up to 4001, 16 heads on 8, 128 elements, fp16: 555 us, 740 TFLOP/s.  Neither the matrix cores (busy 26 and 34 % of the cycles) nor the vector units (51 and 38 %) bound
// it: a wave's chain of product, softmax (per score a multiply-add, a maximum, an exponential, an addition and half a rounding) and product is serial, and the
// two waves or so of a SIMD do not fill its waits (waves wait 48 and 40 % of their cycles).
template <int DT, int DB, bool DIRECT>
__global__ __launch_bounds__(256, 2) void attention_kernel(AttentionArgs a) {
    constexpr int KEYS = 64, ROWS = 128;
    using W = Rows<DT, DB, KEYS>;
    using Tile = typename W::Tile;
    typedef typename Elem<DT>::T E;
    __shared__ __attribute__((aligned(16))) char stages[2][2 * Tile::BYTES];
    __shared__ int any_not_finite;
    int group, tile;
    deal(a.row_tiles, a.causal, group, tile);
    const Sequence s = find_sequence<ROWS>(a, tile);
    if (s.index < 0) return;
    if (threadIdx.x == 0) any_not_finite = 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = s.lq * a.share, first = s.tile * ROWS, mine = first + wave * 32;
    const int most = seen_by(a, s, min(first + ROWS, rows) - 1);
    int t0, t1;
    part_of(a, (most + KEYS - 1) / KEYS, t0, t1);

    const int least_seen = seen_by(a, s, min(mine, rows - 1));
    const int seen = seen_by(a, s, min(mine + (lane & 31), rows - 1));
    const float c = a.scale * LOG2E;
    const E* k = (const E*)a.k + s.k0 * a.k_row + group * a.k_head;
    const E* v = (const E*)a.v + s.k0 * a.v_row + group * a.v_head;
    auto stage = [&](char* to, int t) {
        const int key = t * KEYS, there = min(KEYS, s.lk - key);
        Tile::template stage<256, DIRECT>(to, k + key * a.k_row, a.k_row, there, a.d, threadIdx.x);
        Tile::template stage<256, DIRECT>(to + Tile::BYTES, v + key * a.v_row, a.v_row, there, a.d, threadIdx.x);
    };
    const int unseen = first_unseen<KEYS>(s, seen_by(a, s, first));  // by one of the workgroup's rows: the same for all its waves
    auto next_tile = [&](int t, int turn) {
        lds_loads_arrived();
        __syncthreads();
        if (t + 1 < t1) stage(stages[turn ^ 1], t + 1);
        if (t < unseen) return;
        if (Tile::template clear_not_finite<256>(stages[turn] + Tile::BYTES, threadIdx.x)) any_not_finite = 1;
        __syncthreads();
    };
    if (t0 < t1) stage(stages[0], t0);
    if (mine >= rows) {  // a wave without rows only brings tiles
        for (int t = t0, turn = 0; t < t1; ++t, turn ^= 1) next_tile(t, turn);
        return;
    }
    W w;
    w.begin(a, s, group, mine, rows, lane);
    // Every wave multiplies every tile, the last causal ones too that its rows do not see: passed over, they cost a copy of `out` on every tile.
    for (int t = t0, turn = 0; t < t1; ++t, turn ^= 1) {
        const char* now = stages[turn];
        next_tile(t, turn);
        const int key = t * KEYS;
        w.keys(now, now + Tile::BYTES, c, key, seen, key + KEYS > least_seen, lane);
    }
    if (__builtin_expect(t0 < t1 && any_not_finite, 0)) w.add_not_finite(v, a.v_row, a.d, max(t0, unseen) * KEYS, min(t1 * KEYS, s.lk), seen, lane);
    finish_rows(a, s, group, mine, rows, t0 * KEYS, t0 < t1, w, lane);
}

// Few rows (a token or some at the end of a cache): the time is that of reading the keys once.  Every wave has the same 32 rows and tiles of
// 32 keys of its own, which only it waits for; at the end the four join in LDS.  32 caches of up to 4096 keys, one row for each of 16 heads on 4 of 128, bf16:
// 49 us for 119 MB, 2.4 TB/s (one workgroup a compute unit at 128 KB of stages, and caches whose lengths differ); 32 equal caches of 4096 keys 55 us for
// 268 MB, 4.9 TB/s.
template <int DT, int DB, bool DIRECT>
__global__ __launch_bounds__(256) void attention_few_kernel(AttentionArgs a) {
    constexpr int KEYS = 32, ROWS = 32;
    using W = Rows<DT, DB, KEYS>;
    using Tile = typename W::Tile;
    typedef typename Elem<DT>::T E;
    constexpr int PER_WAVE = 4 * Tile::BYTES;  // two stages of keys and values
    __shared__ __attribute__((aligned(16))) char stages[4 * PER_WAVE];
    int group, tile;
    deal(a.row_tiles, a.causal, group, tile);
    const Sequence s = find_sequence<ROWS>(a, tile);
    if (s.index < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = s.lq * a.share, first = s.tile * ROWS;
    const int most = seen_by(a, s, min(first + ROWS, rows) - 1), least = seen_by(a, s, first);
    int t0, t1;
    part_of(a, (most + KEYS - 1) / KEYS, t0, t1);

    const int seen = seen_by(a, s, min(first + (lane & 31), rows - 1));
    const float c = a.scale * LOG2E;
    const E* k = (const E*)a.k + s.k0 * a.k_row + group * a.k_head;
    const E* v = (const E*)a.v + s.k0 * a.v_row + group * a.v_head;
    char* mine = stages + wave * PER_WAVE;
    auto stage = [&](char* to, int t) {
        const int key = t * KEYS, there = min(KEYS, s.lk - key);
        Tile::template stage<64, DIRECT>(to, k + key * a.k_row, a.k_row, there, a.d, lane);
        Tile::template stage<64, DIRECT>(to + Tile::BYTES, v + key * a.v_row, a.v_row, there, a.d, lane);
    };
    int turn = 0;
    bool cleared = false;
    const int unseen = first_unseen<KEYS>(s, least);
    if (t0 + wave < t1) stage(mine, t0 + wave);
    W w;
    w.begin(a, s, group, first, rows, lane);
    for (int t = t0 + wave; t < t1; t += 4, turn ^= 1) {
        char* now = mine + turn * 2 * Tile::BYTES;
        char* next = mine + (turn ^ 1) * 2 * Tile::BYTES;
        lds_loads_arrived();
        if (t + 4 < t1) stage(next, t + 4);
        const int key = t * KEYS;
        if (__builtin_expect(t >= unseen, 0)) {  // (laid out as if it were usual, 2 us more for one token's caches)
            cleared |= __ballot(Tile::template clear_not_finite<64>(now + Tile::BYTES, lane)) != 0;
            __builtin_amdgcn_wave_barrier();
        }
        w.keys(now, now + Tile::BYTES, c, key, seen, key + KEYS > least, lane);
    }
    if (__builtin_expect(cleared, 0))
#pragma unroll 1
        for (int t = t0 + wave; t < t1; t += 4)
            if (t >= unseen) w.add_not_finite(v, a.v_row, a.d, t * KEYS, min((t + 1) * KEYS, s.lk), seen, lane);
    // The waves' results, each in its own stages' place: top and sum per lane, then the registers.
    __syncthreads();
    float* held = reinterpret_cast<float*>(stages) + wave * (64 * (2 + 16 * DB));
    held[lane] = w.top;
    held[64 + lane] = w.sum;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) held[(2 + 16 * i + r) * 64 + lane] = w.out[i][r];
    __syncthreads();
    if (wave) return;
    const float* all = reinterpret_cast<const float*>(stages);
    constexpr int EACH = 64 * (2 + 16 * DB);
    float top = w.top;
#pragma unroll
    for (int i = 1; i < 4; ++i) top = __builtin_fmaxf(top, all[i * EACH + lane]);
    float sum = 0.f;
    f32x16 out[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) out[i] = (f32x16)(0.f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float* from = all + j * EACH;
        const float keep = weight_beside(from[lane], top, c);
        sum = __builtin_fmaf(from[64 + lane], keep, sum);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) out[i][r] = __builtin_fmaf(from[(2 + 16 * i + r) * 64 + lane], keep, out[i][r]);
    }
    w.top = top;
    w.sum = sum;
#pragma unroll
    for (int i = 0; i < DB; ++i) w.out[i] = out[i];
    finish_rows(a, s, group, first, rows, t0 * KEYS, t0 < t1, w, lane);
}

// Joins the shares of a split call, each share scaled by exp of its maximum less the largest, in the order of the shares (32 x 16 rows: 4.2 us, a launch): groups of 32 lanes, a lane four elements of a row.  Of few rows each has a workgroup, whose eight groups take
// shares in turn; of many (GROUPS == 1) every group has a row of its own.
template <int DT, int GROUPS>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
    __shared__ f32x4 joined[GROUPS][32];
    const int place = threadIdx.x & 31, group = threadIdx.x >> 5, mine = GROUPS == 1 ? 0 : group;
    const int64_t row = GROUPS == 1 ? (int64_t)blockIdx.x * 8 + group : blockIdx.x;
    if (row >= (int64_t)a.tq * a.heads) return;
    const int token = (int)(row / a.heads), head = (int)(row - (int64_t)token * a.heads);
    if (a.cu_q && (token < max(a.cu_q[0], 0) || token >= a.cu_q[a.batch])) return;  // a row of no sequence stays as it is
    const float c = a.scale * LOG2E;
    float top = -__builtin_inff();
    bool sees = false;
    for (int s = place; s < a.splits; s += 32) {
        const float* stats = share_stats(a, s, row);
        top = __builtin_fmaxf(top, stats[0]);
        sees |= stats[1] != 0.f;
    }
#pragma unroll
    for (int step = 1; step < 32; step <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, step));
    sees = (uint32_t)(__ballot(sees) >> (threadIdx.x & 32)) != 0u;
    float sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = mine; s < a.splits; s += GROUPS) {
        // What the share of no keys has for a row was not written, and is read all the same (its memory is there) so that no load waits for another.  A factor of
        // 0 is no reason to pass a share over: it may hold NaN alone, which no maximum tells of, or infinite values.
        const float* stats = share_stats(a, s, row);
        const bool empty = stats[1] == 0.f;
        const float keep = weight_beside(stats[0], top, c);
        sum = empty ? sum : __builtin_fmaf(stats[1] == NO_WEIGHT ? 0.f : stats[1], keep, sum);
        if (4 * place < a.d) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(share_row(a, s, row) + 4 * place);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = empty ? x[e] : __builtin_fmaf(y[e], keep, x[e]);
        }
    }
    if constexpr (GROUPS > 1) {
        __shared__ float sums[GROUPS];
        joined[group][place] = x;
        if (place == 0) sums[group] = sum;
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) x += joined[g][place], sum += sums[g];
    }
    const float scale = sum > 0.f ? 1.f / sum : sees ? __builtin_nanf("") : 0.f;
    const float v[4] = {x[0] * scale, x[1] * scale, x[2] * scale, x[3] * scale};
    if (4 * place < a.d) store_elems<DT, 4>((typename Elem<DT>::T*)a.out + token * a.out_row + head * a.out_head + 4 * place, a.d - 4 * place, v);
    if (place == 0 && a.lse) a.lse[row] = lse_of<DT>(top, sum, a.scale);
}

// From the sizes alone: whether the rows of a sequence are few on average (one wave's worth), and into how many parts the keys may be split: parts of
// the size that makes 320 of them in all, a little more than one a compute unit, and not less than 256 keys, below which a part's start costs more than it
// saves.  Longer sequences than the average have longer parts: as many of the right size for them all would be workgroups without keys for the others, each
// of which holds a compute unit's LDS for 2 us (32 caches of 4096 keys, 4 heads of 128: 57 us when it was measured, with parts for sequences twice as long 66).
struct Plan {
    bool few;
    int row_tiles, splits, part_keys;
};
Plan plan_of(int64_t tq, int64_t tk, int64_t batch, int64_t heads, int64_t groups) {
    Plan p;
    const int64_t rows = tq * (heads / groups);
    p.few = rows <= 32 * batch;
    const int64_t tile = p.few ? 32 : 128;
    p.row_tiles = (int)((rows + tile - 1) / tile + batch - 1);
    if (p.row_tiles > rows) p.row_tiles = (int)rows;
    const int64_t average = tk / batch;
    int64_t part = ((int64_t)p.row_tiles * groups * average / 320 + 127) / 128 * 128;
    if (part < 256) part = 256;
    int64_t splits = (average + part - 1) / part;
    if (splits > MOST_SPLITS) splits = MOST_SPLITS;
    p.splits = splits < 1 ? 1 : (int)splits;
    p.part_keys = (int)(part < MOST_KEYS ? part : MOST_KEYS);
    return p;
}

template <int DT, int DB, bool DIRECT>
hipError_t run(const AttentionArgs& a, const Plan& p, hipStream_t s) {
    const dim3 grid((unsigned)(p.row_tiles * a.groups), (unsigned)p.splits);
    const hipError_t e = p.few ? launch(TK_ATTENTION, attention_few_kernel<DT, DB, DIRECT>, grid, dim3(256), 0, s, a)
                               : launch(TK_ATTENTION, attention_kernel<DT, DB, DIRECT>, grid, dim3(256), 0, s, a);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t rows = (int64_t)a.tq * a.heads;
    return rows < 2048 ? launch(TK_ATTENTION, attention_join_kernel<DT, 8>, dim3((unsigned)rows), dim3(256), 0, s, a)
                       : launch(TK_ATTENTION, attention_join_kernel<DT, 1>, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, s, a);
}

}  // namespace

size_t attention_workspace(int64_t tq, int64_t tk, int64_t batch, int64_t heads, int64_t groups, int64_t d) {
    if (tq < 1) return 0;
    const Plan p = plan_of(tq, tk, batch, heads, groups);
    const int64_t shares = p.splits * tq * heads;
    return p.splits > 1 ? (size_t)(stats_floats(shares) + shares * ((d + 7) / 8 * 8)) * sizeof(float) : 0;
}

hipError_t launch_attention(AttentionArgs a, int dtype, hipStream_t s) {
    if (a.tq < 1) return hipSuccess;
    const Plan p = plan_of(a.tq, a.tk, a.batch, a.heads, a.groups);
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.part_tiles = p.part_keys / (p.few ? 32 : 64);
    a.d_pad = (a.d + 7) / 8 * 8;
    const int blocks = (a.d + 31) / 32;
    auto with_type = [&](auto dt) {
        constexpr int DT = dt.value;
        switch (blocks) {
            case 1: return a.direct ? run<DT, 1, true>(a, p, s) : run<DT, 1, false>(a, p, s);
            case 2: return a.direct ? run<DT, 2, true>(a, p, s) : run<DT, 2, false>(a, p, s);
            case 3: return a.direct ? run<DT, 3, true>(a, p, s) : run<DT, 3, false>(a, p, s);
            default: return a.direct ? run<DT, 4, true>(a, p, s) : run<DT, 4, false>(a, p, s);
        }
    };
    return dtype == FNN_F16 ? with_type(std::integral_constant<int, CT_F16>()) : with_type(std::integral_constant<int, CT_BF16>());
}

}  // namespace fnn
