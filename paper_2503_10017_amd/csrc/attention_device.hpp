// What the attention kernels share: which rows and keys a workgroup works on, tiles of keys and values in LDS, and how matrix
// instructions read them.
#pragma once
#include "net_device.hpp"
#include "net_kernels.hpp"

namespace fnn {

// The heads that share a key head are rows of one problem: row r of a sequence is query r / share under head r % share of the group, so a
// tile of keys is read once for all of them, whether the rows are many tokens or many heads of one token.
struct Sequence {
    int index;          // -1: there is none
    int tile;           // which tile of its rows
    int q0, lq, k0, lk; // first query and key, and how many
};

__device__ __forceinline__ void sequence_bounds(const int32_t* cu, int b, int total, int& first, int& count) {
    // a table that runs past its tensor, or backwards, must not lead outside it
    first = cu ? min(max(cu[b], 0), total) : 0;
    count = cu ? min(max(cu[b + 1], first), total) - first : total;
}

// The sequence that tile number `tile` belongs to when every sequence's rows (its queries times `share`; or its keys) are cut into tiles of
// ROWS.  Every wave finds it for itself: 64 sequences at a time, a prefix sum over their tiles.
template <int ROWS, bool BY_KEYS = false>
__device__ __forceinline__ Sequence find_sequence(const AttentionArgs& a, int tile) {
    Sequence s;
    s.index = -1;
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int b = b0 + lane;
        int first = 0, count = 0, other = 0, others = 0;
        if (b < a.batch) {  // both tables at once: one wait
            sequence_bounds(BY_KEYS ? a.cu_k : a.cu_q, b, BY_KEYS ? a.tk : a.tq, first, count);
            sequence_bounds(BY_KEYS ? a.cu_q : a.cu_k, b, BY_KEYS ? a.tq : a.tk, other, others);
        }
        const int tiles = (int)(((int64_t)count * (BY_KEYS ? 1 : a.share) + ROWS - 1) / ROWS);
        int sum = tiles;
#pragma unroll
        for (int step = 1; step < 64; step <<= 1) {
            const int other = __shfl_up(sum, step);
            if (lane >= step) sum += other;
        }
        const uint64_t past = __ballot(before + sum > tile);
        if (past) {
            const int at = __builtin_amdgcn_readfirstlane(__builtin_ctzll(past));
            s.index = b0 + at;
            s.tile = tile - before - __builtin_amdgcn_readlane(sum - tiles, at);
            const int mine = __builtin_amdgcn_readlane(first, at), many = __builtin_amdgcn_readlane(count, at);
            other = __builtin_amdgcn_readlane(other, at);
            others = __builtin_amdgcn_readlane(others, at);
            s.q0 = BY_KEYS ? other : mine;
            s.lq = BY_KEYS ? others : many;
            s.k0 = BY_KEYS ? mine : other;
            s.lk = BY_KEYS ? many : others;
            return s;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return s;
}

// A tile of ROWS rows of one head's vectors (DIM_BLOCKS blocks of 32 elements, the last of which may end early), 16-bit elements, in LDS:
// RUNS runs of 16 bytes a row, exchanged so that what a wave reads at once lies in different banks.
template <int DT, int DIM_BLOCKS, int ROWS>
struct HeadTile {
    typedef typename Elem<DT>::T E;
    static constexpr int RUNS = DIM_BLOCKS == 1 ? 4 : DIM_BLOCKS == 2 ? 8 : 16, ROW_BYTES = RUNS * 16, BYTES = ROWS * ROW_BYTES;
    // LDS serves 256 bytes at a time: 16 lanes of an along() read (16 rows at one run) and 32 of an across() read (4 rows at 4 runs) have to lie in
    // different 16-byte columns of 256 bytes, which hold 4, 2 or 1 rows.
    static __device__ __forceinline__ int exchanged(int row) {
        if constexpr (RUNS == 4) return row >> 2 & 3;
        else if constexpr (RUNS == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
        else return (row & 3) << 2 | (row >> 2 & 3);
    }

    // Rows base[0 .. rows), the rest zero, by THREADS threads of which this is number `thread` (a wave's start together).  DIRECT: runs lie on
    // 16-byte boundaries and offsets fit, so they go straight to LDS and arrive later (lds_loads_arrived); otherwise through registers.
    template <int THREADS, bool DIRECT>
    static __device__ __forceinline__ void stage(char* lds, const E* base, int64_t stride, int rows, int d, int thread) {
        constexpr int PER_THREAD = ROWS * RUNS / THREADS;
        static_assert(ROWS * RUNS % THREADS == 0 && PER_THREAD > 0, "every thread has as many runs");
        if constexpr (DIRECT) {
            const i32x4 buffer = buffer_of(base, rows > 0 ? (uint32_t)(((rows - 1) * stride + d) * 2) : 0u);
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(lds) + (thread & ~63) * 16);
#pragma unroll
            for (int i = 0; i < PER_THREAD; ++i) {
                const int at = i * THREADS + thread, row = at / RUNS, run = (at % RUNS) ^ exchanged(row);
                load_to_lds(buffer, run * 8 < d ? (uint32_t)row * (uint32_t)(stride * 2) + run * 16 : 0xFFFFFFF0u, to + i * THREADS * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER_THREAD; ++i) {
                const int at = i * THREADS + thread, row = at / RUNS, run = (at % RUNS) ^ exchanged(row);
                uint4 v = {0u, 0u, 0u, 0u};
                if (row < rows) v = load_run<DT>(base + row * stride + run * 8, d - run * 8);
                *reinterpret_cast<uint4*>(lds + at * 16) = v;
            }
        }
    }
    // Infinities and NaN of a tile that has arrived become 0, by THREADS threads of which this is number `thread`; whether it had any.
    template <int THREADS>
    static __device__ __forceinline__ bool clear_not_finite(char* lds, int thread) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < BYTES / 16 / THREADS; ++i) {
            uint4* at = reinterpret_cast<uint4*>(lds + (i * THREADS + thread) * 16);
            // an exponent of ones only: what is missing of it is 0, and 0x8000 less that has its top bit set
            constexpr uint32_t EXPONENTS = DT == CT_F16 ? 0x7C007C00u : 0x7F807F80u;
            uint32_t w[4], found = 0u;
            __builtin_memcpy(w, at, 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) found |= 0x80008000u - (~w[e] & EXPONENTS);
            if (found & 0x80008000u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bad = (0x80008000u - (~w[e] & EXPONENTS)) & 0x80008000u;
                    w[e] &= ~(bad | (bad - (bad >> 15)));
                }
                __builtin_memcpy(at, w, 16);
                any = true;
            }
        }
        return any;
    }
    // Rows 32 block .. + 31, elements 16 step + 8 h .. + 7 of each: an operand whose sum runs along the rows' elements.
    static __device__ __forceinline__ uint4 along(const char* lds, int block, int step, int lane) {
        const int row = 32 * block + (lane & 31), run = (2 * step + (lane >> 5)) ^ exchanged(row);
        return *reinterpret_cast<const uint4*>(lds + row * ROW_BYTES + run * 16);
    }
    // Elements 32 block .. + 31 of rows 16 step + 4 h .. + 3 and 8 more: an operand whose sum runs over the rows, in the order in which mma32
    // leaves 16 of its result rows in a lane's registers 8 (step & 1) .. + 7.
    static __device__ __forceinline__ uint4 across(const char* lds, int block, int step, int lane) {
        const int t = lane & 15, row = 16 * step + 4 * (lane >> 5) + (t >> 2);
        const int run = (4 * block + 2 * ((lane >> 4) & 1) + ((t >> 1) & 1)) ^ exchanged(row);
        const char* at = lds + row * ROW_BYTES + (t & 1) * 8;
        const uint2 lo = read_transposed(at + run * 16), hi = read_transposed(at + 8 * ROW_BYTES + (run ^ 2) * 16);  // rows 8 apart are exchanged by 2 more
        return {lo.x, lo.y, hi.x, hi.y};
    }
};

// Registers 8 half .. + 7 of a block of results as an operand's 16 bytes, each rounded to nearest even.
template <int DT>
__device__ __forceinline__ uint4 round_half(const f32x16& x, int half) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, round_two<DT>(x[8 * half + 2 * i], x[8 * half + 2 * i + 1]));
    return {v[0], v[1], v[2], v[3]};
}

__device__ __forceinline__ float across_halves_max(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float across_halves_sum(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// Which group and tile a workgroup has: groups outermost, and each XCD (workgroups go to the 8 in turn) a run of neighbours, which read
// the same keys through one L2.  late_first: the last tiles first (of causal rows they are the long ones).
__device__ __forceinline__ void deal(int tiles, bool late_first, int& group, int& tile) {
    const int total = gridDim.x, id = blockIdx.x, xcd = id & 7, q = total >> 3, r = total & 7;
    const int mine = xcd * q + min(xcd, r) + (id >> 3);
    group = mine / tiles;
    tile = mine - group * tiles;
    if (late_first) tile = tiles - 1 - tile;
}

// Rows of a sequence are counted in 32 bits (the entry points see to it).
__device__ __forceinline__ int token_of(const AttentionArgs& a, int r) { return a.share == 1 ? r : (int)((uint32_t)r / (uint32_t)a.share); }

// How many keys row r sees.
__device__ __forceinline__ int seen_by(const AttentionArgs& a, const Sequence& s, int r) {
    return a.causal ? min(max(token_of(a, r) + (s.lk - s.lq) + 1, 0), s.lk) : s.lk;
}

// Whether one of a vector's d elements is an infinity or NaN; the same in all of a wave's lanes.
template <typename E>
__device__ __forceinline__ bool not_finite(const E* x, int d, int lane) {
    bool bad = false;
    for (int e = lane; e < d; e += 64) bad |= !(__builtin_fabsf((float)x[e]) < __builtin_inff());
    return __ballot(bad) != 0;
}

// Where row r of a group is in lse and what else has a value per query and head.
__device__ __forceinline__ int64_t flat_row(const AttentionArgs& a, const Sequence& s, int group, int r) {
    const int token = token_of(a, r);
    return (s.q0 + (int64_t)token) * a.heads + group * a.share + (r - token * a.share);
}

// One row's vector in an operand's layout: run i of lane (.., h) is elements 16 i + 8 h .. + 7; nothing of a row that there is not.
template <int DT, int DB>
__device__ __forceinline__ void load_row(const void* data, int64_t row_stride, int64_t head_stride, const AttentionArgs& a, const Sequence& s, int group, int r, int rows,
                                         int lane, uint4 (&to)[2 * DB]) {
    const int token = token_of(a, r), head = group * a.share + (r - token * a.share);
    const typename Elem<DT>::T* from = (const typename Elem<DT>::T*)data + (s.q0 + token) * row_stride + head * head_stride;
#pragma unroll
    for (int i = 0; i < 2 * DB; ++i) {
        const int at = 16 * i + 8 * (lane >> 5);
        to[i] = load_run<DT>(from + at, r < rows ? a.d - at : 0);
    }
}

// The first tile of KEYS keys that holds one which a row that sees only `least` keys does not see.
template <int KEYS>
__device__ __forceinline__ int first_unseen(const Sequence& s, int least) { return least < s.lk ? least / KEYS : 0x7FFFFFFF; }

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

}  // namespace fnn
