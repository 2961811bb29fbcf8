// Kernels of l2kv_prompt_attn and l2kv_tree_attn: attention of many query rows, packed over sequences.
//
// The G query heads of a KV head are rows of one problem: row r of a block is token r / G, head r % G, so K and V are read once for all of
// them.  An item is one block of rows of one (sequence, KV head) over all keys that it sees.  A launch either has one workgroup per item
// (many items: those that run at a time read the same keys), or a fixed number of workgroups that take equal stretches of all items'
// keys laid end to end, whatever the lengths are; what a stretch has of an item that others have parts of goes to memory, and a second
// kernel joins the parts.
#pragma once

#include "attn_tiles.hpp"
#include "l2kv_host.hpp"
#include "rows_attn.hpp"

namespace l2kv {

struct RowsSeq {
    int64_t q_first, row_first;        // first token in Q and O, first cached row in a plane
    int32_t n_q, n_rows, blocks;
};

// Quotient of numbers that are not negative; most have 32 bits, where a division is a tenth of the instructions.
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d) {
    if (((n | d) >> 32) == 0) return (uint32_t)n / (uint32_t)d;
    return (int64_t)((uint64_t)n / (uint64_t)d);
}

__device__ __forceinline__ RowsSeq rows_seq(const RowsArgs& a, int32_t s) {
    const Range q = clamped_range(a.q_off, s, a.total_q), kv = clamped_range(a.kv_off, s, a.total_rows);
    int64_t rows = kv.count < a.most_rows ? kv.count : a.most_rows;
    if (a.kv_lens != nullptr) {
        const int64_t len = a.kv_lens[s];
        rows = len < 0 ? 0 : (len < rows ? len : rows);
    }
    return RowsSeq{q.first, kv.first, (int32_t)q.count, (int32_t)rows, (int32_t)(((uint32_t)q.count + (uint32_t)a.tokens_per_block - 1) / (uint32_t)a.tokens_per_block)};
}
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ RowsSeq uniform(const RowsSeq& q) {
    return RowsSeq{uniform(q.q_first), uniform(q.row_first), __builtin_amdgcn_readfirstlane(q.n_q), __builtin_amdgcn_readfirstlane(q.n_rows),
                   __builtin_amdgcn_readfirstlane(q.blocks)};
}

// Lengths of items, in keys.  A block of a prompt sees the rows up to its last token's limit; a block of a tree all cached rows and all
// nodes, in whole tiles each.  An item counts for some tiles more than it has: what its beginning and its end take, and so that none is empty.
template <bool kTree, int kTileKeys> struct RowsLength {
    static constexpr int kExtra = rows_item_tiles(kTree) * kTileKeys;
    static __device__ __forceinline__ int64_t keys(const RowsArgs& a, const RowsSeq& q, int64_t block) {
        if constexpr (kTree) {
            return (((int64_t)q.n_rows + kTileKeys - 1) / kTileKeys + ((int64_t)q.n_q + kTileKeys - 1) / kTileKeys) * kTileKeys;
        } else {
            const int64_t end = (block + 1) * a.tokens_per_block, limit = (end < q.n_q ? end : q.n_q) + q.n_rows - q.n_q;
            return limit < 0 ? 0 : limit;
        }
    }
    // of the blocks before `block`, together
    static __device__ __forceinline__ int64_t before(const RowsArgs& a, const RowsSeq& q, int64_t block) {
        if constexpr (kTree) {
            return block * (kExtra + keys(a, q, 0));
        } else {
            const int64_t step = a.tokens_per_block, more = (int64_t)q.n_rows - q.n_q;
            const int64_t none = more >= 0 ? 0 : (uint32_t)-more / (uint32_t)step;            // blocks that see nothing
            int64_t sum = block * kExtra;
            if (block > none) sum += step * (block * (block + 1) - none * (none + 1)) / 2 + more * (block - none);
            if (block == q.blocks && block > none) sum -= block * step - q.n_q;
            return sum;
        }
    }
};

// An item and a place in it.
struct RowsItem {
    RowsSeq q;
    int32_t seq, head, block;
    int64_t start, at;                 // of the item in the line of all items, of the place in the item
};

// Inclusive prefix sum of a wave's numbers below 2^56, by two of 32 bits.
__device__ __forceinline__ int64_t wave_prefix(int64_t v) {
    return ((int64_t)wave_inclusive_sum((uint32_t)(v >> 24)) << 24) + wave_inclusive_sum((uint32_t)v & 0xffffffu);
}
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}

__device__ __forceinline__ RowsSeq of_lane(const RowsSeq& q, int lane) {
    return RowsSeq{of_lane(q.q_first, lane), of_lane(q.row_first, lane), __builtin_amdgcn_readlane(q.n_q, lane),
                   __builtin_amdgcn_readlane(q.n_rows, lane), __builtin_amdgcn_readlane(q.blocks, lane)};
}

// Keys of a stretch where all items count for `total`: the same for every workgroup, but at least some tiles, so that short problems are
// not cut to pieces.
template <int kTileKeys> __device__ __forceinline__ int64_t rows_stretch(const RowsArgs& a, int64_t total) {
    const int64_t even = quotient(total + a.workgroups - 1, a.workgroups);
    return even < a.least_tiles * kTileKeys ? a.least_tiles * kTileKeys : even;
}

// The stretch of this workgroup, [begin, end), and the item that it begins in; false if there is none.  A lane for each sequence, 64 at
// a time.
template <bool kTree, int kTileKeys>
__device__ __forceinline__ bool rows_stretch_item(const RowsArgs& a, RowsItem& it, int64_t& stretch, int64_t& end, int lane) {
    using L = RowsLength<kTree, kTileKeys>;
    RowsSeq q = {};
    int64_t mine = 0, upto = 0, total = 0;                     // of the lane's sequence, of those up to it, of all
    int32_t s0 = 0;
    auto look = [&] {
        q = RowsSeq{};
        if (s0 + lane < a.n_seq) q = rows_seq(a, s0 + lane);
        mine = a.Hkv * L::before(a, q, q.blocks);
        upto = wave_prefix(mine);
    };
    for (; s0 < a.n_seq; s0 += kWaveSize) {
        look();
        total += of_lane(upto, kWaveSize - 1);
    }
    stretch = rows_stretch<kTileKeys>(a, total);
    const int64_t begin = blockIdx.x * stretch;
    if (begin >= total) return false;
    end = begin + stretch < total ? begin + stretch : total;
    int64_t base = 0;                                          // of the sequences before s0
    if (a.n_seq > kWaveSize) s0 = 0, look();
    else s0 = 0;
    uint64_t behind;
    while ((behind = __ballot(base + upto > begin)) == 0) {    // ends at the last sequences, where it is total > begin
        base += of_lane(upto, kWaveSize - 1);
        s0 += kWaveSize;
        look();
    }
    const int which = __builtin_ctzll(behind);
    it.seq = s0 + which;
    it.q = of_lane(q, which);
    int64_t rest = begin - base - of_lane(upto - mine, which);
    const int64_t head_keys = L::before(a, it.q, it.q.blocks);
    it.head = (int32_t)quotient(rest, head_keys);
    rest -= it.head * head_keys;
    // the last block that begins at or before the place, 64 candidates a step
    int32_t lo = 0, count = it.q.blocks;
    while (count > 1) {
        const int32_t step = (count + kWaveSize - 1) / kWaveSize;
        const uint64_t found = __ballot((int64_t)lane * step < count && L::before(a, it.q, lo + (int64_t)lane * step) <= rest);
        const int32_t last = found == 0 ? 0 : 63 - __builtin_clzll(found);
        lo += last * step;
        count = count - last * step < step ? count - last * step : step;
    }
    it.block = __builtin_amdgcn_readfirstlane(lo);
    it.head = __builtin_amdgcn_readfirstlane(it.head);
    it.at = uniform(rest - L::before(a, it.q, it.block));
    it.start = uniform(begin - it.at);
    return true;
}

// The item of a workgroup of its own; the last tokens of a sequence see most, so they go first.  Blocks are numbered over the sequences
// without gaps, found by a sum over the offsets, a part of the sequences for each lane (more than 64 in two rounds).  (Workgroups
// without a block behind those that have one do no harm; between them they did, as the hardware deals workgroups out in turn: a batch
// whose every other number was empty ran on half of the device.)
constexpr int32_t kSummedSequences = kWaveSize * kWaveSize;
template <bool kTree, int kTileKeys>
__device__ __forceinline__ bool rows_own_item(const RowsArgs& a, RowsItem& it, int lane) {
    it.head = (int32_t)(blockIdx.x % (uint32_t)a.Hkv);
    it.start = it.at = 0;
    const int32_t number = (int32_t)(blockIdx.x / (uint32_t)a.Hkv);
    int32_t block = 0, lo = 0, count = a.n_seq;
    if (count > kSummedSequences) {
        // Very many, where a sum would be longer than the work: sequence s has the numbers from q_off[s] / tokens_per_block + s on, room for
        // all its blocks, and a search among 64 candidates a round finds the last that begins at or before a number.
        const int32_t id = a.n_blocks - 1 - number;
        while (count > 1) {
            const int32_t step = (count + kWaveSize - 1) / kWaveSize;
            const int64_t mine = lo + (int64_t)lane * step;
            bool at_or_before = false;
            if ((int64_t)lane * step < count) {
                const int64_t first = clamped_range(a.q_off, mine, a.total_q).first;
                at_or_before = (int64_t)((uint32_t)first / (uint32_t)a.tokens_per_block) + mine <= id;
            }
            const uint64_t found = __ballot(at_or_before);
            const int32_t last = found == 0 ? 0 : 63 - __builtin_clzll(found);
            lo += last * step;
            count = count - last * step < step ? count - last * step : step;
        }
        it.seq = __builtin_amdgcn_readfirstlane(lo);
        it.q = uniform(rows_seq(a, it.seq));
        block = id - (int32_t)((uint32_t)it.q.q_first / (uint32_t)a.tokens_per_block) - it.seq;
        it.block = block;
        return block >= 0 && block < it.q.blocks;
    }
    for (bool all = true;; all = false) {
        const int32_t step = (count + kWaveSize - 1) / kWaveSize;
        RowsSeq q = {};
        uint32_t mine = 0;
        if (step <= 1) {
            if (lane < count) q = rows_seq(a, lo + lane);
            mine = (uint32_t)q.blocks;
        } else {
            for (int32_t n = 0; n < step; ++n) {
                const int32_t s = lane * step + n;
                if (s < count) mine += ((uint32_t)clamped_range(a.q_off, lo + s, a.total_q).count + (uint32_t)a.tokens_per_block - 1) / (uint32_t)a.tokens_per_block;
            }
        }
        const uint32_t upto = wave_inclusive_sum(mine);
        if (all) block = __builtin_amdgcn_readlane((int)upto, kWaveSize - 1) - 1 - number;
        const uint64_t behind = __ballot((int32_t)upto > block);
        if (block < 0 || behind == 0) return false;
        const int which = __builtin_ctzll(behind);
        block -= __builtin_amdgcn_readlane((int)(upto - mine), which);
        if (step <= 1) {
            it.seq = lo + which;
            it.q = of_lane(q, which);
            it.block = block;
            return block >= 0 && block < it.q.blocks;
        }
        lo += which * step;
        count = count - which * step < step ? count - which * step : step;
    }
}

template <typename E> __device__ __forceinline__ void store_four(char* at, const float (&v)[4]) {
    if constexpr (E::kBytes == 4) {
        *reinterpret_cast<f32x4_t*>(at) = f32x4_t{v[0], v[1], v[2], v[3]};
    } else {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        const f32x2_t a = {v[0], v[1]}, b = {v[2], v[3]};
        *reinterpret_cast<u32x2_t*>(at) = u32x2_t{__builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2_t)),
                                                  __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2_t))};
    }
}

// kWR x kWK waves: kWR groups of 32 rows each, the keys of a tile shared among kWK waves of a group.  A tile has kWK * kNK * 32 keys;
// kStages of them have room in LDS, all but one on their way while that one is worked on.  kOnce: cached rows are not read again soon.
//
// Prompts are bound by the two units that do not overlap enough: of a tile of 256 rows and 64 keys (bf16, D 128; 1.9 us) the matrix unit is
// busy for 55 % of the cycles, exponentials, maxima and roundings for 46, and the clock falls as they are busier.  A prompt of 32768 tokens (32 query heads, 8 KV heads) takes 7.7 to 8.4 ms
// from card to card, 1.05 to 1.14 PFLOP/s of the 1.37 that a large matrix product reaches.  Batches of trees are bound by memory:
// 64 of 1 to 32 nodes over 500 to 4000 rows 119 to 121 us, 5.1 TB/s (a large copy: 4.80).
template <typename E, int D, int kWR, int kWK, int kNK, int kStages, bool kTree, bool kOnce>
__global__ __launch_bounds__(kWaveSize * kWR * kWK, 2)
void rows_attn_kernel(const RowsArgs a) {
    using R = AttnRow<E, D>;
    constexpr int kWaves = kWR * kWK, kTileKeys = kWK * kNK * kTile, kBlockRows = kWR * kTile;
    constexpr int kHalf = kTileKeys * R::kBytes;               // bytes of a tile of K, and of one of V
    constexpr int kLoads = 2 * kHalf / 1024 / kWaves;          // of a wave, for a tile
    using L = RowsLength<kTree, kTileKeys>;
    // Sized at the launch: the compiler takes a workgroup that fills the LDS for one wave per SIMD whatever else it is told, and spreads its
    // registers over both files, with copies between them in every tile.
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_char_t*)lds;

    const int lane = threadIdx.x % kWaveSize;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int wr = wave % kWR, wk = wave / kWR;
    const TileAddress<E, D> place(lane);

    RowsItem it;
    int64_t end, stretch = 0;                                  // of this workgroup's stretch
    if (a.workgroups == 0) {
        if (!rows_own_item<kTree, kTileKeys>(a, it, lane)) return;
        end = L::kExtra + L::keys(a, it.q, it.block);
    } else {
        if (threadIdx.x == 0) a.joins[blockIdx.x].parts = 0;   // until an item begins here that ends elsewhere
        if (!rows_stretch_item<kTree, kTileKeys>(a, it, stretch, end, lane)) return;
    }
    for (int slot = 0;; slot = 1) {                            // one item after the other
        int row = wr * kTile + lane % kTile, half = lane / kTile;
        asm volatile("" : "+v"(row), "+v"(half));              // what follows from them is not held from item to item: registers
        const int64_t keys = L::keys(a, it.q, it.block), item_end = it.start + L::kExtra + keys;
        const int64_t here_end = (end < item_end ? end : item_end) - it.start;
        // tile t stands at kExtra + t * kTileKeys of its item
        const int32_t first_tile = it.at <= L::kExtra ? 0 : (int32_t)((it.at - L::kExtra + kTileKeys - 1) / kTileKeys);
        const int32_t end_tile = here_end <= L::kExtra ? 0 : (int32_t)((here_end - L::kExtra + kTileKeys - 1) / kTileKeys);
        const bool whole = it.at == 0 && item_end <= end;
        const int32_t first_in_seq = it.block * a.tokens_per_block;
        const int64_t first_token = it.q.q_first + first_in_seq;
        const int32_t tokens = it.q.n_q - first_in_seq < a.tokens_per_block ? it.q.n_q - first_in_seq : a.tokens_per_block;
        const int32_t row_tiles = kTree ? (int32_t)(((int64_t)it.q.n_rows + kTileKeys - 1) / kTileKeys) : 0x7fffffff;
        const bool live = wr * kTile < tokens * a.G;           // this wave has rows

        // of this lane; rows behind the last are copies of it and not stored
        const int32_t t = row / a.G < tokens ? row / a.G : tokens - 1;
        QueryTile<E, D> q;
        auto load_queries = [&](int32_t r) {
            const int32_t own = r / a.G < tokens ? r / a.G : tokens - 1, g = r % a.G;
            load_query<E, D>(q, a.Q + ((first_token + own) * a.q_stride + (int64_t)(it.head * a.G + g) * D) * E::kBytes, half);
        };
        load_queries(row);
        const char* const K = a.K + ((int64_t)it.head * a.kv_head_stride + it.q.row_first * D) * E::kBytes;
        const char* const V = a.V + ((int64_t)it.head * a.kv_head_stride + it.q.row_first * D) * E::kBytes;
        const int64_t node_base = kTree ? ((int64_t)it.head * a.total_q + it.q.q_first) * R::kBytes : 0;

        auto stage = [&](int32_t tile, int where) {
            const bool nodes = kTree && tile >= row_tiles;
            const int64_t k0 = (int64_t)(nodes ? tile - row_tiles : tile) * kTileKeys;
            const int64_t rows = nodes ? it.q.n_q : it.q.n_rows;
            stage_rows<E, D, kTileKeys, kWaves, false, kOnce>(nodes ? a.Kt + node_base : K, k0, rows, lds_at + where, wave, lane);
            stage_rows<E, D, kTileKeys, kWaves, true, kOnce>(nodes ? a.Vt + node_base : V, k0, rows, lds_at + where + kHalf, wave, lane);
        };
        // Which of the 32 keys from k0 on the lane's row sees.
        auto seen = [&](bool nodes, int64_t k0) -> uint32_t {
            int64_t bound = (nodes ? it.q.n_q : it.q.n_rows) - k0;
            if constexpr (!kTree) bound = (int64_t)first_in_seq + t + 1 + it.q.n_rows - it.q.n_q - k0;
            uint32_t bits = bound >= kTile ? ~0u : (bound <= 0 ? 0u : (1u << bound) - 1u);
            if constexpr (kTree) {
                if (nodes) {
                    const int64_t word = k0 / kTile;
                    bits &= word < a.mask_words ? a.mask[(first_token + t) * a.mask_words + word] : 0u;
                }
            }
            return bits;
        };
        // Tiles of which every row sees every key come first: no masks, and nothing that only masks need.
        const int64_t open_keys = kTree ? it.q.n_rows : (int64_t)first_in_seq + 1 + it.q.n_rows - it.q.n_q;
        int32_t open_end = open_keys < kTileKeys ? 0 : (int32_t)(open_keys / kTileKeys);
        open_end = open_end < end_tile ? open_end : end_tile;

        RowState<E, D> st;
        st.clear();
        TileAddress<E, D> at = place;
        auto open_tile = [&](const char* here) {
#pragma unroll
            for (int j = 0; j < kNK; ++j) {
                const char* const k = here + (wk * kNK + j) * kTile * R::kBytes;
                if constexpr (R::kBytes == 512) at.forget();
                f32x16_t s;
                Weights<E> p;
                scores<E, D>(k, at, q, s);
                if constexpr (R::kBytes == 512) {
                    softmax_step<E, D>(st, s, p, a.scale);
                    weighted_values<E, D>(k + kHalf, at, p, st.o);
                } else {
                    ValueTile<E, D> values;
                    load_values<E, D>(k + kHalf, at, values);
                    softmax_step<E, D>(st, s, p, a.scale);
                    weighted_values<E, D>(values, p, st.o);
                }
            }
        };
        auto masked_tile = [&](const char* here, int32_t tile) {
            const bool nodes = kTree && tile >= row_tiles;
            const int64_t k0 = (int64_t)(nodes ? tile - row_tiles : tile) * kTileKeys;
#pragma unroll 1
            for (int j = 0; j < kNK; ++j) {
                const int sub = (wk * kNK + j) * kTile;
                const char* const k = here + sub * R::kBytes;
                const uint32_t bits = seen(nodes, k0 + sub);
                if (__ballot(bits != 0) == 0) continue;
                TileAddress<E, D> at = place;
                if constexpr (R::kBytes == 512) {
                    // queries are read again and places worked out again instead of held: registers, for the few tiles with masks
                    int32_t again = row;
                    asm volatile("" : "+v"(again));
                    load_queries(again);
                    at.forget();
                }
                f32x16_t s;
                Weights<E> p;
                scores<E, D>(k, at, q, s);
                const uint32_t mine = bits >> (4 * half);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = (mine >> (8 * (i / 4) + i % 4)) & 1 ? s[i] : -__builtin_inff();
                softmax_step<E, D>(st, s, p, a.scale);
                ValueTile<E, D> values;
                constexpr bool kLook = R::kBytes == 128 || (R::kBytes == 256 && E::kBytes == 4);
                if constexpr (kLook) load_values<E, D>(k + kHalf, at, values);
                // Long rows have no registers for two ways of adding the same products: they take the careful one always.
                bool careful = R::kBytes == 512;
                if constexpr (kLook) careful = values_not_finite<E, D>(values);
                else if constexpr (R::kBytes < 512) careful = values_not_finite<E, D>(k + kHalf, lane);
                if (careful) {
                    if (finite_values<E, D>(k + kHalf, at, p, st.o)) other_values<E, D>(k + kHalf, at, p, bits, st.o, lane);
                } else {
                    if constexpr (!kLook) load_values<E, D>(k + kHalf, at, values);
                    weighted_values<E, D>(values, p, st.o);
                }
            }
        };
        int32_t tile = first_tile, staged = first_tile;
        int here = 0, there = 0;                               // where the tile is, and where the next one goes
        auto after = [&](int slot_at) { return slot_at + 2 * kHalf < kStages * 2 * kHalf ? slot_at + 2 * kHalf : 0; };
        auto stage_next = [&] {
            if (staged < end_tile) {
                stage(staged++, there);
                there = after(there);
            }
        };
        // The tile is there for all waves, and the one before it is not read any more: its place takes the next.
        auto next_tile = [&] {
            wait_loads_to_lds<kLoads, kStages - 2>(staged - tile - 1);
            __syncthreads();
            stage_next();
        };
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) stage_next();
        for (; tile < open_end; ++tile) {
            next_tile();
            if (live) open_tile(lds + here);
            here = after(here);
        }
        for (; tile < end_tile; ++tile) {
            next_tile();
            if (live) masked_tile(lds + here, tile);
            here = after(here);
        }

        if constexpr (kWK > 1) {
            // the waves of a group join what they have of the same rows
            __syncthreads();
            float* const all = reinterpret_cast<float*>(lds);
            constexpr int kWaveFloats = (D / 2 + 2) * kWaveSize;
            if (wk > 0) {
                float* const to = all + ((wk - 1) * kWR + wr) * kWaveFloats + lane;
                to[0] = st.m;
                to[kWaveSize] = st.l;
#pragma unroll
                for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[(2 + d * 16 + i) * kWaveSize] = st.o[d][i];
            }
            __syncthreads();
            if (wk == 0) {
#pragma unroll 1
                for (int other = 1; other < kWK; ++other) {
                    const float* const from = all + ((other - 1) * kWR + wr) * kWaveFloats + lane;
                    const float mo = from[0], m = fmaxf(st.m, mo);
                    const float f = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
                    const float fo = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(mo - m);
                    st.m = m;
                    st.l = st.l * f + from[kWaveSize] * fo;
#pragma unroll
                    for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) st.o[d][i] = st.o[d][i] * f + from[(2 + d * 16 + i) * kWaveSize] * fo;
                }
            }
        }

        const float l = sum_of_halves(st.l);
        int32_t out_row = row, out_half = half;
        asm volatile("" : "+v"(out_row), "+v"(out_half));      // nor from its beginning to its end
        const int32_t token = out_row / a.G;
        if (wk == 0 && token < tokens) {
            if (whole) {
                const float f = l == 0.f ? 0.f : 1.f / l;      // no key: zeros
                char* const to = a.O + (((first_token + token) * (int64_t)(a.Hkv * a.G) + it.head * a.G + out_row - token * a.G) * D) * E::kBytes;
#pragma unroll
                for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x16_t& o = st.o[d];
                        const float v[4] = {o[4 * i] * f, o[4 * i + 1] * f, o[4 * i + 2] * f, o[4 * i + 3] * f};
                        store_four<E>(to + (d * kTile + 8 * i + 4 * out_half) * E::kBytes, v);
                    }
            } else {
                float* const to = a.partial + (((int64_t)blockIdx.x * 2 + slot) * kBlockRows + out_row) * rows_partial_floats(D);
#pragma unroll
                for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x16_t& o = st.o[d];
                        *reinterpret_cast<f32x4_t*>(to + d * kTile + 8 * i + 4 * out_half) = f32x4_t{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
                    }
                if (out_half == 0) *reinterpret_cast<float2*>(to + D) = make_float2(st.m, l);
            }
        }
        if (item_end >= end) {
            if (it.at == 0 && item_end > end && threadIdx.x == 0)
                a.joins[blockIdx.x] = RowsJoin{first_token * (a.Hkv * a.G) + it.head * a.G, (int32_t)quotient(item_end - 1, stretch) - (int32_t)blockIdx.x + 1,
                                               tokens * a.G, slot, 0};
            return;
        }
        // the next item, from its beginning
        it.start = item_end;
        it.at = 0;
        if (++it.block >= it.q.blocks) {
            it.block = 0;
            if (++it.head == a.Hkv) {
                it.head = 0;
                do it.q = uniform(rows_seq(a, ++it.seq));      // one with tokens follows: the stretch does not end here
                while (it.q.blocks == 0 && it.seq + 1 < a.n_seq);
            }
        }
        __syncthreads();                                       // before the first tile goes where this item's were
    }
}

// Joins what several workgroups have of an item, for the workgroup in whose stretch it begins (blockIdx.y; rows come first in the launch,
// so that those of one item are spread over all dies).  Four elements of a row a lane; the parts of a row in the order of the keys,
// eight on their way at a time.
constexpr int kJoinThreads = 256;
template <typename E, int D, int kBlockRows>
__global__ __launch_bounds__(kJoinThreads)
void rows_join_kernel(const RowsArgs a) {
    constexpr int64_t kPart = (int64_t)kBlockRows * rows_partial_floats(D);
    constexpr int kLanes = D / 4, kAhead = 8;
    const RowsJoin join = a.joins[blockIdx.y];
    const int32_t row = blockIdx.x * (kJoinThreads / kLanes) + threadIdx.x / kLanes, parts = join.parts;
    if (row >= join.rows || parts == 0) return;
    const int c = threadIdx.x % kLanes;
    const float* const mine = a.partial + ((int64_t)blockIdx.y * 2 * kBlockRows + row) * rows_partial_floats(D);
    float m = -__builtin_inff(), l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int32_t p = 0; p < parts; p += kAhead) {
        f32x4_t x[kAhead];
        float2 ml[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u < parts) {
                // two parts for each workgroup; the first may be its second, where another item ends before it
                const float* const from = mine + (p + u == 0 ? join.slot : 2 * (p + u)) * kPart;
                x[u] = *reinterpret_cast<const f32x4_t*>(from + 4 * c);
                ml[u] = *reinterpret_cast<const float2*>(from + D);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (p + u < parts) {
                // A maximum of minus infinity says that no score of the part is above it, not that the row sees no key there: NaN of such a
                // part (scores that are all NaN, values that are not finite under a weight of zero) is in its sums, and goes on.
                const float top = fmaxf(m, ml[u].x);
                const float old = top == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - top);
                const float f = top == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(ml[u].x - top);
                m = top;
                l = l * old + ml[u].y * f;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = o[i] * old + x[u][i] * f;
            }
        }
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const int32_t token = row / a.G, g = row - token * a.G;
    const float v[4] = {o[0] * f, o[1] * f, o[2] * f, o[3] * f};
    store_four<E>(a.O + ((join.first_row + (int64_t)token * (a.Hkv * a.G) + g) * D + 4 * c) * E::kBytes, v);
}

// The shapes of workgroup a row type has: rows of a block (32 * kWR) and keys of a tile (32 * kWK * kNK).  The widest fills a compute unit
// (8 waves of up to 256 registers), of the others two share one; the narrowest has two waves for the same rows, so that short items of
// few rows use all four SIMDs.  Two tiles in LDS, one read and one on its way: 3 and 4 of them measured slower (256 rows: a prompt of 32768
// tokens 8.5 ms against 7.9; 128 rows, trees of a batch: 200 us against 152), 32 keys a tile for 128 rows as well (582 against 570).
// Measured against the widest: 16 waves' worth of rows in 4 waves of 64 (half the LDS reads, one wave a SIMD) 8.45 ms, halves of a workgroup
// in opposite phases 8.04, raised priority for products 8.44.  Rows of 512 bytes have 32 keys a tile: registers and LDS.
template <int kRowBytes, int kShape> struct RowsShape;
template <int kRowBytes> struct RowsShape<kRowBytes, 0> { static constexpr int kWR = 8, kWK = 1, kNK = 2, kStages = 2; };
template <int kRowBytes> struct RowsShape<kRowBytes, 1> { static constexpr int kWR = 4, kWK = 1, kNK = 2, kStages = 2; };
template <int kRowBytes> struct RowsShape<kRowBytes, 2> { static constexpr int kWR = 2, kWK = 2, kNK = 1, kStages = 2; };
template <> struct RowsShape<512, 0> { static constexpr int kWR = 8, kWK = 1, kNK = 1, kStages = 4; };
template <> struct RowsShape<512, 1> { static constexpr int kWR = 4, kWK = 1, kNK = 1, kStages = 2; };
template <> struct RowsShape<512, 2> { static constexpr int kWR = 2, kWK = 2, kNK = 1, kStages = 2; };

template <typename E, int D, int kShape, bool kTree>
l2kv_status rows_attn_launch_shape(const RowsArgs& a, hipStream_t stream) {
    using S = RowsShape<AttnRow<E, D>::kBytes, kShape>;
    constexpr int kRows = S::kWR * kTile;
    constexpr unsigned kLds = S::kStages * 2 * S::kWK * S::kNK * kTile * AttnRow<E, D>::kBytes;
    static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
    static_assert((S::kWK - 1) * S::kWR * (D / 2 + 2) * kWaveSize * sizeof(float) <= kLds, "room for what the waves of a group join");
    const dim3 grid((unsigned)(a.workgroups == 0 ? a.n_blocks * a.Hkv : a.workgroups));
    const dim3 block(S::kWR * S::kWK * kWaveSize);
    if (kTree && a.once)
        hipLaunchKernelGGL((rows_attn_kernel<E, D, S::kWR, S::kWK, S::kNK, S::kStages, kTree, kTree>), grid, block, kLds, stream, a);
    else
        hipLaunchKernelGGL((rows_attn_kernel<E, D, S::kWR, S::kWK, S::kNK, S::kStages, kTree, false>), grid, block, kLds, stream, a);
    if (a.workgroups > 1) {
        if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        // (of a few tokens not all rows of a block: 7 nodes take 2.8 us, the 64 rows of a block 5.8)
        const int64_t rows = a.total_q * a.G < kRows ? a.total_q * a.G : kRows;
        const dim3 join_grid((unsigned)((rows * (D / 4) + kJoinThreads - 1) / kJoinThreads), (unsigned)a.workgroups);
        hipLaunchKernelGGL((rows_join_kernel<E, D, kRows>), join_grid, dim3(kJoinThreads), 0, stream, a);
    }
    return launch_status();
}

template <typename E, int D, bool kTree>
l2kv_status rows_attn_launch(const RowsArgs& a, int shape, hipStream_t stream) {
    switch (shape) {
        case 0: return rows_attn_launch_shape<E, D, 0, kTree>(a, stream);
        case 1: return rows_attn_launch_shape<E, D, 1, kTree>(a, stream);
        default: return rows_attn_launch_shape<E, D, 2, kTree>(a, stream);
    }
}

}  // namespace l2kv
