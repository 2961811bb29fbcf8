// Kernels of l2kv_prompt_attn and l2kv_tree_attn: attention of many query rows, packed over sequences.
//
// The G query heads of a KV head are rows of one problem: row r of a block is token r / G, head r % G, so K and V are read once for all of
// them.  One workgroup takes a block of rows of one (sequence, KV head), over all its keys or, where rows are few, over a share of the
// tiles of keys; the shares are joined by a second kernel.
#pragma once

#include "attn_tiles.hpp"
#include "l2kv_host.hpp"
#include "rows_attn.hpp"

namespace l2kv {

// Block `id` of the launch: which tokens of which sequence, and the keys they see.
struct RowsBlock {
    int32_t seq;
    int64_t first_token;       // in Q and O
    int32_t tokens;            // 0: no such block
    int32_t first_in_seq;      // of its first token
    int32_t n_tokens;          // of the sequence
    int64_t first_row;         // of the sequence's cached rows in a plane
    int32_t n_rows;
    int32_t row_tiles, tiles;  // over cached rows, and over nodes as well
};

// Blocks are counted so that sequence s has ids from q_off[s] / tokens_per_block + s on: room for all its blocks, and which sequence an
// id belongs to is found among the offsets alone, 64 at a time.
template <bool kTree, int kTileKeys>
__device__ __forceinline__ RowsBlock rows_block(const RowsArgs& a, int32_t id, int lane) {
    RowsBlock b;
    int32_t lo = 0, count = a.n_seq;
    while (count > 1) {
        const int32_t step = (count + kWaveSize - 1) / kWaveSize;
        const int32_t mine = lo + lane * step;
        bool at_or_before = false;
        if (lane * step < count) {
            const int64_t off = a.q_off[mine];
            at_or_before = off / a.tokens_per_block + mine <= id;
        }
        const uint64_t found = __ballot(at_or_before);
        const int32_t last = found == 0 ? 0 : 63 - __builtin_clzll(found);
        const int32_t left = count - last * step;
        lo += last * step;
        count = left < step ? left : step;
    }
    b.seq = __builtin_amdgcn_readfirstlane(lo);
    const Range q = clamped_range(a.q_off, b.seq, a.total_q);
    const int64_t at = (id - (q.first / a.tokens_per_block + b.seq)) * a.tokens_per_block;
    b.tokens = 0;
    if (at < 0 || at >= q.count) return b;
    b.first_token = q.first + at;
    b.first_in_seq = (int32_t)at;
    b.n_tokens = (int32_t)q.count;
    b.tokens = (int32_t)(q.count - at < a.tokens_per_block ? q.count - at : a.tokens_per_block);
    const Range kv = clamped_range(a.kv_off, b.seq, a.total_rows);
    b.first_row = kv.first;
    int64_t rows = kv.count;
    if (a.kv_lens != nullptr) {
        const int64_t len = a.kv_lens[b.seq];
        rows = len < 0 ? 0 : (len < kv.count ? len : kv.count);
    }
    b.n_rows = (int32_t)rows;
    int64_t last = rows;                                       // cached rows that any of the tokens sees
    if constexpr (!kTree) {
        const int64_t limit = at + b.tokens + rows - q.count;
        last = limit < 0 ? 0 : limit;
    }
    b.row_tiles = (int32_t)((last + kTileKeys - 1) / kTileKeys);
    b.tiles = b.row_tiles + (kTree ? (int32_t)((q.count + kTileKeys - 1) / kTileKeys) : 0);
    return b;
}

__device__ __forceinline__ int32_t rows_shares(const RowsArgs& a, const RowsBlock& b) {
    const int32_t n = (b.tiles + a.tiles_per_share - 1) / a.tiles_per_share;
    return n < 1 ? 1 : (n < a.max_shares ? n : a.max_shares);
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

// kWR x kWK waves: kWR groups of 32 * kNQ rows each, the keys of a tile shared among kWK waves of a group.  A tile has kWK * kNK * 32 keys.
template <typename E, int D, int kNQ, int kWR, int kWK, int kNK, bool kTree>
__global__ __launch_bounds__(kWaveSize * kWR * kWK, kWR * kWK >= 8 ? 2 : 1)
void rows_attn_kernel(const RowsArgs a) {
    using R = AttnRow<E, D>;
    constexpr int kWaves = kWR * kWK, kTileKeys = kWK * kNK * kTile;
    constexpr int kHalf = kTileKeys * R::kBytes;               // bytes of a tile of K, and of one of V
    constexpr int kJoinFloats = (kWK - 1) * kWR * kNQ * (D / 2 + 2) * kWaveSize;
    static_assert(kJoinFloats * 4 <= 4 * kHalf, "the waves' results fit where the tiles were");
    __shared__ __attribute__((aligned(16))) char lds[4 * kHalf];

    const int lane = threadIdx.x % kWaveSize, half = lane / kTile;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWaveSize);
    const int wr = wave % kWR, wk = wave / kWR;
    const int32_t head = blockIdx.x % a.Hkv;
    const int32_t id = a.n_blocks - 1 - (int32_t)(blockIdx.x / a.Hkv);      // the last tokens of a sequence see most: they go first
    const RowsBlock b = rows_block<kTree, kTileKeys>(a, id, lane);
    if (b.tokens == 0) return;
    const int32_t shares = rows_shares(a, b), share = blockIdx.y;
    if (share >= shares) return;
    const int32_t first_tile = share * a.tiles_per_share;
    const int32_t end_tile = share + 1 == shares ? b.tiles : first_tile + a.tiles_per_share;

    // rows of this lane
    QueryTile<E, D> q[kNQ];
    int32_t token[kNQ], g[kNQ];
#pragma unroll
    for (int n = 0; n < kNQ; ++n) {
        const uint32_t row = (wr * kNQ + n) * kTile + lane % kTile;
        token[n] = (int32_t)(row / (uint32_t)a.G);
        g[n] = (int32_t)(row - (uint32_t)token[n] * (uint32_t)a.G);
        const int32_t t = token[n] < b.tokens ? token[n] : b.tokens - 1;
        load_query<E, D>(q[n], a.Q + ((b.first_token + t) * a.q_stride + (int64_t)(head * a.G + g[n]) * D) * E::kBytes, half);
    }
    const char* const K = a.K + ((int64_t)head * a.kv_head_stride + b.first_row * D) * E::kBytes;
    const char* const V = a.V + ((int64_t)head * a.kv_head_stride + b.first_row * D) * E::kBytes;
    const int64_t node_base = kTree ? ((int64_t)head * a.total_q + b.first_token - b.first_in_seq) * R::kBytes : 0;

    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_char_t*)lds;
    auto stage = [&](int32_t tile, int where) {
        const uint32_t to = lds_at + where;
        const bool nodes = kTree && tile >= b.row_tiles;
        const int64_t k0 = (int64_t)(nodes ? tile - b.row_tiles : tile) * kTileKeys;
        const char* const k = nodes ? a.Kt + node_base : K;
        const char* const v = nodes ? a.Vt + node_base : V;
        const int64_t rows = nodes ? b.n_tokens : b.n_rows;
        stage_rows<E, D, kTileKeys, kWaves, false>(k, k0, rows, to, wave, lane);
        stage_rows<E, D, kTileKeys, kWaves, true>(v, k0, rows, to + kHalf, wave, lane);
    };
    // Which of the 32 keys from k0 on a row sees.
    auto seen = [&](bool nodes, int64_t k0, int n) -> uint32_t {
        int64_t bound = (nodes ? b.n_tokens : b.n_rows) - k0;
        if constexpr (!kTree) bound = (int64_t)b.first_in_seq + token[n] + 1 + b.n_rows - b.n_tokens - k0;
        uint32_t bits = bound >= kTile ? ~0u : (bound <= 0 ? 0u : (1u << bound) - 1u);
        if constexpr (kTree) {
            if (nodes) {
                const int64_t word = k0 / kTile;
                const int32_t t = token[n] < b.tokens ? token[n] : b.tokens - 1;
                bits &= word < a.mask_words ? a.mask[(b.first_token + t) * a.mask_words + word] : 0u;
            }
        }
        return bits;
    };

    // Tiles of which every row sees every key come first: no masks, and nothing that only masks need.
    const int64_t open_keys = kTree ? b.n_rows : (int64_t)b.first_in_seq + 1 + b.n_rows - b.n_tokens;
    int32_t open_end = open_keys < kTileKeys ? 0 : (int32_t)(open_keys / kTileKeys);
    open_end = open_end < end_tile ? open_end : end_tile;

    const TileAddress<E, D> at(lane);
    RowState<E, D, kNQ> st;
    st.clear();
    auto open_tile = [&](const char* here) {
#pragma unroll
        for (int j = 0; j < kNK; ++j) {
            const char* const k = here + (wk * kNK + j) * kTile * R::kBytes;
            f32x16_t s[kNQ];
            Weights<E> p[kNQ];
            scores<E, D, kNQ>(k, at, q, s);
            softmax_step<E, D, kNQ>(st, s, p, a.scale);
            weighted_values<E, D, kNQ>(k + kHalf, at, p, st.o);
        }
    };
    auto masked_tile = [&](const char* here, int32_t tile) {
        const bool nodes = kTree && tile >= b.row_tiles;
        const int64_t k0 = (int64_t)(nodes ? tile - b.row_tiles : tile) * kTileKeys;
#pragma unroll 1
        for (int j = 0; j < kNK; ++j) {
            const int sub = (wk * kNK + j) * kTile;
            const char* const k = here + sub * R::kBytes;
            uint32_t bits[kNQ];
            bool any = false;
#pragma unroll
            for (int n = 0; n < kNQ; ++n) {
                bits[n] = seen(nodes, k0 + sub, n);
                any |= bits[n] != 0;
            }
            if (__ballot(any) == 0) continue;
            f32x16_t s[kNQ];
            Weights<E> p[kNQ];
            scores<E, D, kNQ>(k, at, q, s);
#pragma unroll
            for (int n = 0; n < kNQ; ++n) {
                const uint32_t mine = bits[n] >> (4 * half);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[n][i] = (mine >> (8 * (i / 4) + i % 4)) & 1 ? s[n][i] : -__builtin_inff();
            }
            softmax_step<E, D, kNQ>(st, s, p, a.scale);
            if (values_not_finite<E, D>(k + kHalf, lane)) {
#pragma unroll
                for (int n = 0; n < kNQ; ++n) weighted_values_seen<E, D>(k + kHalf, at, p[n], bits[n], st.o[n], lane);
            } else {
                weighted_values<E, D, kNQ>(k + kHalf, at, p, st.o);
            }
        }
    };
    int32_t tile = first_tile;
    if (tile < end_tile) stage(tile, 0);
    int here = 0;
    for (; tile < open_end; ++tile) {
        wait_loads_to_lds();
        __syncthreads();                                       // the tile is there, and nobody reads the other one any more
        if (tile + 1 < end_tile) stage(tile + 1, here ^ (2 * kHalf));
        open_tile(lds + here);
        here ^= 2 * kHalf;
    }
    for (; tile < end_tile; ++tile) {
        wait_loads_to_lds();
        __syncthreads();
        if (tile + 1 < end_tile) stage(tile + 1, here ^ (2 * kHalf));
        masked_tile(lds + here, tile);
        here ^= 2 * kHalf;
    }

    if constexpr (kWK > 1) {
        // the waves of a group join what they have of the same rows
        __syncthreads();
        float* const all = reinterpret_cast<float*>(lds);
        constexpr int kWaveFloats = kNQ * (D / 2 + 2) * kWaveSize;
        if (wk > 0) {
            float* const mine = all + ((wk - 1) * kWR + wr) * kWaveFloats + lane;
#pragma unroll
            for (int n = 0; n < kNQ; ++n) {
                float* const to = mine + n * (D / 2 + 2) * kWaveSize;
                to[0] = st.m[n];
                to[kWaveSize] = st.l[n];
#pragma unroll
                for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[(2 + d * 16 + i) * kWaveSize] = st.o[n][d][i];
            }
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll 1
        for (int other = 1; other < kWK; ++other) {
#pragma unroll
            for (int n = 0; n < kNQ; ++n) {
                const float* const from = all + ((other - 1) * kWR + wr) * kWaveFloats + n * (D / 2 + 2) * kWaveSize + lane;
                const float mo = from[0], m = fmaxf(st.m[n], mo);
                const float f = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(st.m[n] - m);
                const float fo = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(mo - m);
                st.m[n] = m;
                st.l[n] = st.l[n] * f + from[kWaveSize] * fo;
#pragma unroll
                for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) st.o[n][d][i] = st.o[n][d][i] * f + from[(2 + d * 16 + i) * kWaveSize] * fo;
            }
        }
    }

#pragma unroll
    for (int n = 0; n < kNQ; ++n) {
        const float l = sum_of_halves(st.l[n]);
        if (token[n] >= b.tokens) continue;
        if (shares == 1) {
            const float f = l == 0.f ? 0.f : 1.f / l;          // no key: zeros
            char* const to = a.O + (((b.first_token + token[n]) * (int64_t)(a.Hkv * a.G) + head * a.G + g[n]) * D) * E::kBytes;
#pragma unroll
            for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v[4] = {st.o[n][d][4 * i] * f, st.o[n][d][4 * i + 1] * f, st.o[n][d][4 * i + 2] * f, st.o[n][d][4 * i + 3] * f};
                    store_four<E>(to + (d * kTile + 8 * i + 4 * half) * E::kBytes, v);
                }
        } else {
            const int64_t row = (((int64_t)id * a.Hkv + head) * a.max_shares + share) * a.block_rows + token[n] * a.G + g[n];
            float* const to = a.partial + row * (D + 2);
            // rows of D + 2 floats: eight bytes are what they are aligned to
#pragma unroll
            for (int d = 0; d < D / kTile; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        *reinterpret_cast<float2*>(to + d * kTile + 8 * i + 4 * half + 2 * j) =
                            make_float2(st.o[n][d][4 * i + 2 * j], st.o[n][d][4 * i + 2 * j + 1]);
            if (half == 0) *reinterpret_cast<float2*>(to + D) = make_float2(st.m[n], l);
        }
    }
}

// One wave per query row: the shares of the row's block, each relative to its own maximum, in the order of the keys.
template <typename E, int D, int kTileKeys, bool kTree>
__global__ __launch_bounds__(256)
void rows_join_kernel(const RowsArgs a) {
    constexpr int kPer = D / kWaveSize;                        // elements of a lane: consecutive
    const int lane = threadIdx.x % kWaveSize;
    const int32_t head = blockIdx.x % a.Hkv, id = blockIdx.x / a.Hkv;
    const RowsBlock b = rows_block<kTree, kTileKeys>(a, id, lane);
    if (b.tokens == 0) return;
    const int32_t shares = rows_shares(a, b);
    if (shares == 1) return;
    for (int32_t row = blockIdx.y * 4 + threadIdx.x / kWaveSize; row < b.tokens * a.G; row += gridDim.y * 4) {
        const float* const first = a.partial + ((((int64_t)id * a.Hkv + head) * a.max_shares) * a.block_rows + row) * (D + 2);
        const int64_t step = (int64_t)a.block_rows * (D + 2);
        float m = -__builtin_inff();
        for (int32_t s = 0; s < shares; ++s) m = fmaxf(m, first[s * step + D]);
        float l = 0.f, o[kPer] = {};
        for (int32_t s = 0; s < shares; ++s) {
            const float ms = first[s * step + D], f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(ms - m);
            if (ms == -__builtin_inff()) continue;             // a share without a key that the row sees
            l += first[s * step + D + 1] * f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) o[i] += first[s * step + lane * kPer + i] * f;
        }
        const float f = l == 0.f ? 0.f : 1.f / l;
        const int32_t token = row / a.G, g = row % a.G;
        char* const at = a.O + (((b.first_token + token) * (int64_t)(a.Hkv * a.G) + head * a.G + g) * D + lane * kPer) * E::kBytes;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if constexpr (E::kBytes == 4) reinterpret_cast<float*>(at)[i] = o[i] * f;
            else reinterpret_cast<__bf16*>(at)[i] = (__bf16)(o[i] * f);
        }
    }
}

// The two shapes of workgroup a row type has.  wide: many rows, the keys of a tile seen by all waves; narrow: 32 rows, the keys of a
// tile divided among the waves.
template <typename E, int D> struct RowsShapes {
    static constexpr bool kLong = AttnRow<E, D>::kBytes == 512;
    static constexpr int kWideNQ = 1, kWideWR = kLong ? 4 : 8, kWideNK = kLong ? 1 : 2;
    static constexpr int kNarrowWK = kLong ? 2 : 4;
    static constexpr int kWideRows = kWideNQ * kWideWR * kTile, kWideKeys = kWideNK * kTile, kNarrowKeys = kNarrowWK * kTile;
};

template <typename E, int D, bool kTree>
l2kv_status rows_attn_launch(const RowsArgs& a, bool wide, hipStream_t stream) {
    using S = RowsShapes<E, D>;
    const dim3 grid((unsigned)(a.n_blocks * a.Hkv), (unsigned)a.max_shares);
    if (wide)
        hipLaunchKernelGGL((rows_attn_kernel<E, D, S::kWideNQ, S::kWideWR, 1, S::kWideNK, kTree>), grid, dim3(S::kWideWR * kWaveSize), 0, stream, a);
    else
        hipLaunchKernelGGL((rows_attn_kernel<E, D, 1, 1, S::kNarrowWK, 1, kTree>), grid, dim3(S::kNarrowWK * kWaveSize), 0, stream, a);
    if (a.max_shares > 1) {
        if (l2kv_status st = launch_status(); st != L2KV_OK) return st;
        const dim3 join((unsigned)(a.n_blocks * a.Hkv), (unsigned)((a.block_rows + 3) / 4));
        if (wide) hipLaunchKernelGGL((rows_join_kernel<E, D, S::kWideKeys, kTree>), join, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((rows_join_kernel<E, D, S::kNarrowKeys, kTree>), join, dim3(256), 0, stream, a);
    }
    return launch_status();
}

}  // namespace l2kv
