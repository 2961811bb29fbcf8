// Plan and dispatch of l2kv_prompt_attn and l2kv_tree_attn (kernels in rows_attn_kernels.hpp, one translation unit per row type).
#include "rows_attn_kernels.hpp"

namespace l2kv {

extern template l2kv_status rows_attn_launch<BF16, 64, false>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 64, true>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, false>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, true>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, false>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, true>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, false>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, true>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, false>(const RowsArgs&, bool, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, true>(const RowsArgs&, bool, hipStream_t);

template <typename E, int D> static void shapes(bool wide, int32_t* rows, int32_t* keys) {
    using S = RowsShapes<E, D>;
    *rows = wide ? S::kWideRows : kTile;
    *keys = wide ? S::kWideKeys : S::kNarrowKeys;
}

RowsPlan rows_plan(int32_t n_seq, int32_t Hkv, int32_t G, int64_t total_q, int64_t max_kv, int32_t D, l2kv_dtype dt) {
    RowsPlan p;
    // rows of an average sequence; a workgroup of the wide shape reads the keys once for all its rows
    const int64_t mean_rows = total_q * G / n_seq;
    p.wide = mean_rows > kTile;
    int32_t keys;
    if (dt == L2KV_F32) {
        if (D == 64) shapes<F32, 64>(p.wide, &p.block_rows, &keys);
        else shapes<F32, 128>(p.wide, &p.block_rows, &keys);
    } else if (D == 64) {
        shapes<BF16, 64>(p.wide, &p.block_rows, &keys);
    } else if (D == 128) {
        shapes<BF16, 128>(p.wide, &p.block_rows, &keys);
    } else {
        shapes<BF16, 256>(p.wide, &p.block_rows, &keys);
    }
    p.tokens_per_block = p.block_rows / G;
    const int64_t blocks = total_q / p.tokens_per_block + n_seq;
    p.n_blocks = (int32_t)blocks;                               // at most 2^32 (checked by the caller): total_q, n_seq < 2^31
    const int64_t tiles = (max_kv + keys - 1) / keys;
    const int64_t work = blocks * Hkv, want = 2 * device_compute_units();
    int64_t shares = work >= want / 2 ? 1 : want / work;
    const int64_t least = 4;                                    // tiles of a share
    if (shares > tiles / least) shares = tiles / least < 1 ? 1 : tiles / least;
    p.tiles_per_share = (int32_t)((tiles + shares - 1) / shares);
    if (p.tiles_per_share < 1) p.tiles_per_share = 1;
    p.max_shares = (int32_t)((tiles + p.tiles_per_share - 1) / p.tiles_per_share);
    if (p.max_shares < 1) p.max_shares = 1;
    p.partial_bytes = p.max_shares == 1 ? 0 : (size_t)blocks * Hkv * p.max_shares * p.block_rows * (D + 2) * sizeof(float);
    return p;
}

l2kv_status rows_attn_dispatch(RowsArgs a, const RowsPlan& p, int32_t D, l2kv_dtype dt, bool tree, hipStream_t stream) {
    a.block_rows = p.block_rows;
    a.tokens_per_block = p.tokens_per_block;
    a.n_blocks = p.n_blocks;
    a.tiles_per_share = p.tiles_per_share;
    a.max_shares = p.max_shares;
#define L2KV_ROWS(E, D_) return tree ? rows_attn_launch<E, D_, true>(a, p.wide, stream) : rows_attn_launch<E, D_, false>(a, p.wide, stream)
    if (dt == L2KV_F32) {
        if (D == 64) L2KV_ROWS(F32, 64);
        L2KV_ROWS(F32, 128);
    }
    if (D == 64) L2KV_ROWS(BF16, 64);
    if (D == 128) L2KV_ROWS(BF16, 128);
    L2KV_ROWS(BF16, 256);
#undef L2KV_ROWS
}

}  // namespace l2kv
