// Plan and dispatch of l2kv_prompt_attn and l2kv_tree_attn (kernels in rows_attn_kernels.hpp, one translation unit per row type).
#include "rows_attn_kernels.hpp"

namespace l2kv {

extern template l2kv_status rows_attn_launch<BF16, 64, false>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 64, true>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, false>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, true>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, false>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, true>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, false>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, true>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, false>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, true>(const RowsArgs&, int, hipStream_t);

struct ShapeSizes { int32_t rows, keys; };
template <int kRowBytes, int kShape> static constexpr ShapeSizes sizes_of() {
    using S = RowsShape<kRowBytes, kShape>;
    return {S::kWR * kTile, S::kWK * S::kNK * kTile};
}
template <int kRowBytes> static ShapeSizes shape_sizes(int shape) {
    constexpr ShapeSizes all[4] = {sizes_of<kRowBytes, 0>(), sizes_of<kRowBytes, 1>(), sizes_of<kRowBytes, 2>(), sizes_of<kRowBytes, 3>()};
    return all[shape];
}

RowsPlan rows_plan(int32_t n_seq, int32_t Hkv, int32_t G, int64_t total_q, int64_t max_kv, int32_t D, l2kv_dtype dt) {
    const int row_bytes = D * (dt == L2KV_F32 ? 4 : 2);
    auto sizes = [&](int shape) { return row_bytes == 128 ? shape_sizes<128>(shape) : (row_bytes == 256 ? shape_sizes<256>(shape) : shape_sizes<512>(shape)); };
    RowsPlan p;
    // the smallest block that takes the rows of a sequence, somewhat more than the average where there are several
    const int64_t rows = total_q * G / n_seq, room = n_seq == 1 ? rows : rows + rows / 4;
    p.shape = 3;
    while (p.shape > 0 && sizes(p.shape).rows < room) --p.shape;
    const ShapeSizes s = sizes(p.shape);
    p.tokens_per_block = s.rows / G;
    const int64_t blocks = total_q / p.tokens_per_block + n_seq;
    p.n_blocks = (int32_t)blocks;
    const int64_t items = blocks * Hkv, slots = device_compute_units();
    const int64_t tiles = max_kv / s.keys + 2;                     // of an item, at most (its nodes in one)
    // Many items, or items that are not worth cutting: a workgroup each.
    p.workgroups = 0;
    // Two tiles of keys and the one that an item counts for by itself: 7 nodes over 2048 rows of 32 heads take 18.3 us, 23.0 with
    // four tiles.
    p.least_tiles = 3;
    if (items < 4 * slots && tiles > 6 && n_seq <= 1024) {
        const int64_t most = items * tiles / (p.least_tiles - 1);
        p.workgroups = (int32_t)(most < slots ? most : slots);
    }
    p.partial_bytes = p.workgroups < 2 ? 0 : (size_t)p.workgroups * 2 * s.rows * rows_partial_floats(D) * sizeof(float);
    p.bytes = p.workgroups < 2 ? 0 : p.partial_bytes + (size_t)p.workgroups * sizeof(RowsJoin);
    return p;
}

l2kv_status rows_attn_dispatch(RowsArgs a, const RowsPlan& p, int32_t D, l2kv_dtype dt, bool tree, hipStream_t stream) {
    a.tokens_per_block = p.tokens_per_block;
    a.n_blocks = p.n_blocks;
    a.workgroups = p.workgroups < 2 ? 0 : p.workgroups;
    a.least_tiles = p.least_tiles;
    a.joins = reinterpret_cast<RowsJoin*>(reinterpret_cast<char*>(a.partial) + p.partial_bytes);
#define L2KV_ROWS(E, D_) return tree ? rows_attn_launch<E, D_, true>(a, p.shape, stream) : rows_attn_launch<E, D_, false>(a, p.shape, stream)
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
