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

constexpr int kNarrowest = 2;              // of the shapes; 0 is the widest
struct ShapeSizes { int32_t rows, keys; };
template <int kRowBytes, int kShape> static constexpr ShapeSizes sizes_of() {
    using S = RowsShape<kRowBytes, kShape>;
    return {S::kWR * kTile, S::kWK * S::kNK * kTile};
}
template <int kRowBytes> static ShapeSizes shape_sizes(int shape) {
    constexpr ShapeSizes all[3] = {sizes_of<kRowBytes, 0>(), sizes_of<kRowBytes, 1>(), sizes_of<kRowBytes, 2>()};
    return all[shape];
}

// Which block of rows a launch takes and whether a workgroup has an item for itself or an equal stretch of all of them.  Wide blocks read
// K and V least often; two workgroups of a narrow one share a compute unit, so that one computes while the other begins or ends an item, and
// there are more of them.  Measured (bf16, D 128, 8 KV heads of 4 query heads, us):
//                                       256 rows  128 rows  64 rows  stretches
//   1 prompt of 8192 tokens                  510       529      603        595    (most work: the widest block)
//   64 prompts of 64                        35.5      30.3     37.9       38.6    (two and more 128-row workgroups for each compute unit)
//   1 prompt of 512                         22.2      19.2     14.3       24.4    (few: the narrowest)
//   4 trees of 64 nodes over 16000 rows      389       328      244         92    (few and long: stretches, of the block that takes the rows)
//   1 tree of 64 nodes over 8192             204       172      106       29.9    (K and V are in the caches: stretches of the narrowest; the widest 36)
// Over 90 sizes of all row types what this chooses took 3 % longer than the best of the six (the best single one, stretches of 128 rows: 33 %).
// It knows the longest sequence and not the sum: a batch with one that is much longer than the others may get workgroups of their own where
// stretches are far better (64 trees of 8 nodes, one over 131072 rows and the others over 2000: 2006 us, stretches 197).
RowsPlan rows_plan(int32_t n_seq, int32_t Hkv, int32_t G, int64_t total_q, int64_t max_kv, int32_t D, l2kv_dtype dt, bool tree) {
    const int row_bytes = D * (dt == L2KV_F32 ? 4 : 2);
    const int64_t units = device_compute_units(), mean = (total_q + n_seq - 1) / n_seq;
    auto sizes = [&](int shape) { return row_bytes == 128 ? shape_sizes<128>(shape) : (row_bytes == 256 ? shape_sizes<256>(shape) : shape_sizes<512>(shape)); };
    auto items = [&](int shape) {
        const int64_t tokens = sizes(shape).rows / G;
        return (mean + tokens - 1) / tokens * n_seq * Hkv;
    };
    // the smallest block that takes the rows of a sequence, somewhat more than the average where there are several
    const int64_t rows = mean * G, room = n_seq == 1 ? rows : rows + rows / 4;
    RowsPlan p;
    p.shape = kNarrowest;
    while (p.shape > 0 && sizes(p.shape).rows < room) --p.shape;
    const int64_t longest = max_kv + (tree ? mean : 0);            // keys of an item
    const double bytes = 2.0 * (double)max_kv * n_seq * Hkv * row_bytes;     // of K and V, at most
    bool stretches = false;
    if (p.shape == 0 && longest >= 2048 && items(0) >= 2 * units) {
    } else if (p.shape < kNarrowest && items(1) >= 2 * units) {
        p.shape = 1;
    } else {
        // Of the narrowest block: the keys of the longest item, with something for two in a compute unit, against those of a stretch, with
        // 8 tiles' time for its beginning and the join.  Stretches of the widest block take 0.6 of the time for the same keys.
        const int64_t n = items(kNarrowest), tile = sizes(kNarrowest).keys;
        if (p.shape == 0 && bytes <= 40e6) p.shape = kNarrowest;           // a little more than the L2s hold
        const double own = (double)longest * (n > units ? 1.3 : 1.0);
        const double keys = (double)longest - (tree ? 0.0 : 0.5 * (double)(mean < longest ? mean : longest));
        const double even = (double)(8 * tile) + (double)n * keys / (double)units * (p.shape == 0 ? 0.6 : 1.0);
        stretches = n < 2 * units && own > even && n_seq <= 1024;      // the search for a stretch's beginning goes over all sequences
        if (!stretches) p.shape = kNarrowest;
    }
    // A tree's cached rows are read once (or by a few workgroups at about the same time), and more of them than the memory-side cache holds
    // are not there when the next call comes: 64 trees over 500 to 4000 rows 124 us, 135 through the caches; 64 over 1000 56 and 63.  16
    // over 1000 rows, which stay there from call to call, would take 28 us instead of 23.
    p.once = tree && bytes > 256e6;
    const ShapeSizes s = sizes(p.shape);
    p.tokens_per_block = s.rows / G;
    const int64_t blocks = total_q / p.tokens_per_block + n_seq;
    p.n_blocks = (int32_t)blocks;
    // Two tiles of keys and what an item counts for by itself: 7 nodes over 2048 rows of 32 heads take 15.0 us, 17.0 with four tiles.
    p.least_tiles = rows_item_tiles(tree) + 2;
    p.workgroups = 0;
    if (stretches) {
        const int64_t most = blocks * Hkv * (max_kv / s.keys + 2) / 2;
        p.workgroups = (int32_t)(most < units ? most : units);
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
    a.once = p.once;
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
