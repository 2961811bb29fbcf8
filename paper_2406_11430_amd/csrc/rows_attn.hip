// Plan and dispatch of l2kv_prompt_attn, l2kv_tree_attn and l2kv_paged_attn (kernels in rows_attn_kernels.hpp, one translation unit per row type).
#include "token_attn_kernels.hpp"

namespace l2kv {

extern template l2kv_status rows_attn_launch<BF16, 64, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 64, kRowsTree>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 64, kRowsPaged>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, kRowsTree>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 128, kRowsPaged>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, kRowsTree>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<BF16, 256, kRowsPaged>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, kRowsTree>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 64, kRowsPaged>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, kRowsTree>(const RowsArgs&, int, hipStream_t);
extern template l2kv_status rows_attn_launch<F32, 128, kRowsPaged>(const RowsArgs&, int, hipStream_t);

extern template l2kv_status token_attn_launch<BF16, 64>(const RowsArgs&, hipStream_t);
extern template l2kv_status token_attn_launch<BF16, 128>(const RowsArgs&, hipStream_t);
extern template l2kv_status token_attn_launch<BF16, 256>(const RowsArgs&, hipStream_t);
extern template l2kv_status token_attn_launch<F32, 64>(const RowsArgs&, hipStream_t);
extern template l2kv_status token_attn_launch<F32, 128>(const RowsArgs&, hipStream_t);

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

// One new token a sequence, as a rule: a workgroup for each compute unit and equal stretches, or, where the join of stretches costs more than
// it brings, a workgroup for each (token, KV head).  us, one for each item / 128 / 256 / 512 stretches (bf16, D 128, groups of 4):
//   1 sequence of 300 rows, 8 KV heads   8.7 /  9.9 / 10.0 / 10.0      4 of 16384                215 /  61 / 49 / 52
//   8 of 500                            11.6 / 13.8 / 12.3 / 13.1      1 of 131072              1690 / 116 / 89 / 97
//   64 of 700 (D 64, groups of 3)       18.2 / 32.8 / 22.9 / 20.6      64 of 500 to 4000         105 / 143 / 102 / 102
//   1 of 8192                            109 / 17.8 / 17.0 / 19.6      256 of 500 to 700         120 / 193 / 122 / 122
constexpr int kTokens = 3;                 // the shape of such launches
// The rows at which both take as long go by what a row costs a workgroup, its bytes and the heads it is for: bf16 D 128 with groups of 1 800, of 8
// 470, D 64 of 8 780, D 256 of 3 380, fp32 D 128 of 7 340; twice as many where there are
// items for all compute units.  How the tokens are spread over the sequences is not known here: a batch of 256 places of which one has 200 tokens over
// 8000 rows takes 807 us, that chunk alone 57; 16 of 64 sequences with 4 tokens each over 4000 rows 170 and 48.  1025 sequences, one of 131072 rows and the
// others of 100, 1860 us, 1024 of them in stretches 250.  Over 140 sizes what this chooses takes 1.4 % longer than the better of the two (512 and 1024 rows for all: 3.5 %).
static int64_t token_own_rows(int32_t G, int row_bytes, bool many) {
    const int64_t few = 900 * 9 * 256 / ((row_bytes < 192 ? 192 : row_bytes) * (8 + G));
    return many ? 2 * few : few;
}
static RowsPlan token_plan(int32_t n_seq, int32_t Hkv, int32_t G, int64_t total_q, int64_t max_kv, int32_t D, int row_bytes) {
    const int64_t units = device_compute_units(), items = total_q * Hkv;
    const int32_t keys = row_bytes == 128 ? TokenGeometry<BF16, 64>::kBlock : TokenGeometry<BF16, 128>::kBlock;
    RowsPlan p = {};
    p.shape = kTokens;
    p.tokens_per_block = 1;
    p.n_blocks = (int32_t)(total_q + n_seq);
    p.least_tiles = rows_item_tiles(false) + 1;
    // the search for a stretch's beginning goes over all sequences
    if (n_seq <= 1024 && max_kv > token_own_rows(G, row_bytes, items >= units)) {
        const int64_t most = items * (max_kv / keys + 2) / 2;
        p.workgroups = (int32_t)(most < units ? most : units);
    }
    p.partial_bytes = p.workgroups < 2 ? 0 : (size_t)p.workgroups * 2 * kTokenRows * rows_partial_floats(D) * sizeof(float);
    p.bytes = p.workgroups < 2 ? 0 : p.partial_bytes + (size_t)p.workgroups * sizeof(RowsJoin);
    return p;
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
RowsPlan rows_plan(int32_t n_seq, int32_t Hkv, int32_t G, int64_t total_q, int64_t max_kv, int32_t D, l2kv_dtype dt, RowsKind kind) {
    const bool tree = kind == kRowsTree;
    const int row_bytes = D * (dt == L2KV_F32 ? 4 : 2);
    const int64_t units = device_compute_units(), mean = (total_q + n_seq - 1) / n_seq;
    auto sizes = [&](int shape) { return row_bytes == 128 ? shape_sizes<128>(shape) : (row_bytes == 256 ? shape_sizes<256>(shape) : shape_sizes<512>(shape)); };
    auto items = [&](int shape) {
        const int64_t tokens = sizes(shape).rows / G;
        return (mean + tokens - 1) / tokens * n_seq * Hkv;
    };
    // the smallest block that takes the rows of a sequence, somewhat more than the average where there are several
    const int64_t rows = mean * G, room = n_seq == 1 ? rows : rows + rows / 4;
    // (a launch has fewer than 2^32 lanes)
    if (kind == kRowsPaged && total_q <= n_seq && (total_q + n_seq) * Hkv < (1 << 24)) return token_plan(n_seq, Hkv, G, total_q, max_kv, D, row_bytes);
    RowsPlan p;
    p.shape = kNarrowest;
    while (p.shape > 0 && sizes(p.shape).rows < room) --p.shape;
    const int64_t longest = max_kv + (tree ? mean : 0);            // keys of an item
    const double bytes = 2.0 * (double)max_kv * n_seq * Hkv * row_bytes;     // of K and V, at most
    bool stretches = false;
    int64_t per_unit = 1;
    // Chunks over rows in pages, whose lengths differ more than those of prompts.  Wide blocks where there is one for each compute unit (8 chunks of
    // 1 to 512 tokens over 1k to 8k rows, 265 us, 246 so), and stretches of them where each has eight tiles and more: the narrowest
    // would read K and V four times as often (2 chunks of 273 to 1062 tokens over 733 to 22124 rows, groups of 8, 749 and 463; 4 of D 256 over 14000
    // 1585 and 704).  fp32 products take so long that two of half the width share a unit (10 of 30 to 200 over 2000 311 and 254).
    const double tiles = (double)items(0) * ((double)longest - 0.5 * (double)(mean < longest ? mean : longest)) / sizes(0).keys / (double)units;
    const bool chunks = kind == kRowsPaged && p.shape == 0;
    if (p.shape == 0 && longest >= 2048 && items(0) >= (chunks && dt != L2KV_F32 ? units : 2 * units)) {
    } else if (p.shape < kNarrowest && items(1) >= 2 * units) {
        p.shape = 1;
    } else if (chunks && tiles >= 8.0 && n_seq <= 1024) {
        stretches = true;
        if (dt == L2KV_F32) p.shape = 1, per_unit = 2;
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
    // Two tiles of keys and what an item counts for by itself: 7 nodes over 2048 rows of 32 heads take 15.0 us, 17.0 with four tiles.  Chunks
    // over pages two in all: three fp32 ones of 1 to 77 tokens over 511 to 1533 rows 22.2 us, 18.6 so.
    p.least_tiles = kind == kRowsPaged ? 2 : rows_item_tiles(tree) + 2;
    p.workgroups = 0;
    if (stretches) {
        // (less four: their parts and joins then fit where those of wide ones do)
        const int64_t most = blocks * Hkv * (max_kv / s.keys + 2) / 2, wanted = per_unit == 1 ? units : per_unit * units - 4;
        p.workgroups = (int32_t)(most < wanted ? most : wanted);
    }
    p.partial_bytes = p.workgroups < 2 ? 0 : (size_t)p.workgroups * 2 * s.rows * rows_partial_floats(D) * sizeof(float);
    p.bytes = p.workgroups < 2 ? 0 : p.partial_bytes + (size_t)p.workgroups * sizeof(RowsJoin);
    return p;
}

l2kv_status rows_attn_dispatch(RowsArgs a, const RowsPlan& p, int32_t D, l2kv_dtype dt, RowsKind kind, hipStream_t stream) {
    a.tokens_per_block = p.tokens_per_block;
    a.n_blocks = p.n_blocks;
    a.workgroups = p.workgroups < 2 ? 0 : p.workgroups;
    a.least_tiles = p.least_tiles;
    a.once = p.once;
    a.joins = reinterpret_cast<RowsJoin*>(reinterpret_cast<char*>(a.partial) + p.partial_bytes);
    if (p.shape == kTokens) {
        if (dt == L2KV_F32) return D == 64 ? token_attn_launch<F32, 64>(a, stream) : token_attn_launch<F32, 128>(a, stream);
        return D == 64 ? token_attn_launch<BF16, 64>(a, stream) : (D == 128 ? token_attn_launch<BF16, 128>(a, stream) : token_attn_launch<BF16, 256>(a, stream));
    }
#define L2KV_ROWS(E, D_)                                                                 \
    return kind == kRowsTree    ? rows_attn_launch<E, D_, kRowsTree>(a, p.shape, stream)  \
           : kind == kRowsPaged ? rows_attn_launch<E, D_, kRowsPaged>(a, p.shape, stream) \
                                : rows_attn_launch<E, D_, kRowsPrompt>(a, p.shape, stream)
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
