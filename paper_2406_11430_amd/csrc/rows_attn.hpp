// Plan and arguments of the attention of many query rows (prompts, drafted trees): plain C++, no device code.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace l2kv {

// An item that several workgroups have parts of, as the one in whose stretch it begins leaves it for the join.
struct RowsJoin {
    int64_t first_row;         // of O: (token, query head) of its first row
    int32_t parts, rows, slot, unused;
};

struct RowsArgs {
    const char *Q, *K, *V, *Kt, *Vt;
    char* O;
    float* partial;
    RowsJoin* joins;
    const int64_t *q_off, *kv_off;
    const int32_t* kv_lens;
    const uint32_t* mask;
    int64_t total_q, total_rows, kv_head_stride, q_stride;      // strides in elements
    int64_t most_rows;                                          // of a sequence: where the next head begins
    int32_t n_seq, Hkv, G, mask_words;
    int32_t tokens_per_block, n_blocks, workgroups, least_tiles;
    float scale;                                                // softmax scale times log2(e)
    bool once;                                                  // trees: cached rows pass the caches by
};

// What an item counts for besides its keys, in tiles of them: of a prompt one for its beginning and its end and one because its
// diagonal may lie in a tile more (fp32, odd lengths: 34.9 us, 35.7 with one tile), of a tree one (7 fp32 nodes over 4000 rows: 35.5 us, 38.9 with two).
constexpr int rows_item_tiles(bool tree) { return tree ? 1 : 2; }

// How a launch is cut: the shape of its workgroups, which takes blocks of so many tokens, and the number of workgroups that take equal
// stretches of all keys (0: one workgroup per block and KV head).
struct RowsPlan {
    int shape;
    int32_t tokens_per_block, n_blocks, workgroups, least_tiles;
    bool once;
    size_t partial_bytes, bytes;       // of the parts, and of the joins behind them as well
};

// One row of what a workgroup has of an item: D sums, the maximum that they are relative to, the sum of weights; 16-byte aligned.
constexpr int rows_partial_floats(int D) { return D + 4; }

}  // namespace l2kv
