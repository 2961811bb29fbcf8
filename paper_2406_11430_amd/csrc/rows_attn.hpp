// Plan and arguments of the attention of many query rows (prompts, drafted trees): plain C++, no device code.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace l2kv {

struct RowsArgs {
    const char *Q, *K, *V, *Kt, *Vt;
    char* O;
    float* partial;
    const int64_t *q_off, *kv_off;
    const int32_t* kv_lens;
    const uint32_t* mask;
    int64_t total_q, total_rows, kv_head_stride, q_stride;      // strides in elements
    int32_t n_seq, Hkv, G, mask_words;
    int32_t block_rows, tokens_per_block, n_blocks, tiles_per_share, max_shares;
    float scale;                                                // softmax scale times log2(e)
};

// How a launch is cut: blocks of query rows, and shares of the tiles of keys.
struct RowsPlan {
    bool wide;
    int32_t block_rows, tokens_per_block, n_blocks, tiles_per_share, max_shares;
    size_t partial_bytes;
};

}  // namespace l2kv
