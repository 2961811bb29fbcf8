// Prompt and tree attention over bf16 rows of 128 elements: one translation unit per row type, so that they compile in parallel.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<BF16, 128, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
template l2kv_status rows_attn_launch<BF16, 128, kRowsTree>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
