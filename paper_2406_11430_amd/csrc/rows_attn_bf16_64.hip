// Prompt and tree attention over bf16 rows of 64 elements: one translation unit per row type, so that they compile in parallel.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<BF16, 64, false>(const RowsArgs&, int, hipStream_t);
template l2kv_status rows_attn_launch<BF16, 64, true>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
