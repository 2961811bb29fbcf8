// Prompt and tree attention over f32 rows of 128 elements: one translation unit per row type, so that they compile in parallel.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<F32, 128, kRowsPrompt>(const RowsArgs&, int, hipStream_t);
template l2kv_status rows_attn_launch<F32, 128, kRowsTree>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
