// Attention over bf16 rows of 128 elements in pages.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<BF16, 128, kRowsPaged>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
