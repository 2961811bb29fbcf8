// Attention over bf16 rows of 256 elements in pages.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<BF16, 256, kRowsPaged>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
