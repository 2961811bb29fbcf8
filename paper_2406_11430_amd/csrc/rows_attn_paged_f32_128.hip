// Attention over fp32 rows of 128 elements in pages.
#include "rows_attn_kernels.hpp"

namespace l2kv {
template l2kv_status rows_attn_launch<F32, 128, kRowsPaged>(const RowsArgs&, int, hipStream_t);
}  // namespace l2kv
