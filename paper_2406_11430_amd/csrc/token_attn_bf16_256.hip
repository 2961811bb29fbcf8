// Attention of single tokens over bf16 rows of 256 elements in pages.
#include "token_attn_kernels.hpp"

namespace l2kv {
template l2kv_status token_attn_launch<BF16, 256>(const RowsArgs&, hipStream_t);
}  // namespace l2kv
