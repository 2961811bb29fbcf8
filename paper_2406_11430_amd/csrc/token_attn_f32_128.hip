// Attention of single tokens over fp32 rows of 128 elements in pages.
#include "token_attn_kernels.hpp"

namespace l2kv {
template l2kv_status token_attn_launch<F32, 128>(const RowsArgs&, hipStream_t);
}  // namespace l2kv
