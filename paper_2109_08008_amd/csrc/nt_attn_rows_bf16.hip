// Attention of many query rows, bf16.
#include "nt_attn_rows.h"

namespace nt {
hipError_t attn_prompt_bf16(const RowsAttnArgs& a, hipStream_t s) { return rows_head<bf16, bf16, false>(a, s); }
hipError_t attn_tree_bf16(const RowsAttnArgs& a, hipStream_t s) {
  return rows_head<bf16, bf16, true>(a, s);
}
}  // namespace nt
