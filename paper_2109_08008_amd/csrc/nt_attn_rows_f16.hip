// Attention of many query rows, f16.
#include "nt_attn_rows.h"

namespace nt {
hipError_t attn_prompt_f16(const RowsAttnArgs& a, hipStream_t s) { return rows_head<f16, f16, false>(a, s); }
hipError_t attn_tree_f16(const RowsAttnArgs& a, hipStream_t s) {
  return a.c.fp8 ? rows_head<f16, uint8_t, true>(a, s) : rows_head<f16, f16, true>(a, s);
}
}  // namespace nt
