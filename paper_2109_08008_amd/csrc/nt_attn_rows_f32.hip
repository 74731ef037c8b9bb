// Attention of many query rows, f32.
#include "nt_attn_rows.h"

namespace nt {
hipError_t attn_prompt_f32(const RowsAttnArgs& a, hipStream_t s) { return rows_head<float, float, false>(a, s); }
hipError_t attn_tree_f32(const RowsAttnArgs& a, hipStream_t s) {
  return rows_head<float, float, true>(a, s);
}
}  // namespace nt
