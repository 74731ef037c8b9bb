// How attention of many query rows is cut, and which data type's kernels take it.
#include <algorithm>

#include "nt_kernels.h"

namespace nt {

void attn_prompt_plan(RowsAttnArgs* a) {
  a->tile = ROWS_128;
  a->rblocks = (int)(((long long)a->n_rows + 127) / 128);
  a->parts = 1;
  a->chunk = 0;
}

void attn_tree_plan(RowsAttnArgs* a) {
  const long long rows = (long long)std::max(a->max_new, 1) * a->group;
  a->tile = rows <= 16 ? ROWS_16 : rows <= 32 ? ROWS_32 : ROWS_128;
  const int bm = a->tile == ROWS_16 ? 16 : a->tile == ROWS_32 ? 32 : 128;
  a->rblocks = (int)((rows + bm - 1) / bm);
  const long long tasks = std::max<long long>(1, (long long)a->n_seqs * a->c.n_kv_heads * a->rblocks);
  long long parts = std::max<long long>(1, 1024 / tasks);
  long long chunk = (a->max_len + parts - 1) / parts;
  chunk = std::max<long long>(512, (chunk + 511) / 512 * 512);
  a->chunk = (int)std::min<long long>(chunk, 1 << 30);
  a->parts = (int)std::max<long long>(1, (a->max_len + (long long)a->chunk - 1) / a->chunk);
}

hipError_t attn_prompt(const RowsAttnArgs& a, hipStream_t s) {
  if (a.n_rows <= 0) return hipSuccess;
  switch (a.c.dt) {
    case DT::F32: return attn_prompt_f32(a, s);
    case DT::F16: return attn_prompt_f16(a, s);
    case DT::BF16: return attn_prompt_bf16(a, s);
  }
  return hipErrorInvalidValue;
}

hipError_t attn_tree(const RowsAttnArgs& a, hipStream_t s) {
  if (a.n_rows <= 0 || a.n_seqs <= 0) return hipSuccess;
  if (a.c.fp8 && a.c.dt != DT::F16) return hipErrorInvalidValue;
  switch (a.c.dt) {
    case DT::F32: return attn_tree_f32(a, s);
    case DT::F16: return attn_tree_f16(a, s);
    case DT::BF16: return attn_tree_bf16(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nt
