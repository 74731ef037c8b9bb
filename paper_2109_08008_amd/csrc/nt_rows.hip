// How attention of many query rows is cut, by sizes that the host knows, and which data type's kernels take it.
#include <algorithm>

#include "nt_kernels.h"

namespace nt {

// The largest tile that still gives the CUs enough workgroups: a large one reads keys less often, a
// small one ends sooner (its waves share the keys of a tile, and join in LDS).  Measured, us, with
// tiles of 16 / 32 / 64 / 128 rows, one fp16 prompt: 8 heads, d_head 64, 100 tokens 7.1 / 7.1 / 7.8 / 7.8,
// 300 7.8 / 7.7 / 9.8 / 10.7, 1000 10.1 / 12.1 / 18.5 / 25, 3000 36 / 30 / 45 / 65; 16 heads, d_head 128,
// 300 10.5 / 10.3 / 12.4 / 13.6, 1000 32 / 23 / 24 / 32, 3000 170 / 109 / 64 / 88, 8000 - / 648 / 335 / 286.
// Sequences of less than 128 rows on average: waves of 16 rows and tiles of 32 keys pass over fewer keys of
// other sequences, and four to five workgroups instead of two or three are on a CU.  40000 rows of sequences
// of 1..n tokens, 16 heads, fp16, tiles of 128 / so, us: n = 8 d_head 32 61 / 60, 64 89 / 83, 128 154 / 138;
// 150 73 / 75, 107 / 104, 185 / 176; 400 99 / 101, 139 / 144, 243 / 244; 1500 178 / 177, 239 / 272, 416 / 462.
// fp32 with them at every length, from 64 channels on: n = 8 210 / 148, 418 / 258; 150 344 / 275, 691 / 503;
// 1500 1486 / 1410, 2886 / 2641.
// Where a workgroup of four waves fills a CU's LDS (keys of 256 bytes and more: 128 KB) and there are more of
// them than CUs, two waves: 16 heads of 128, fp16 and bf16, 300 tokens 9.2 / 8.6, 450 11.7 / 10.7, 30 sequences of
// 5..25 9.3 / 6.6; fp32 300 tokens 13.5 / 20.5, the 30 12.1 / 9.2.
void attn_prompt_plan(RowsAttnArgs* a) {
  auto groups = [&](int rows) { return (a->n_rows + (long long)rows - 1) / rows * a->n_heads; };
  a->tile = groups(128) >= 768 ? ROWS_128 : groups(64) >= 512 ? ROWS_64 : groups(32) >= 400 ? ROWS_32 : ROWS_16;
  const bool fine = a->tile == ROWS_128 && a->c.d_head >= 64 && (a->c.dt == DT::F32 || a->n_rows < 128ll * a->n_seqs);
  if (fine) a->tile = ROWS_64_FINE;
  const int rows = fine ? 64 : 16 << a->tile;
  a->rblocks = (int)((a->n_rows + (long long)rows - 1) / rows);
  if (a->tile == ROWS_16 && a->c.d_head * dt_bytes(a->c.dt) >= 256 && groups(16) > 256 &&
      (a->c.dt != DT::F32 || a->n_rows < 128ll * a->n_seqs))
    a->tile = ROWS_16_PAIR;
  a->parts = 1;
  a->chunk = 0;
}

// A key head's rows (new tokens times the heads that share it) in one tile if they fit: a second block of
// rows reads the keys again.  Measured, us, with 16 / 64 / 128 rows: 64 requests of 100..4000 bf16
// positions, 8 key heads of 128 channels (597 MB), 8 rows 110 / 108 / 126, 32 rows 176 / 109 / 117, 1..96 rows
// - / 157 / 121, 256 rows - / 245 / 200.
// Lengths are cut into parts of about chunk keys, a multiple of 512, alike within a sequence (its length
// decides how many): the longest into 512 / tasks parts, rounded down, which is up to two workgroups a CU
// (nothing is cut from 257 tasks on); with more than two blocks of rows, where matrix products bound it and a
// workgroup's own time is long, into 3200 / tasks, though no more than 8 unless 512 / tasks is.  That is
// twelve workgroups a CU by the largest sizes; ragged batches leave many of them empty or short, and their ends even
// out.  Measured, us, uncut / 4096 / 2048 / 1024
// keys: 12 requests of 1000..8000 positions and 200..500 new tokens, 4 key heads of four 228 / 174 / 164 /
// 184, forty 498 / 498 / 498 / 511; three such in 3 / 4 / 8 parts 68 / 61 / 51; six of 2000..16000 positions and
// 500..1000 new, 8 key heads of four, in 1 / 2 / 4 parts 576 / 492 / 507; one of 30000 positions, 512 new, in
// 8 / 12 / 18 / 25 parts 269 / 279 / 290 / 300; one of 131001 E4M3 positions, 64 new, uncut / 4096 / 2048 /
// 1024 keys 3150 / 119 / 90 / 106.  With parts of exactly chunk keys and a rest: 187 for the first's 174.
// 1600 / 3200 / 6400 for tasks of more than two blocks, fp16, us: 16 heads on 4, 12 requests of 1000..8000 and
// 200..500 new 174 / 165 / 185, 24 of them 364 / 340 / 352, 40 508 / 507 / 526; 32 heads on 8, 6 of 2000..16000 and
// 500..1000 new (bf16) 579 / 497 / 514, 16 of 1000..3000 and 100..300 new 149 / 160 / 172; 8 on 8, 30 of
// 500..4000 and 150..300 new 126 / 126 / 151; 8 on 2, 100 of 300..3000 and 70..300 new 167 / 166 / 199; one to three
// requests within 1.5 % of each other.
// One sequence much longer than the others is cut as they are: 64 requests, 8 key heads of 128 bf16 channels, 8
// new tokens each, all of 4000 positions 161, one of them of 131001 2365, that one alone 92.
// Never more than 32768 parts in all, however far max_len is above the lengths.
// 16 rows by two waves instead of four, for the same reason as prompts, and for many short sequences: 8 key heads
// of 128, up to 8 new tokens, 500 requests of 5..100 bf16 positions 88 / 53, of E4M3 44 / 29; 8 of 500..3000 29 / 25,
// 64 of 100..4000 110 / 108, one of 16000 20.2 / 21.3; of 64 channels 500 of 5..100 37 / 24, 300 of 100..300 33 / 27,
// 160 of 100..1000 37.8 / 38.1, 256 of 100..4000 174 / 182, 64 of 100..4000 54 / 66, 4 of 13..68 5.8 / 6.9.
// fp32 goes by its bytes too, four waves / two: 8 key heads of 128, 500 of 5..100 121 / 80, 300 of 100..300 140 / 114, 8 of
// 500..3000 56 / 48, 64 of 100..4000 274 / 280, 40 of 50..900 62 / 67; of 64 channels, 500 of 5..100 54 / 39, but 64 of
// 100..4000 125 / 200.
void attn_tree_plan(RowsAttnArgs* a) {
  const long long rows = (long long)std::max(a->max_new, 1) * a->group;
  a->tile = rows <= 16 ? ROWS_16 : rows <= 64 ? ROWS_64 : ROWS_128;
  a->rblocks = (int)((rows + (16ll << a->tile) - 1) >> (4 + a->tile));
  const long long tasks = std::max<long long>(1, (long long)a->n_seqs * a->c.n_kv_heads * a->rblocks);
  const long long want = std::max({1ll, 512 / tasks, a->rblocks > 2 ? std::min(8ll, 3200 / tasks) : 0ll});
  const long long least = std::max<long long>(1, a->max_len * tasks / 32768);
  long long chunk = std::max({(a->max_len + want - 1) / want, least, 512ll});
  a->chunk = (int)std::min<long long>((chunk + 511) / 512 * 512, 1 << 30);
  a->parts = (int)std::max<long long>(1, (a->max_len + (long long)a->chunk - 1) / a->chunk);
  const size_t key = a->c.d_head * (a->c.fp8 ? 1 : dt_bytes(a->c.dt));
  if (a->tile == ROWS_16 && (key >= 256 ? tasks * a->parts > 256 : tasks > 1024 && a->max_len < 1024)) a->tile = ROWS_16_PAIR;
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
