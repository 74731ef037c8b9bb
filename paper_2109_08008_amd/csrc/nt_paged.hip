// A paged key/value cache: appending new tokens' keys and values, and attention of one new
// token a sequence over it.
//
// The cache is a pool of pages [n_pages][kv head][slot][d_head] for the keys and one for the
// values, and a table that names each sequence's pages in order: position p of sequence b is
// slot p % page_len of page table[b][p / page_len].  A head's share of a page is contiguous
// (page_len * d_head elements), so a wave that reads one head's keys in order reads whole
// lines.  page_len is a power of two of at least 16: 16 keys, one MFMA block, are always on
// one page, and the page is the same in every lane.
#include <algorithm>
#include <type_traits>

#include "nt_gemm_common.h"

namespace nt {
namespace {
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// E4M3 codes of four values, e4m3_rne's: the hardware's conversion rounds to nearest even and keeps
// subnormals, but does not saturate (a NaN passes the comparisons and gives 0x7F).
__device__ __forceinline__ unsigned e4m3_4(float a, float b, float c, float d) {
  auto sat = [](float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; };
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), lo, true);
}

// ---- append ----------------------------------------------------------------------------
// A move of rows: HBM and the launch bound it.  A wave takes a.wave_rows rows in turns of `across`
// at a time, 1 << piece_shift lanes (16-byte pieces) a row, U turns' loads of keys and values under
// way together, and each lane finds one of the rows' places meanwhile: its sequence (off is sorted) by
// 64 probes that the lanes share and a search between two of them.  Measured, us (GB/s): 19.8k rows of
// 16 x 64 fp16 values to E4M3 26.5 (4680; a copy reaches 4940), of 8 x 128 bf16 26.3 (6140); 73k rows
// of 4 x 32 bf16 14.9 (5050; one row a wave took 36); 96 rows of 8 x 64 3.9.  Eight turns for rows of
// more than one turn, four for the others (the second case with four 30; 200k rows of 32 fp32 values,
// with eight 23.5, four 19.7).
template <typename T, bool F8, int U>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  constexpr int VN = Vec<T>::N;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int first = (blockIdx.x * 4 + wave) * a.wave_rows;
  if (first >= a.rows) return;
  const int width = a.c.n_kv_heads * a.c.d_head, pieces = width / VN;
  const int lanes = 1 << a.piece_shift, across = kWave >> a.piece_shift;
  const int r = lane >> a.piece_shift, p = lane & (lanes - 1);
  const int chunks = (pieces + lanes - 1) >> a.piece_shift;   // turns a row
  const int turns = a.wave_rows / across * chunks;
  const T* k = static_cast<const T*>(a.k);
  const T* v = static_cast<const T*>(a.v);
  struct Turn { int t, row, piece; };   // of the lane, rows counted from `first`
  auto next = [&](Turn& n) {
    ++n.t;
    n.piece += lanes;
    if (n.piece - p >= chunks * lanes) {
      n.piece = p;
      n.row += across;
    }
  };
  u32x4 kq[U], vq[U];
  Turn ahead{0, r, p};
  auto load = [&] {                     // (past the rows' or the row's end: the last again, not stored)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (ahead.t >= turns) break;
      const size_t at = (size_t)min(first + ahead.row, a.rows - 1) * a.ld + min(ahead.piece, pieces - 1) * VN;
      kq[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + at));
      vq[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v + at));
      next(ahead);
    }
  };
  load();
  // lane l: the cell of row first + l, -1 if it has none
  long long cell = -1;
  {
    const int row = first + min(lane, a.wave_rows - 1);
    int b = row, behind = 1;            // the sequence's last new row is its last position
    if (a.off) {
      // entries off[1 .. n_seqs] at or below the row: lo of them
      const int step = (a.n_seqs + kWave - 1) / kWave;
      const int probe = a.off[min((lane + 1) * step, a.n_seqs)];
      int lo = 0;
#pragma unroll
      for (int s = kWave / 2; s; s >>= 1)
        if (__shfl(probe, lo + s - 1, kWave) <= row) lo += s;
      if (lo == kWave - 1 && __shfl(probe, kWave - 1, kWave) <= row) lo = kWave;
      int hi = min((lo + 1) * step - 1, a.n_seqs);
      lo = min(lo * step, a.n_seqs);
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.off[mid] <= row) lo = mid;
        else hi = mid - 1;
      }
      b = lo;
      behind = b < a.n_seqs && a.off[b] <= row ? a.off[b + 1] - row : 0;   // 0: not a row of any sequence
    }
    if (lane < a.wave_rows && row < a.rows && behind > 0) {
      const int pos = max(a.lens[b], 0) - behind;
      if (pos >= 0 && (pos >> a.c.page_shift) < a.c.max_pages) {
        const int page = a.c.table[(size_t)b * a.c.max_pages + (pos >> a.c.page_shift)];
        if ((unsigned)page < (unsigned)a.c.n_pages)
          cell = (((long long)page * a.c.n_kv_heads) << a.c.page_shift) + (pos & ((1 << a.c.page_shift) - 1));
      }
    }
  }
  const int dsh = 31 - __builtin_clz(a.c.d_head);   // 32, 64 or 128
  for (Turn now{0, r, p};;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (now.t >= turns) break;
      const long long at0 = __shfl(cell, now.row, kWave);
      const int e = now.piece * VN, h = e >> dsh, x = e & (a.c.d_head - 1);
      const bool has = now.piece < pieces && at0 >= 0;
      next(now);
      if (!has) continue;
      const size_t at = ((size_t)at0 + ((size_t)h << a.c.page_shift)) * a.c.d_head + x;
      if constexpr (F8) {
        static_assert(VN == 8, "E4M3 caches take 16-bit rows");
        auto codes = [](u32x4 q) {
          const half8 e = __builtin_bit_cast(half8, q);
          return u32x2{e4m3_4((float)e[0], (float)e[1], (float)e[2], (float)e[3]),
                       e4m3_4((float)e[4], (float)e[5], (float)e[6], (float)e[7])};
        };
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.k) + at) = codes(kq[u]);
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.c.v) + at) = codes(vq[u]);
      } else {
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.k) + at) = kq[u];
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.v) + at) = vq[u];
      }
    }
    if (now.t >= turns) break;
    load();
  }
}

// ---- attention -------------------------------------------------------------------------
// out_h = sum_j e^{s_j - m} V_j / sum_j e^{s_j - m},  s_j = scale q_h . K_j.
//
// A stream over the cache, bound by HBM once there are enough keys in flight: the key and
// value of a position are used once by each of the heads that share them.  Those heads (up
// to 16 a block) are the rows of the matrix products, which cost the same for one head as
// for 16 and stay far below the stream's time.  A wave takes a tile of keys at a time
// (tile_keys), the next tile's keys and values on their way to registers meanwhile; both go
// through its own LDS, since whole lines come in row by row and the products want them by
// lane.  Scores are transposed, S^T = K.Q^T, so that lane l holds head l % 16's scores of
// four keys of each 16, which are the ones it supplies to P.V; the values are read key-major
// (16-bit and E4M3: the transposing LDS reads).  The softmax's running maximum and sum are
// fp32, in powers of two; with 16-bit values P enters P.V as two terms of that type (two_terms),
// a matrix product each, so that the output's own rounding is what 16 bits cost.  (With P rounded
// once the output was off by 1.2 times that, and where the values cancel by any factor of it.)
// For fp16 P is 2^14 times as large there (p_scale), as far up as e^{s - m} <= 1 goes: what is lost
// of a probability is at most 2^-39 of the largest one.  (As they are, probabilities below 2^-14
// would lose bits and those below 2^-25 would leave the product while the sum keeps them: one key
// 17.4 above 131000 equal ones gave those no weight instead of 0.0036.)  The factor goes with the
// division by the sum.
//
// SW waves share a task (sequence, key head, block of 16 heads, part of the length): they
// take its tiles in turn and join in LDS at the end.  A length is split into parts of
// `chunk` keys over workgroups when there are few tasks; the parts' (max, sum, unnormalised
// output) go to the workspace and paged_join_kernel merges them.
//
// Measured, us (GB/s of keys and values): 2160 x 16 heads of up to 231 bf16 keys, d_head 64, 160
// (6420), of up to 64 65 (4570), of up to 48 58 (3950); 16 x 8 of 2048..32768 fp16, d_head 128, four
// query heads each, 171 (6070), the join 4.6 of it; one sequence, 4 x 131001 E4M3, d_head 128, 28 (4790),
// the join 4.5; 64 x 8 of up to 48 fp16 keys 4.6; 32 x 8 of 500..8000 fp32 keys, d_head 64, 119 (5070),
// d_head 128, 207 (5810).  Plain reads reach 6200, non-temporal ones 7000.  (Keys straight to the products'
// registers, 16 bytes of a row a lane: 231 and 198 for the first two.)
typedef short short4v __attribute__((ext_vector_type(4)));
// Four 16-bit values of one column, rows r..r+3 of an LDS tile: each lane of 16 names the
// 8 bytes at row r + lane / 4, columns 4 (lane % 4).., and receives column lane.
__device__ __forceinline__ uint2 lds_column4(const unsigned char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) short4v*)(p)));
}
__device__ __forceinline__ void wave_fence() {   // orders a wave's own LDS accesses
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
}

typedef int int2v __attribute__((ext_vector_type(2)));
// Eight bytes of one column likewise: each lane of 16 names the 8 bytes at row r + lane / 2 (any
// eight rows), columns 8 (lane % 2).., and receives column lane.
__device__ __forceinline__ uint2 lds_column8(const unsigned char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                       (__attribute__((address_space(3))) int2v*)(p)));
}

// Keys of a tile: those of a P.V step, and twice that for the short rows of E4M3 keys, so that they
// too have bytes enough under way (us with 32 / 64 keys: E4M3, d_head 64, 79 x 3 heads of 76..7691
// keys 32.7 / 32.5; but d_head 128, 2184 x 16 of 9 keys 50 / 84).
template <typename T, int DH, typename KV>
constexpr int tile_keys() {
  return sizeof(T) == 4 ? (DH == 32 ? 32 : 16) : sizeof(KV) == 1 && DH <= 64 ? 64 : 32;
}

// What the probabilities are multiplied by in the second product.
template <typename T>
constexpr float p_scale() {
  return std::is_same<T, f16>::value ? 16384.f : 1.f;
}

// Eight probabilities, p_scale times as large, as hi + lo of the type.  hi is below each p by a few
// of its last places and never equal to it, so that both terms are positive, as p is, and an
// infinite value gives an infinite output, not inf - inf or 0 * inf (fp16: for p of 2^-28 and more).
//  fp16: hi = p (1 - 2^-10) cut, lo = p - hi < 2^-9 p cut: 2^-19 p is lost, or 2^-24 (of p_scale);
//  bf16: hi = the last fp32 value below p, cut, lo = p - hi <= 2^-7 p rounded: 2^-16 p.
template <typename T>
__device__ __forceinline__ void two_terms(const float (&p)[8], u32x4& hi, u32x4& lo) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a = p[2 * w], b = p[2 * w + 1];
    if constexpr (std::is_same<T, f16>::value) {
      constexpr float S = p_scale<T>(), BELOW = S * (1.0f - 1.0f / 1024);
      const auto h = __builtin_amdgcn_cvt_pkrtz(a * BELOW, b * BELOW);
      const auto l = __builtin_amdgcn_cvt_pkrtz(fmaf(a, S, -(float)h[0]), fmaf(b, S, -(float)h[1]));
      hi[w] = __builtin_bit_cast(unsigned, h);
      lo[w] = __builtin_bit_cast(unsigned, l);
    } else {
      const unsigned x = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u);   // (0 stays 0)
      const unsigned y = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);
      hi[w] = __builtin_amdgcn_perm(y, x, 0x07060302);
      const T l[2] = {from_f32<T>(a - __uint_as_float(x & 0xffff0000u)), from_f32<T>(b - __uint_as_float(y & 0xffff0000u))};
      lo[w] = __builtin_bit_cast(unsigned, l);
    }
  }
}

template <typename T, int DH, typename KV, int SW, bool ONCE>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int EB = sizeof(T), EC = sizeof(KV);
  constexpr bool F8 = EC == 1;
  constexpr int TK = tile_keys<T, DH, KV>();
  constexpr int NB = TK / 16;                         // 16-key blocks of a tile
  constexpr int SB = EB == 2 ? 2 : 1;                 // of them in an MFMA step of P.V
  constexpr int QK = DH * EB / 64;                    // MFMA steps over the channels
  constexpr int CB = DH / 16;                         // blocks of 16 channels of the output
  constexpr int RB = DH * EC;                         // bytes of a key
  constexpr int ROWP = RB / 16;                       // 16-byte pieces of a key
  constexpr int NP = TK * ROWP / kWave;               // pieces a lane takes of a tile's keys
  constexpr int RPL = kWave / ROWP;                   // rows that one load of the wave covers
  constexpr float PS = p_scale<T>();
  // LDS rows, padded against bank conflicts
  constexpr int KSTR = RB + 16, VSTR = RB + (EC == 2 ? 32 : 16), OSTR = DH * EB + 16;
  constexpr int KBYTES = TK * KSTR, WBYTES = KBYTES + TK * VSTR;
  static_assert(TK * ROWP % kWave == 0 && NB % SB == 0, "a tile's rows split evenly over the lanes");
  static_assert((SW == 1 ? 16 * OSTR : 16 * DH * 4) <= WBYTES && WBYTES % 16 == 0, "outputs fit in the tiles' LDS");
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * WBYTES];
  __shared__ float jm[4][16], jl[4][16];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int grp = lane >> 4, ln = lane & 15;
  // Blocks of 16 heads of one key head read the same keys (ONCE: there is one block, and the reads
  // are non-temporal): side by side in a workgroup, or eight workgroups apart, on one XCD, whose L2
  // then has them.
  const int heads = a.n_seqs * a.c.n_kv_heads;
  int unit, qb;
  if constexpr (SW == 1) {
    unit = blockIdx.x * 4 + wave;
    qb = unit % a.qblocks;
    unit /= a.qblocks;
  } else {
    const int x = blockIdx.x / 8;
    qb = x % a.qblocks;
    unit = x / a.qblocks * 8 + blockIdx.x % 8;
  }
  const int part = unit / heads, bh = unit - part * heads;
  if (part >= a.parts) return;                        // the grid's tail
  const int hk = bh % a.c.n_kv_heads, b = bh / a.c.n_kv_heads;
  const int len = max(0, min(a.lens[b], a.max_len));  // max_len is at most the table's reach
  const int c0 = part * a.chunk, c1 = min(len, c0 + a.chunk);
  if (c0 >= len && part > 0) return;                  // nothing here; the join does not look
  const int nq = min(16, a.group - qb * 16);          // heads of this block
  const int h0 = hk * a.group + qb * 16;

  const char* qrow = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (size_t)b * a.q_ld +
                                                   (size_t)(h0 + min(ln, nq - 1)) * DH);
  u32x4 qf[QK];
#pragma unroll
  for (int st = 0; st < QK; ++st) {
    // E4M3 keys of 64 channels and more come 16 a lane: steps 2p and 2p + 1 take a half each
    const int at = F8 && DH >= 64 ? st / 2 * 128 + grp * 32 + st % 2 * 16 : st * 64 + grp * 16;
    qf[st] = *reinterpret_cast<const u32x4*>(qrow + at);
  }

  const int sh = a.c.page_shift, slots = 1 << sh;
  const int* table = a.c.table + (size_t)b * a.c.max_pages;
  const size_t head_bytes = (size_t)RB << sh;         // a head's share of a page
  const char* Kp = static_cast<const char*>(a.c.k) + hk * head_bytes;
  const char* Vp = static_cast<const char*>(a.c.v) + hk * head_bytes;
  const size_t page_bytes = head_bytes * a.c.n_kv_heads;

  struct Pages { int id[NB]; };                       // of a tile's 16-key blocks; -1: none
  auto pages_of = [&](int t) {
    Pages p;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int key = t + 16 * j;
      const int id = table[min(key >> sh, a.c.max_pages - 1)];
      p.id[j] = key < len && (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
    }
    return p;
  };
  auto any_hole = [&](const Pages& p) {
    int x = p.id[0];
#pragma unroll
    for (int j = 1; j < NB; ++j) x |= p.id[j];
    return x < 0;
  };
  // A tile's rows of a pool, whole lines a load: lane l takes piece l % ROWP of row l / ROWP + RPL u.
  // Rows behind the length re-read the last one; of a hole, some page's (both masked below).
  const int row0 = lane / ROWP, col = lane % ROWP * 16;
  auto load = [&](const char* pool, int t, const Pages& p, u32x4 (&r)[NP]) {
    const char* at[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) at[j] = pool + max(p.id[j], 0) * page_bytes + (size_t)((t + 16 * j) & (slots - 1)) * RB + col;
    const int last = len - 1 - t;
    if (last >= TK - 1) {
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        const int row = row0 + u * RPL;
        const char* base = RPL <= 16 ? at[u * RPL / 16] : row0 >= 16 ? at[u * RPL / 16 + 1] : at[u * RPL / 16];
        const u32x4* q = reinterpret_cast<const u32x4*>(base + (row & 15) * RB);
        if constexpr (ONCE) r[u] = __builtin_nontemporal_load(q);
        else r[u] = *q;
      }
    } else {
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        const int row = min(row0 + u * RPL, last);
        const char* base = at[0];
#pragma unroll
        for (int j = 1; j < NB; ++j) base = row >= 16 * j ? at[j] : base;
        const u32x4* q = reinterpret_cast<const u32x4*>(base + (row & 15) * RB);
        if constexpr (ONCE) r[u] = __builtin_nontemporal_load(q);
        else r[u] = *q;
      }
    }
  };

  float m = -INFINITY, lsum = 0.f;                    // of head ln; lsum: this lane's keys only
  floatx4 o[CB];                                      // O[head 4 * grp + r][c * 16 + ln]
#pragma unroll
  for (int c = 0; c < CB; ++c) o[c] = floatx4{0.f, 0.f, 0.f, 0.f};
  unsigned char* ks = lds + wave * WBYTES;
  unsigned char* vs = ks + KBYTES;

  u32x4 kr[NP], vr[NP];
  const int step = SW * TK;
  int t = c0 + (SW == 1 ? 0 : wave * TK);
  if (t < c1) {
    Pages pg = pages_of(t);
    load(Kp, t, pg, kr);
    load(Vp, t, pg, vr);
    for (;;) {
      const int tn = t + step;
      const bool more = tn < c1;
      Pages pn = pg;
      if (more) pn = pages_of(tn);
#pragma unroll
      for (int u = 0; u < NP; ++u) *reinterpret_cast<u32x4*>(ks + (row0 + u * RPL) * KSTR + col) = kr[u];
      if (more) load(Kp, tn, pn, kr);
      wave_fence();
      floatx4 sc[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const unsigned char* krow = ks + (16 * j + ln) * KSTR;
        floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < QK; ++st) {
          u32x4 kf;
          if constexpr (!F8) {
            kf = *reinterpret_cast<const u32x4*>(krow + st * 64 + grp * 16);
          } else if constexpr (DH == 32) {
            const uint2 w = *reinterpret_cast<const uint2*>(krow + grp * 8);
            kf = f8_to_f16x8(w.x, w.y);
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(krow + st / 2 * 64 + grp * 16 + st % 2 * 8);
            kf = f8_to_f16x8(w.x, w.y);
          }
          acc = Mfma<T>::step(kf, qf[st], acc);
        }
        sc[j] = acc;
      }
      // The tile's values to LDS.  What lies behind the length, or on no page, may be anything: no
      // 0 * NaN from it
      if (t + TK > len || any_hole(pg)) {
#pragma unroll
        for (int u = 0; u < NP; ++u) {
          const int row = row0 + u * RPL;
          int id = pg.id[0];
#pragma unroll
          for (int j = 1; j < NB; ++j) id = row >= 16 * j ? pg.id[j] : id;
          if (t + row >= len || id < 0) vr[u] = u32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int u = 0; u < NP; ++u) *reinterpret_cast<u32x4*>(vs + (row0 + u * RPL) * VSTR + col) = vr[u];
      if (more) load(Vp, tn, pn, vr);
      float cmax = -INFINITY;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = t + 16 * j + 4 * grp + r;
          sc[j][r] = key < len && pg.id[j] >= 0 ? sc[j][r] * a.scale_log2 : -INFINITY;
          cmax = fmaxf(cmax, sc[j][r]);
        }
      cmax = fmaxf(cmax, __shfl_xor(cmax, 16, kWave));
      cmax = fmaxf(cmax, __shfl_xor(cmax, 32, kWave));
      const float mn = fmaxf(m, cmax);
      const float ref = mn == -INFINITY ? 0.f : mn;   // nothing but masked keys so far
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      float ps = 0.f;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[j][r] = __builtin_amdgcn_exp2f(sc[j][r] - ref);
          ps += sc[j][r];
        }
      lsum = lsum * alpha + ps;
      m = mn;
      if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float ar = __shfl(alpha, 4 * grp + r, kWave);
#pragma unroll
          for (int c = 0; c < CB; ++c) o[c][r] *= ar;
        }
      }
      wave_fence();
#pragma unroll
      for (int j = 0; j < NB; j += SB) {
        if constexpr (EB == 2) {
          float p[8];
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) p[4 * i + r] = sc[j + i][r];
          u32x4 hi, lo;
          two_terms<T>(p, hi, lo);
          // the lane's part of the columns' reads: rows 4 grp.. of both blocks
          const unsigned char* vcol = F8 ? vs + (16 * (j + (ln >> 3)) + 4 * grp + (ln >> 1 & 3)) * VSTR + (ln & 1) * 8
                                         : vs + (16 * j + 4 * grp + (ln >> 2)) * VSTR + (ln & 3) * 8;
#pragma unroll
          for (int c = 0; c < CB; ++c) {
            if constexpr (F8) {
              const uint2 w = lds_column8(vcol + c * 16);
              const u32x4 vf = f8_to_f16x8(w.x, w.y);
              o[c] = Mfma<T>::step(lo, vf, o[c]);
              o[c] = Mfma<T>::step(hi, vf, o[c]);
            } else {
              const uint2 v0 = lds_column4(vcol + c * 32), v1 = lds_column4(vcol + 16 * VSTR + c * 32);
              const u32x4 vf = u32x4{v0.x, v0.y, v1.x, v1.y};
              o[c] = Mfma<T>::step(lo, vf, o[c]);
              o[c] = Mfma<T>::step(hi, vf, o[c]);
            }
          }
        } else {
          const u32x4 pf = __builtin_bit_cast(u32x4, sc[j]);
          const unsigned char* vrow = vs + (16 * j + 4 * grp) * VSTR + ln * 4;
#pragma unroll
          for (int c = 0; c < CB; ++c) {
            u32x4 vf;
#pragma unroll
            for (int r = 0; r < 4; ++r) vf[r] = *reinterpret_cast<const unsigned*>(vrow + r * VSTR + c * 64);
            o[c] = Mfma<T>::step(pf, vf, o[c]);
          }
        }
      }
      wave_fence();
      if (!more) break;
      t = tn;
      pg = pn;
    }
  }
  lsum += __shfl_xor(lsum, 16, kWave);
  lsum += __shfl_xor(lsum, 32, kWave);

  T* out = static_cast<T*>(a.out) + (size_t)b * a.out_ld + (size_t)h0 * DH;
  const size_t prow = ((size_t)part * a.n_seqs + b) * a.n_heads + h0;   // of the workspace
  if constexpr (SW == 1) {   // the rows through LDS, to leave in 16-byte pieces
    const float inv = lsum == 0.f ? 0.f : 1.0f / (lsum * PS);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * grp + r;
      const float ir = __shfl(inv, i, kWave);
      if (i < nq)
#pragma unroll
        for (int c = 0; c < CB; ++c)
          *reinterpret_cast<T*>(ks + i * OSTR + (c * 16 + ln) * EB) = from_f32<T>(o[c][r] * ir);
    }
    wave_fence();
    constexpr int OP = DH * EB / 16;
    for (int e = lane; e < nq * OP; e += kWave)
      *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(out + e / OP * DH) + e % OP * 16) =
          *reinterpret_cast<const u32x4*>(ks + e / OP * OSTR + e % OP * 16);
    return;
  } else {
    // a wave's outputs lie where its own tiles were
    constexpr int JW = WBYTES / 4;
    float* jo = reinterpret_cast<float*>(lds);
    if (grp == 0) {
      jm[wave][ln] = m;
      jl[wave][ln] = lsum;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * grp + r;
      if (i < nq)
#pragma unroll
        for (int c = 0; c < CB; ++c) jo[wave * JW + i * DH + c * 16 + ln] = o[c][r];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < nq * (DH / 4); e += 256) {
      const int i = e / (DH / 4), x = e % (DH / 4) * 4;
      float mm = jm[0][i];
#pragma unroll
      for (int w = 1; w < SW; ++w) mm = fmaxf(mm, jm[w][i]);
      const float ref = mm == -INFINITY ? 0.f : mm;
      float l = 0.f;
      floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < SW; ++w) {
        const float f = __builtin_amdgcn_exp2f(jm[w][i] - ref);
        l += f * jl[w][i];
        s += f * (1.0f / PS) * *reinterpret_cast<const floatx4*>(jo + w * JW + i * DH + x);
      }
      if (a.parts == 1) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        alignas(16) T t4[4] = {from_f32<T>(s.x * inv), from_f32<T>(s.y * inv), from_f32<T>(s.z * inv), from_f32<T>(s.w * inv)};
        if constexpr (EB == 2) *reinterpret_cast<uint2*>(out + i * DH + x) = *reinterpret_cast<const uint2*>(t4);
        else *reinterpret_cast<uint4*>(out + i * DH + x) = *reinterpret_cast<const uint4*>(t4);
      } else {
        *reinterpret_cast<floatx4*>(a.part_o + (prow + i) * DH + x) = s;
        if (x == 0) *reinterpret_cast<float2*>(a.part_ml + (prow + i) * 2) = make_float2(mm, l);
      }
    }
  }
}

// Merges the parts of a (sequence, head): one workgroup, whose DH / 4 columns of threads take
// four channels each of every (1024 / DH)-th part, U parts' loads in flight (one round trip
// for up to 64 parts at d_head 128), each with a running maximum of its own.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int COLS = DH / 4, ROWS = 256 / COLS, U = 8;
  __shared__ __attribute__((aligned(16))) float so[ROWS][DH];
  __shared__ float sm[ROWS], sl[ROWS];
  const int bh = blockIdx.x, b = bh / a.n_heads, h = bh - b * a.n_heads;
  const int len = max(0, min(a.lens[b], a.max_len));
  const int n = max(1, (len + a.chunk - 1) / a.chunk);   // (part 0 is written for an empty row too)
  const size_t stride = (size_t)a.n_seqs * a.n_heads;
  const float* ml = a.part_ml + (size_t)bh * 2;
  const int row = threadIdx.x / COLS, x = threadIdx.x % COLS * 4;
  const float* po = a.part_o + (size_t)bh * DH + x;
  floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int p0 = row; p0 < n; p0 += ROWS * U) {
    float2 q[U];
    floatx4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t p = min(p0 + u * ROWS, n - 1);
      q[u] = *reinterpret_cast<const float2*>(ml + p * stride * 2);
      v[u] = *reinterpret_cast<const floatx4*>(po + p * stride * DH);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p0 + u * ROWS >= n) q[u] = make_float2(-INFINITY, 0.f);
      mn = fmaxf(mn, q[u].x);
    }
    const float ref = mn == -INFINITY ? 0.f : mn, f0 = __builtin_amdgcn_exp2f(m - ref);
    l *= f0;
    s *= f0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = __builtin_amdgcn_exp2f(q[u].x - ref);
      l += f * q[u].y;
      // (a part past the last is the last one's again, its weight 0)
      if (p0 + u * ROWS < n) s += f * v[u];
    }
    m = mn;
  }
  *reinterpret_cast<floatx4*>(&so[row][x]) = s;
  if (x == 0) {
    sm[row] = m;
    sl[row] = l;
  }
  __syncthreads();
  if (threadIdx.x < DH) {
    float mm = sm[0], sum = 0.f, z = 0.f;
#pragma unroll
    for (int r = 1; r < ROWS; ++r) mm = fmaxf(mm, sm[r]);
    const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float f = __builtin_amdgcn_exp2f(sm[r] - ref);
      sum += f * so[r][threadIdx.x];
      z += f * sl[r];
    }
    static_cast<T*>(a.out)[(size_t)b * a.out_ld + (size_t)h * DH + threadIdx.x] = from_f32<T>(z == 0.f ? 0.f : sum / z);
  }
}

template <typename T, int DH, typename KV, bool ONCE>
hipError_t attn_launch(const PagedAttnArgs& a, hipStream_t s) {
  const unsigned units = (unsigned)(a.n_seqs * a.c.n_kv_heads * a.parts);
  if (a.waves == 1) {
    NT_LAUNCH((paged_attn_kernel<T, DH, KV, 1, ONCE>), dim3((units * a.qblocks + 3) / 4), dim3(256), 0, s, a);
  } else {
    NT_LAUNCH((paged_attn_kernel<T, DH, KV, 4, ONCE>), dim3((units + 7) / 8 * 8 * a.qblocks), dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  NT_LAUNCH((paged_join_kernel<T, DH>), dim3((unsigned)(a.n_seqs * a.n_heads)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH, typename KV>
hipError_t attn_once(const PagedAttnArgs& a, hipStream_t s) {
  return a.qblocks == 1 ? attn_launch<T, DH, KV, true>(a, s) : attn_launch<T, DH, KV, false>(a, s);
}

template <typename T, typename KV>
hipError_t attn_dh(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.c.d_head) {
    case 32: return attn_once<T, 32, KV>(a, s);
    case 64: return attn_once<T, 64, KV>(a, s);
    case 128: return attn_once<T, 128, KV>(a, s);
    default: return hipErrorInvalidValue;
  }
}

template <typename T, bool F8>
void append_launch(const KvAppendArgs& a, bool wide, dim3 grid, hipStream_t s) {
  if (wide) NT_LAUNCH((kv_append_kernel<T, F8, 8>), grid, dim3(256), 0, s, a);
  else NT_LAUNCH((kv_append_kernel<T, F8, 4>), grid, dim3(256), 0, s, a);
}

}  // namespace

hipError_t kv_append(const KvAppendArgs& args, hipStream_t s) {
  if (args.rows <= 0) return hipSuccess;
  KvAppendArgs a = args;
  const int pieces = (int)(a.c.n_kv_heads * a.c.d_head * dt_bytes(a.c.dt) / 16);   // 4 at least
  a.piece_shift = 2;
  while (a.piece_shift < 6 && 1 << a.piece_shift < pieces) ++a.piece_shift;
  const int chunks = (pieces + (1 << a.piece_shift) - 1) >> a.piece_shift;
  const bool wide = chunks > 1;
  a.wave_rows = (kWave >> a.piece_shift) * std::max(1, (wide ? 8 : 4) / chunks);   // at most 64
  // few rows: as many waves as there are
  while (a.wave_rows > kWave >> a.piece_shift && (long long)a.rows < 4096ll * a.wave_rows) a.wave_rows /= 2;
  const dim3 grid((unsigned)((a.rows + 4ll * a.wave_rows - 1) / (4 * a.wave_rows)));
  if (a.c.fp8 && a.c.dt != DT::F16) return hipErrorInvalidValue;   // the E4M3 cache pairs with fp16
  switch (a.c.dt) {
    case DT::F32: append_launch<float, false>(a, wide, grid, s); break;
    case DT::F16:
      if (a.c.fp8) append_launch<f16, true>(a, wide, grid, s);
      else append_launch<f16, false>(a, wide, grid, s);
      break;
    case DT::BF16: append_launch<bf16, false>(a, wide, grid, s); break;
  }
  return hipGetLastError();
}

// How a call is cut, by sizes that the host knows.  Parts are multiples of 128 keys (four waves'
// tiles), as long as 512 workgroups come of it, two a CU, and at most 1024 keys: more and shorter
// ones only add to the join, longer ones leave CUs idle at the end of ragged batches.  Measured, us,
// as it is / half as long / twice: 16 x 8 heads of 2048..32768 keys (d_head 128, 1.18 GB) 196 / 200 /
// 192; one sequence, 4 heads, 131001 E4M3 keys (d_head 128) 30 / 34 / 37; 8 x 8 heads of 4000 keys
// (d_head 64) 15.9 / 17.4 / 19.4, of 16000 51 / 48 / 46; 32 x 8 of 500..8000 fp32 keys (d_head 128,
// 1.20 GB) 207 / 203 / 236.
// Never more than 32768 parts in all, however far max_len is above the lengths: empty ones cost a
// workgroup each, and every one its place in the workspace.
// Where tasks fill the GPU by themselves and are short, a wave takes one alone and nothing is joined
// (four waves a task / one): 2160 x 16 heads of up to 231 keys 194 / 164, 2048 x 8 of up to 64
// 63 / 34, of up to 256 106 / 93; but 256 x 8 of up to 256 17.2 / 17.9, 64 x 8 of up to 48 4.6 / 5.8,
// 2048 x 8 of up to 768 250 / 266.
void paged_attn_plan(PagedAttnArgs* a) {
  a->group = a->n_heads / a->c.n_kv_heads;
  a->qblocks = (a->group + 15) / 16;
  const int tasks = a->n_seqs * a->c.n_kv_heads * a->qblocks;
  const int tiles = (a->max_len + 127) / 128;
  const long long units = (long long)tiles * tasks;
  const int per = (int)std::min<long long>(
      std::max({1ll, std::min(8ll, (units + 511) / 512), (units + 32767) / 32768}), std::max(tiles, 1));
  a->chunk = per * 128;
  a->parts = std::max(1, (tiles + per - 1) / per);
  // one wave a task instead of four that share it
  a->waves = a->max_len <= 256 && tasks >= 2048 ? 1 : 4;
  if (a->waves == 1) {
    a->parts = 1;
    a->chunk = 256;
  }
}

hipError_t paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  if (a.n_seqs <= 0) return hipSuccess;
  if (a.c.fp8 && a.c.dt != DT::F16) return hipErrorInvalidValue;
  switch (a.c.dt) {
    case DT::F32: return attn_dh<float, float>(a, s);
    case DT::F16: return a.c.fp8 ? attn_dh<f16, uint8_t>(a, s) : attn_dh<f16, f16>(a, s);
    case DT::BF16: return attn_dh<bf16, bf16>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nt
