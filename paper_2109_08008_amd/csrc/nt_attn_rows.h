// Attention of many query rows: packed prompts (nt_op_attn_prompt) and several new tokens a
// sequence over a paged cache (nt_op_attn_tree).  Included once per data type.
//
//   out_i = sum_j e^{s_ij - m_i} V_j / sum_j e^{s_ij - m_i},  s_ij = scale q_i . K_j,
//
// j over the keys that row i sees; m_i is a reference near the row's largest score.  One pass over the
// keys with running sums in fp32, nothing of the scores in memory.
//
// Layout.  S^T = K Q^T, so that a lane holds one query's (lane % 16) scores of four keys a block, and
// O^T = V^T P^T takes them as its operand as they stand: the softmax goes without exchanges between
// lanes, and the factors of a moved reference are a lane's own.  Queries stay in registers; keys and values
// go through LDS, two tiles each, loaded there without registers, chunks swizzled so that no read meets
// a bank twice, values read back transposed.  The waves of a workgroup share a tile of keys: with many rows
// each has rows of its own, with few some of the tile's keys, and they join in LDS.
//
// Roundings.  16-bit probabilities are rounded once to the type, for the second product and their sum
// alike (the sum is a product with ones).  With u half a step of the type and A = sum_j p_j |V_j| that adds at
// most u (A + |o|) to the output's own u |o|, and in fp16, where probabilities below 2^-14 of the scaled ones
// have fewer bits, 2^-32 of the largest value a key.  Measured on normal inputs: 2.0e-4 .. 2.6e-4 from 64 bits (fp16),
// 1.7e-3 .. 1.9e-3 (bf16), where fp32 throughout has 2.0e-4 and 1.6e-3.  Two terms of P, as nt_op_attn_paged
// has them, would be half the products again.
//
// What bounds it, one MI355X.  Long rows: the issue of a SIMD's two waves, of which the matrix cores have
// 58 % and the softmax (a fused multiply-add, an exponential, half a conversion, a maximum an element) most of the
// rest: 16383 tokens, 16 heads of 128 channels, causal, 0.98 .. 1.0 ms = 1.1 PFLOP/s, above what a large fp16
// product reaches (1.05).  Few rows over a cache: HBM, 5.1 TB/s (64 requests of 100..4000 positions, 8 key
// heads).  Short sequences: a workgroup's reads in series (offsets, queries, tiles) with five workgroups a CU:
// 540 of 1..150 tokens, 16 heads of 64: 104 us, 3.2 TB/s.
#pragma once
#include <algorithm>

#include "nt_gemm_common.h"

namespace nt {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef int int2v __attribute__((ext_vector_type(2)));
// Four 16-bit values of one column, rows r..r+3 of an LDS tile: each lane of 16 names the
// 8 bytes at row r + lane / 4, columns 4 (lane % 4).., and receives column lane.
__device__ __forceinline__ uint2 lds_column4(const unsigned char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) short4v*)(p)));
}
// Eight bytes of one column: each lane of 16 names the 8 bytes at row r + lane / 2 (any eight
// rows), columns 8 (lane % 2).., and receives column lane.
__device__ __forceinline__ uint2 lds_column8(const unsigned char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                                       (__attribute__((address_space(3))) int2v*)(p)));
}

template <typename T>
__device__ __forceinline__ unsigned pair_of(float a, float b) {
  typedef float float2v __attribute__((ext_vector_type(2)));
  typedef T pair __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v{a, b}), pair));
}

// ---- matrix products on fixed accumulators ----
// c += A.B^T (mma) or c = A.B^T (mma0), as Mfma<T>::step, but always in the registers of c: results
// are forwarded from one product to the next only there.  The compiler does not look into the
// blocks for the wait states that gfx9 leaves to software.  So ready() stands between the vector
// instructions that form an operand and the products that take it (two are due), and settle() between
// the last product and the first other use of its result (8 after a 16-bit product, 10 after an
// fp32 one).  tests/test_device_waits.py holds the built code to them.
template <typename T>
__device__ __forceinline__ void mma(floatx4& c, u32x4 a, u32x4 b) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int w = 0; w < 4; ++w) asm("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c) : "v"(a[w]), "v"(b[w]));
  } else if constexpr (std::is_same<T, f16>::value) {
    asm("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
  } else {
    asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
  }
}
template <typename T>
__device__ __forceinline__ void mma0(floatx4& c, u32x4 a, u32x4 b) {
  if constexpr (sizeof(T) == 4) {
    asm("v_mfma_f32_16x16x4_f32 %0, %1, %2, 0" : "=&v"(c) : "v"(a[0]), "v"(b[0]));
#pragma unroll
    for (int w = 1; w < 4; ++w) asm("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+v"(c) : "v"(a[w]), "v"(b[w]));
  } else if constexpr (std::is_same<T, f16>::value) {
    asm("v_mfma_f32_16x16x32_f16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b));
  } else {
    asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "v"(b));
  }
}
template <typename V>
__device__ __forceinline__ void ready(V& x) { asm("s_nop 1" : "+v"(x)); }
template <typename V>
__device__ __forceinline__ void ready(V& x, V& y) { asm("s_nop 1" : "+v"(x), "+v"(y)); }
// The products that form c[0 .. N) are done (four at a time: all of them wait).
template <int N>
__device__ __forceinline__ void settle(floatx4* c) {
  if constexpr (N >= 4) {
    asm("s_nop 9" : "+v"(c[0]), "+v"(c[1]), "+v"(c[2]), "+v"(c[3]));
    if constexpr (N > 4) settle<N - 4>(c + 4);
  } else if constexpr (N >= 2) {
    asm("s_nop 9" : "+v"(c[0]), "+v"(c[1]));
    if constexpr (N > 2) settle<N - 2>(c + 2);
  } else {
    asm("s_nop 9" : "+v"(c[0]));
  }
}

// 0 times a word's values of T: NaN where one is no number.
template <typename T>
__device__ __forceinline__ unsigned times_zero(unsigned x) {
  constexpr unsigned E = sizeof(T) == 4 ? 0x7f800000u : std::is_same<T, f16>::value ? 0x7c00u : 0x7f80u;
  if constexpr (sizeof(T) == 4) return (x & E) == E ? 0x7fffffffu : 0u;
  else return ((x & E) == E ? 0x7fffu : 0u) | ((x & E << 16) == E << 16 ? 0x7fff0000u : 0u);
}

// Four consecutive values (uint8_t: E4M3) as fp32.
template <typename E>
__device__ __forceinline__ void four_values(const char* p, float (&x)[4]) {
  if constexpr (sizeof(E) == 1) {
    const unsigned w = *reinterpret_cast<const unsigned*>(p);
    const half2v u = __builtin_bit_cast(half2v, f8x2<false>(w)), v = __builtin_bit_cast(half2v, f8x2<true>(w));
    x[0] = (float)u[0], x[1] = (float)u[1], x[2] = (float)v[0], x[3] = (float)v[1];
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = to_f32(reinterpret_cast<const E*>(p)[r]);
  }
}

// What the probabilities are multiplied by (a power of two, 2^P_SHIFT) and how far a row's scores
// may pass its reference before that is moved (LAZY, in powers of two): fp16 probabilities stay
// below 2^(LAZY + P_SHIFT) < 65504.
constexpr float LAZY = 8.f;
template <typename T>
constexpr float p_shift() {
  return std::is_same<T, f16>::value ? 7.f : 0.f;
}

// The weight of a wave's or part's sums, whose largest score is m, beside those of largest score top.  A row whose
// scores are all -inf has a sum that is not 0 and no average; it comes out as no number unless another
// part has a score above.
__device__ __forceinline__ float share_of(float m, float top) {
  return top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
}
__device__ __forceinline__ bool no_average(float m, float l) { return m == -INFINITY && l != 0.f; }

// 16 bytes a lane, 1024 consecutive ones of LDS from dst on.  The compiler does not see the load: it
// would wait for all of them before the next read of LDS, whatever that reads.
__device__ __forceinline__ void load_to_lds(const char* base, unsigned at, unsigned dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(base), "s"(dst)
               : "memory", "m0");
}
// The same of what is read once.
__device__ __forceinline__ void load_to_lds_once(const char* base, unsigned at, unsigned dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(at), "s"(base), "s"(dst)
               : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(const char* src, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst) : "memory", "m0");
}
// An address that is the same in every lane, where the compiler cannot tell.
__device__ __forceinline__ const char* scalar(const char* p) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(p);
  return reinterpret_cast<const char*>((uintptr_t)(unsigned)__builtin_amdgcn_readfirstlane((int)x) |
                                       (uintptr_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}
// Waits until at most N of the wave's loads, those into LDS among them, are under way.
template <int N>
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }

// Which sequences a few neighbouring packed rows belong to: a wave reads 64 of the offsets, a lane one
// of them, from one that is at or below its first row on (64 probes of what is left at a time find it), and
// its lanes look their rows up there.
struct Offsets {
  const int* off;
  int n_seqs, first, mine;                    // first: of the 64; mine: off[first + lane], clamped to the last
  __device__ __forceinline__ Offsets(const int* off_, int n, int row, int lane) : off(off_), n_seqs(n), first(0) {
    for (int left = n; left >= kWave;) {      // (uniform) the last one at or below row is in [first, first + left]
      const int step = (left + kWave - 1) / kWave;
      const unsigned long long below = __ballot(off[min(first + lane * step, n)] <= row);
      first += below ? (63 - __builtin_clzll(below)) * step : 0;
      left = step;
    }
    mine = n > 0 ? off[min(first + lane, n)] : 0;
  }
  // A lane's row: the last b in [0, n_seqs] with off[b] <= row (0 if there is none; n_seqs: behind the
  // last sequence), its first row and the row behind its last one.
  __device__ __forceinline__ int find(int row, int& start, int& end) const {
    int at = 0;
#pragma unroll
    for (int s = kWave / 2; s; s >>= 1)
      if (__shfl(mine, at + s, kWave) <= row) at += s;
    start = __shfl(mine, at, kWave);
    end = __shfl(mine, min(at + 1, kWave - 1), kWave);
    int b = min(first + at, n_seqs);
    if (at == kWave - 1 && b < n_seqs) {      // beyond the 64
      int hi = n_seqs;
      while (b < hi) {
        const int mid = (b + hi + 1) >> 1;
        if (off[mid] <= row) b = mid;
        else hi = mid - 1;
      }
      start = off[b];
      end = off[min(b + 1, n_seqs)];
    }
    return b;
  }
};

// Keys of a part of a sequence's length: about a.chunk, alike in all of them; with few rows, which a join
// costs less, a.chunk at most.  Measured, us, about / at most: 12 requests of 200..500 new tokens 160 / 169,
// 16 of up to 16 new tokens over 1000..16000 positions 116 / 108.
__device__ __forceinline__ int part_keys(const RowsAttnArgs& a, int len) {
  const int n = max(1, min(a.parts, (len + (a.rblocks > 2 ? a.chunk / 2 : a.chunk - 1)) / a.chunk));
  return n == 1 ? len : ((len + n - 1) / n + 127) & ~127;
}

// A workgroup takes BM = RW * QB * 16 query rows; KW waves share the keys of a tile (BK = KW * TK).
template <typename T, int DH, typename KV, bool PAGED, int QB, int RW, int KW, int TK>
__global__ __launch_bounds__(64 * RW * KW) __attribute__((amdgpu_waves_per_eu(2))) void attn_rows_kernel(RowsAttnArgs a) {
  constexpr int EB = sizeof(T), EC = sizeof(KV);
  constexpr bool F8 = EC == 1;
  constexpr int W = RW * KW, BM = RW * QB * 16, BK = KW * TK;
  constexpr int NB = TK / 16;                 // 16-key blocks of a wave's keys of a tile
  constexpr int QK = DH * EB / 64;            // MFMA steps over the channels
  constexpr int CB = DH / 16;                 // blocks of 16 channels of the output
  constexpr int RB = DH * EC;                 // bytes of a key
  constexpr int CH = RB / 16;                 // 16-byte chunks of a key
  constexpr int TILE = BK * RB;               // bytes of a tile's keys
  constexpr int NP = TILE / (W * 1024);       // loads a lane issues for them
  constexpr int RPL = 1024 / RB;              // rows that one load of a wave covers
  constexpr int RPB = RB < 256 ? 256 / RB : 1;   // rows that the 64 banks hold side by side
  constexpr float PSH = p_shift<T>(), P1 = PSH == 0.f ? 1.f : 128.f;   // 2^PSH, a probability of 1
  static_assert(PSH == 0.f || PSH == 7.f, "P1 is its power");
  static_assert(TILE % (W * 1024) == 0 && NP >= 1, "a tile's rows split evenly over the waves");
  static_assert(EB == 4 || NB % 2 == 0, "16-bit products take 32 keys");
  // LDS: two tiles of keys, two of values; the join of waves that share rows
  constexpr int JOIN = KW > 1 ? W * QB * 16 * DH * 4 : 0;
  constexpr int LDS_BYTES = std::max(4 * TILE, JOIN);
  __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS_BYTES];
  __shared__ float jm[KW > 1 ? W : 1][QB * 16], jl[KW > 1 ? W : 1][QB * 16];
  __shared__ bool jlive[KW > 1 ? BM : 1];
  int (*range)[2] = reinterpret_cast<int(*)[2]>(lds);   // (before the first tile)

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int grp = lane >> 4, ln = lane & 15;
  const int rw = wave / KW, kw = wave % KW;

  // ---- the workgroup's rows and keys ----
  int hk, part = 0, b = 0, r0, base = 0, len = 0, n_new = 0, row_first = 0, n_live;
  int head = 0;                               // prompt: the query head
  if constexpr (PAGED) {
    const int x = blockIdx.x / 8, rb = x % a.rblocks;
    int unit = x / a.rblocks * 8 + blockIdx.x % 8;
    const int heads = a.n_seqs * a.c.n_kv_heads;
    part = unit / heads;
    unit -= part * heads;
    if (part >= a.parts) return;              // the grid's tail
    hk = unit % a.c.n_kv_heads;
    b = unit / a.c.n_kv_heads;
    r0 = rb * BM;
    row_first = a.off ? min(max(a.off[b], 0), a.n_rows) : b;
    n_new = a.off ? max(min(max(a.off[b + 1], 0), a.n_rows) - row_first, 0) : 1;
    n_live = min(n_new, a.max_new) * a.group;   // rows are (new token, head of the group)
    const int whole = a.lens[b];
    len = max(0, min(whole, a.max_len));
    base = whole - n_new;
    if (r0 >= n_live) return;
  } else {
    const int nkv = a.c.n_kv_heads, idx = blockIdx.x % a.n_heads;
    hk = idx % nkv;
    head = hk * a.group + idx / nkv;
    r0 = (a.rblocks - 1 - (int)(blockIdx.x / a.n_heads)) * BM;
    n_live = a.n_rows;
  }

  // ---- tiles of keys and values into LDS ----
  // Chunk c of row r lies at chunk c ^ f(r): 16 rows of one chunk (keys), 8 rows of two or 4 of four
  // (values' columns) fall on different banks.
  auto kswz = [](int row) { return (row / RPB) & (CH < 16 ? CH - 1 : 15); };
  auto vswz = [](int row) {
    if constexpr (EB == 4) return ((row >> 2) & 3) * 4 & (CH - 1);
    else if constexpr (F8) return ((row / RPB) & (CH - 1)) ^ (row >> 4 & 1) * (CH / 2);   // (rows of two blocks a read)
    else return ((row / RPB) & (CH / 2 - 1)) * 2;
  };
  const int sh = PAGED ? a.c.page_shift : 0, slots = 1 << sh;
  const int* table = PAGED ? a.c.table + (size_t)b * a.c.max_pages : nullptr;
  const size_t head_bytes = (size_t)RB << sh, page_bytes = head_bytes * a.c.n_kv_heads;
  const char* Kp = PAGED ? static_cast<const char*>(a.c.k) + hk * head_bytes : static_cast<const char*>(a.k) + (size_t)hk * RB;
  const char* Vp = PAGED ? static_cast<const char*>(a.c.v) + hk * head_bytes : static_cast<const char*>(a.v) + (size_t)hk * RB;
  const size_t ldb = (size_t)a.kv_ld * EB;
  // Pages of 64 blocks of 16 keys from `window` on, a block a lane, and of the 64 behind them; -1: none.
  constexpr int SPAN = 64 * 16;
  auto pages_from = [&](int t) {
    const int key = t + lane * 16;
    int id = -1;
    if (key < len) {
      id = table[min(key >> sh, a.c.max_pages - 1)];
      if ((unsigned)id >= (unsigned)a.c.n_pages) id = -1;
    }
    return id;
  };
  int window = 0, ids0 = -1, ids1 = -1;
  unsigned long long holes = 0;                         // of ids0, a bit a block
  const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)NT_LDS(lds) + wave * 1024);
  // A lane's places in the rows that its loads cover (of a page's 16 keys, or of the tile): constant, so
  // that a load takes a scalar base and no vector instruction.
  constexpr bool UNIFORM = !PAGED || RPL <= 16;         // a load's rows are on one page
  unsigned kat[UNIFORM ? NP : 1], vat[UNIFORM ? NP : 1];
  if constexpr (UNIFORM) {
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int row = (u * W + wave) * RPL + lane / CH, ch = lane % CH;
      const unsigned at = PAGED ? (row & 15) * RB : row * (unsigned)ldb;
      kat[u] = at + ((ch ^ kswz(row)) << 4);
      vat[u] = at + ((ch ^ vswz(row)) << 4);
    }
  }
  auto issue = [&](int t, int buf) {
    const unsigned kdst = lds0 + buf * TILE, vdst = kdst + 2 * TILE;
    const int ids = t - window < SPAN ? ids0 : ids1, block0 = ((t - window) >> 4) & 63;
    if constexpr (PAGED && UNIFORM) {
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        const int block = (u * W + wave) * RPL / 16;
        const int id = __builtin_amdgcn_readlane(ids, block0 + block);
        const size_t at = (size_t)max(id, 0) * page_bytes + (size_t)((t + block * 16) & (slots - 1)) * RB;
        if (a.rblocks == 1) {
          load_to_lds_once(Kp + at, kat[u], kdst + u * W * 1024);
          load_to_lds_once(Vp + at, vat[u], vdst + u * W * 1024);
        } else {
          load_to_lds(Kp + at, kat[u], kdst + u * W * 1024);
          load_to_lds(Vp + at, vat[u], vdst + u * W * 1024);
        }
      }
    } else if (!PAGED && t + BK <= a.n_rows) {
      const char *ks = scalar(Kp + t * ldb), *vs = scalar(Vp + t * ldb);
      asm volatile("s_nop 4" : "+s"(ks), "+s"(vs));     // (a load waits for scalars that vector instructions wrote)
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        load_to_lds(ks, kat[u], kdst + u * W * 1024);
        load_to_lds(vs, vat[u], vdst + u * W * 1024);
      }
    } else {                                            // rows past the buffer's: its last again
      int here = lane;
      asm volatile("" : "+v"(here));                    // (what follows from it is not kept over the loop)
#pragma unroll
      for (int u = 0; u < NP; ++u) {
        const int row = (u * W + wave) * RPL + here / CH, ch = here % CH;
        size_t at;
        if constexpr (PAGED) at = (size_t)max(__shfl(ids, block0 + row / 16, kWave), 0) * page_bytes + (size_t)((t + row) & (slots - 1)) * RB;
        else at = (size_t)min(t + row, a.n_rows - 1) * ldb;
        load_to_lds(Kp + at + ((ch ^ kswz(row)) << 4), kdst + u * W * 1024);
        load_to_lds(Vp + at + ((ch ^ vswz(row)) << 4), vdst + u * W * 1024);
      }
    }
  };
  // A lane's rows: row ln of each of the wave's QB blocks.  It sees keys [lo, hi), and of a tree the
  // new tokens of `bits`, which start at `base`.
  int lo[QB], hi[QB];
  unsigned long long bits[QB];
  const char* qrow[QB];
  bool live[QB];
  const int row0 = r0 + rw * QB * 16;         // the wave's first
  const Offsets offsets(PAGED ? nullptr : a.off, PAGED ? 0 : a.n_seqs, row0, lane);
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    const int r = row0 + q * 16 + ln;
    live[q] = r < n_live;
    bits[q] = 0;
    if constexpr (PAGED) {
      const int rr = min(r, n_live - 1), i = rr / a.group, h = hk * a.group + rr - i * a.group;
      lo[q] = 0;
      hi[q] = min(base + i + 1, len);
      if (a.mask) {
        hi[q] = min(base, len);
        const int n = max(0, min(n_new, len - base));     // (positions from len on are not read)
        bits[q] = a.mask[row_first + i] & (n >= 64 ? ~0ull : (1ull << n) - 1);
      }
      qrow[q] = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (size_t)(row_first + i) * a.q_ld + (size_t)h * DH);
    } else {
      int start, end;
      const int s = offsets.find(r, start, end);
      start = min(max(start, 0), a.n_rows);
      end = s < a.n_seqs ? min(max(end, start), a.n_rows) : start;
      live[q] = live[q] && r >= start && r < end;
      lo[q] = start;
      hi[q] = !live[q] ? start : a.causal ? r + 1 : end;
      qrow[q] = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (size_t)min(r, a.n_rows - 1) * a.q_ld +
                                              (size_t)head * DH);
    }
  }
  // Of the wave's rows: the largest lo and smallest hi (between them no mask is needed), and the range
  // outside which no row sees anything.  Both grow with the row.
  const int lo_first = __builtin_amdgcn_readlane(lo[0], 0), lo_last = __builtin_amdgcn_readlane(lo[QB - 1], 15);
  const int hi_first = __builtin_amdgcn_readlane(hi[0], 0);
  int hi_last = __builtin_amdgcn_readlane(hi[QB - 1], 15);
  int k0, k1;
  if constexpr (PAGED) {
    if (a.mask) hi_last = len;
    if (row0 >= n_live) hi_last = 0;                    // no rows
    const int keys = part_keys(a, len);
    k0 = (int)min((long long)part * keys, (long long)len);
    k1 = min(len, k0 + keys);
    if (!a.mask) k1 = min(k1, max(0, min(base + (min(r0 + BM, n_live) - 1) / a.group + 1, len)));
    if (k0 >= len && part > 0) return;                  // nothing here; the join does not look
  } else {
    k0 = lo_first;
    k1 = hi_last;
    if constexpr (RW > 1) {
      if (lane == 0 && kw == 0) {
        range[rw][0] = k0;
        range[rw][1] = k1;
      }
      __syncthreads();
      k0 = __builtin_amdgcn_readfirstlane(range[0][0]);
      k1 = __builtin_amdgcn_readfirstlane(range[RW - 1][1]);
      __syncthreads();                        // (read, before the first tile's loads)
    }
  }

  if constexpr (PAGED) {
    window = k0;
    ids0 = pages_from(k0);
    ids1 = pages_from(k0 + SPAN);
    holes = __ballot(ids0 < 0);
  }
  u32x4 qf[QB][QK];
#pragma unroll
  for (int q = 0; q < QB; ++q)
#pragma unroll
    for (int st = 0; st < QK; ++st) {
      // E4M3 keys of 64 channels and more come 16 a lane: steps 2p and 2p + 1 take a half each
      const int at = F8 && DH >= 64 ? st / 2 * 128 + grp * 32 + st % 2 * 16 : st * 64 + grp * 16;
      qf[q][st] = *reinterpret_cast<const u32x4*>(qrow[q] + at);
    }
  if (a.q_xor | ~a.q_and) {                             // a scale below or equal to 0
#pragma unroll
    for (int q = 0; q < QB; ++q)
#pragma unroll
      for (int st = 0; st < QK; ++st)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const unsigned x = qf[q][st][w];
          qf[q][st][w] = ((x & a.q_and) ^ a.q_xor) | (times_zero<T>(x) & ~a.q_and);
        }
  }

  // What lies behind the last key, or on no page, may be anything: its values become zeros (no 0 * NaN).
  const int real_end = PAGED ? len : k1;
  auto clear = [&](int t, unsigned none_of, int buf) {
    unsigned char* dst = lds + (2 + buf) * TILE + wave * 1024 + lane * 16;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
      const int row = (u * W + wave) * RPL + lane / CH;
      bool none = t + row >= real_end;
      if constexpr (PAGED) none |= (none_of >> (row / 16)) & 1;
      if (none) *reinterpret_cast<u32x4*>(dst + u * W * 1024) = u32x4{0, 0, 0, 0};
    }
  };

  float m[QB], l[QB], ref[QB];                // ref: what is added to a scaled score, p_shift - m
  floatx4 ls[QB];                             // 16-bit: the sums, by a product with ones
  floatx4 o[CB][QB];                          // O[channel c * 16 + 4 grp + r][row ln]
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    m[q] = -INFINITY;
    l[q] = ref[q] = 0.f;
    ls[q] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CB; ++c) o[c][q] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float sl = a.scale_log2;
  const unsigned one = std::is_same<T, f16>::value ? 0x3c003c00u : 0x3f803f80u;
  u32x4 ones = u32x4{one, one, one, one};
  if constexpr (EB == 2) asm volatile("" : "+v"(ones));   // kept, not formed again before each product

  auto sees = [&](int q, int key) {           // (without branches)
    if constexpr (PAGED) {
      const unsigned j = key - base;
      const unsigned w = (unsigned)(j & 32 ? bits[q] >> 32 : bits[q]) >> (j & 31);
      return (key < hi[q]) | ((j < 64u) & (w & 1u));
    } else {
      return (key >= lo[q]) & (key < hi[q]);
    }
  };

  // ---- pieces of a tile's work (ks, vs: the wave's keys and values of a tile) ----
  // Read i of the KR that a lane takes of a 16-key block's keys; a channel block's values of 32 keys (fp32: 16).
  constexpr int KR = F8 ? (QK + 1) / 2 : QK;
  auto read_k = [&](const unsigned char* ks, int j, int i) {
    const int row = 16 * j + ln, f = kswz(kw * TK + row);
    const unsigned char* krow = ks + row * RB;
    if constexpr (F8 && DH == 32) {
      const uint2 w = *reinterpret_cast<const uint2*>(krow + (((grp >> 1) ^ f) << 4) + (grp & 1) * 8);
      return u32x4{w.x, w.y, 0, 0};
    } else {
      return *reinterpret_cast<const u32x4*>(krow + (((i * 4 + grp) ^ f) << 4));
    }
  };
  auto read_v = [&](const unsigned char* vs, int j, int c) {
    if constexpr (EB == 4) {
      const int row = 16 * j + 4 * grp;
      u32x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        x[r] = *reinterpret_cast<const unsigned*>(vs + (row + r) * RB +
                                                 (((c * 4 + (ln >> 2)) ^ vswz(kw * TK + row + r)) << 4) + (ln & 3) * 4);
      return x;
    } else if constexpr (F8) {
      const int row = 16 * (j + (ln >> 3)) + 4 * grp + (ln >> 1 & 3), f = vswz(kw * TK + row);
      const uint2 w = lds_column8(vs + row * RB + (ln & 1) * 8 + ((c ^ f) << 4));
      return u32x4{w.x, w.y, 0, 0};
    } else {
      const int row = 16 * j + 4 * grp + (ln >> 2), f = vswz(kw * TK + row), h = vswz(kw * TK + row + 16);
      const unsigned char* vrow = vs + row * RB + (ln & 1) * 8;
      const int ch = 2 * c + (ln >> 1 & 1);
      const uint2 v0 = lds_column4(vrow + ((ch ^ f) << 4)), v1 = lds_column4(vrow + 16 * RB + ((ch ^ h) << 4));
      return u32x4{v0.x, v0.y, v1.x, v1.y};
    }
  };
  // One MFMA step of a block's scores; one channel block of the output.
  auto score = [&](u32x4 kf, int st, floatx4 (&s)[QB]) {
    if constexpr (F8) {
      kf = st % 2 ? f8_to_f16x8(kf.z, kf.w) : f8_to_f16x8(kf.x, kf.y);
      ready(kf);
    }
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      if (st == 0) mma0<T>(s[q], kf, qf[q][0]);
      else mma<T>(s[q], kf, qf[q][st]);
    }
  };
  auto product = [&](u32x4 vf, const u32x4 (&pf)[QB], int c) {
    if constexpr (F8) {
      vf = f8_to_f16x8(vf.x, vf.y);
      ready(vf);
    }
#pragma unroll
    for (int q = 0; q < QB; ++q) mma<T>(o[c][q], vf, pf[q]);
  };
  // A key that a lane's row does not see counts -inf.  Which ones: an interval of the row's (a tile's
  // keys against it by comparisons with constants), holes (none_of), a tree's new tokens.  sc: blocks from key t0 on.
  auto mask = [&](auto& sc, int t0, unsigned none_of) {
    constexpr int N = sizeof(sc) / sizeof(sc[0]);
    if (t0 >= lo_last && t0 + 16 * N <= hi_first && !(none_of & ((1u << N) - 1))) return;
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      const int end = hi[q] - t0 - 4 * grp, first = lo[q] - t0 - 4 * grp;
      unsigned long long tree = 0;                      // bit c: key t0 + 16 j + 4 grp + c, j a multiple of 4
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (PAGED && j % 4 == 0) {
          const int shift = base - t0 - 16 * j - 4 * grp;
          tree = shift >= 64 || shift <= -64 ? 0 : shift >= 0 ? bits[q] << shift : bits[q] >> -shift;
        }
        const unsigned part = (unsigned)(tree >> (j * 16 & 63));
        const bool there = !((none_of >> j) & 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          bool s = 16 * j + r < end;
          if constexpr (PAGED) s = (s | ((part >> r) & 1)) & there;
          else s = s & (16 * j + r >= first);
          sc[j][q][r] = s ? sc[j][q][r] : -INFINITY;
        }
      }
    }
  };
  // The reference moves only when a score (top: a lane's largest, not scaled) passes it by LAZY.
  auto move_reference = [&](float (&top)[QB]) {
    bool pass = false;
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      top[q] *= sl;
      pass = pass || top[q] > m[q] + LAZY;
    }
    if (!__ballot(pass)) return;
    settle<CB * QB>(&o[0][0]);
    settle<QB>(ls);
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      float x = top[q];
      x = fmaxf(x, __shfl_xor(x, 16, kWave));
      x = fmaxf(x, __shfl_xor(x, 32, kWave));
      const float mn = fmaxf(m[q], x);
      const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[q] - mn);
      m[q] = mn;
      ref[q] = mn == -INFINITY ? 0.f : PSH - mn;
      l[q] *= alpha;
      ls[q] *= alpha;
#pragma unroll
      for (int c = 0; c < CB; ++c) o[c][q] *= alpha;
    }
  };
  auto prob = [&](float s, int q) {
    const float p = __builtin_amdgcn_exp2f(fmaf(s, sl, ref[q]));
    if constexpr (EB == 4) l[q] += p;
    return p;
  };
  // Probabilities of 32 keys (fp32: 16) as operands, and their sums.
  auto pack = [&](const auto& sc, int j, u32x4 (&pf)[QB]) {
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      if constexpr (EB == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int w = 0; w < 2; ++w) pf[q][2 * i + w] = pair_of<T>(sc[j + i][q][2 * w], sc[j + i][q][2 * w + 1]);
      } else {
        pf[q] = __builtin_bit_cast(u32x4, sc[j][q]);
      }
      ready(pf[q]);
      if constexpr (EB == 2) mma<T>(ls[q], ones, pf[q]);
    }
  };
  constexpr int SB = EB == 2 ? 2 : 1;                   // 16-key blocks of a step of the second product
  constexpr int NE = SB * QB * 4;                       // a step's scores of a lane
  const int see_first = lo_first, see_last = min(hi_last, k1);   // the wave's rows see nothing outside

  auto compute = [&](int t, unsigned none_of, int buf) {
    const int t0 = t + kw * TK;
    if (t0 >= see_last || t0 + TK <= see_first) return;
    const unsigned char* ks = lds + buf * TILE + kw * TK * RB;
    const unsigned char* vs = lds + (2 + buf) * TILE + kw * TK * RB;
    // Scores, two blocks at a time in turn (a product waits for the one before it on the same accumulator),
    // fragments read three products' turns ahead.
    constexpr int PB = NB > 1 ? 2 : 1, NR = NB * KR, AHEAD = 3;
    floatx4 sc[NB][QB];
    u32x4 kr[AHEAD + 1];
    auto next_k = [&](int i) {
      if (i < NR) kr[i % (AHEAD + 1)] = read_k(ks, i / (PB * KR) * PB + i % PB, i % (PB * KR) / PB);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) next_k(i);
    // A wave among its products goes before the SIMD's other wave, whose softmax fills what they leave: 5 %
    // (one fp16 prompt of 16383 tokens, 16 heads of 128 channels: 1018 -> 971 us; 200..500 new tokens of 12
    // requests over 1000..8000 positions, 4 key heads of four: 196 -> 183).
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < NB * QK; ++i) {
      const int st = i % (PB * QK) / PB, j = i / (PB * QK) * PB + i % PB;
      const int read = i / (PB * QK) * PB * KR + (F8 ? st / 2 : st) * PB + i % PB;
      if (!F8 || st % 2 == 1 || QK == 1) next_k(read + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
      score(kr[read % (AHEAD + 1)], st, sc[j]);
    }
    // Values are read a group of VC channel blocks ahead, the first during the softmax.
    constexpr int VC = EB == 2 ? (CB < 4 ? CB : 4) : 1, VG = NB / SB * (CB / VC);
    u32x4 vr[2][VC];
    auto read_group = [&](int g) {
#pragma unroll
      for (int c = 0; c < VC; ++c) vr[g & 1][c] = read_v(vs, g / (CB / VC) * SB, g % (CB / VC) * VC + c);
    };
    read_group(0);
    __builtin_amdgcn_s_setprio(0);
    settle<NB * QB>(&sc[0][0]);
    mask(sc, t0, none_of >> (kw * NB));
    float top[QB];
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      top[q] = -INFINITY;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) top[q] = fmaxf(top[q], sc[j][q][r]);
    }
    move_reference(top);
    // The first step's probabilities, then each step's products with the next one's between them.
    constexpr int PER = (NE + CB - 1) / CB;
    auto next_probs = [&](int j, int first) {
#pragma unroll
      for (int e = first; e < min(first + PER, NE); ++e) {
        const int i = j + e / (QB * 4), q = e / 4 % QB, r = e % 4;
        sc[i][q][r] = prob(sc[i][q][r], q);
      }
    };
#pragma unroll
    for (int e = 0; e < NE; e += PER) next_probs(0, e);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = 0; j < NB; j += SB) {
      u32x4 pf[QB];
      pack(sc, j, pf);
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        const int g = j / SB * (CB / VC) + c / VC;
        if (c % VC == 0 && g + 1 < VG) read_group(g + 1);
        __builtin_amdgcn_sched_barrier(0);
        product(vr[g & 1][c % VC], pf, c);
        if (j + SB < NB) next_probs(j + SB, c * PER);
      }
    }
    __builtin_amdgcn_s_setprio(0);
  };
  if (k0 < k1) issue(k0, 0);
  int buf = 0;
  for (int t = k0; t < k1; t += BK) {
    loads_done<0>();                                  // this tile's
    unsigned none_of = 0;                             // blocks of the tile without a page
    if constexpr (PAGED) none_of = (unsigned)(holes >> ((t - window) >> 4)) & (unsigned)((1ull << (BK / 16)) - 1);
    if (none_of || t + BK > real_end) clear(t, none_of, buf);
    __syncthreads();
    if (t + BK < k1) issue(t + BK, buf ^ 1);
    compute(t, none_of, buf);
    buf ^= 1;
    if constexpr (PAGED) {
      if (t + BK - window == SPAN) {
        window += SPAN;
        ids0 = ids1;
        holes = __ballot(ids0 < 0);
        ids1 = pages_from(window + SPAN);
      }
    }
  }
  settle<CB * QB>(&o[0][0]);
  settle<QB>(ls);
#pragma unroll
  for (int q = 0; q < QB; ++q) {
    if constexpr (EB == 2) {
      l[q] = ls[q][0];                        // (every element of a lane is its row's sum)
    } else {
      l[q] += __shfl_xor(l[q], 16, kWave);
      l[q] += __shfl_xor(l[q], 32, kWave);
    }
  }

  // From here on o is the average of the values, which l weighs in a join: a sum of finite values may pass
  // fp32's largest number, an average of them does not.
  float inv[QB];
#pragma unroll
  for (int q = 0; q < QB; ++q) inv[q] = l[q] == 0.f ? 0.f : 1.0f / l[q];

  // Where a row came out as no number, its wave's rows are formed again key by key, so that a key or
  // value that is none (or a product that overflows) reaches the rows that see it and no others.  So are
  // scores past 2^24: a row's largest product and its reference, the same product rounded, differ by
  // steps of 1 and more, so that its probability is not 1 but may be any, 0 among them.  So are sums of values
  // that overflow: here o is the sum times the power of two that brings l into [1/4, 1/2), `down`.  And so are
  // rows that came out with nothing though they see some of the wave's keys: with scores of -inf.
  {
    float bad = 0.f;
    bool nothing = false;
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      float x = l[q] * 0.f;
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) x = fmaf(o[c][q][r], 0.f, x);
      if (m[q] > -INFINITY && l[q] < 0.5f * P1) x = 1.f;
      if (live[q]) bad += x;
      nothing |= live[q] & (m[q] == -INFINITY);
    }
    if (__ballot(nothing)) {
      auto below = [&](int x) {                         // the wave's keys below x
        const int d = max(x, k0) - k0;
        return d / BK * TK + min(max(d % BK - kw * TK, 0), TK);
      };
      unsigned long long mine = 0;                      // of a tree's new tokens
      if (PAGED && a.mask) {
        const int key = (int)((unsigned)base + lane);
        mine = __ballot(key >= k0 && key < k1 && below(key + 1) > below(key));
      }
      bool sees_some = false;
#pragma unroll
      for (int q = 0; q < QB; ++q)
        sees_some |= live[q] && m[q] == -INFINITY && ((bits[q] & mine) || below(min(hi[q], k1)) > below(lo[q]));
      if (__ballot(sees_some)) {
        bool there = !PAGED;                            // (not where a sequence has no pages at all)
        for (int t = k0; t < k1 && !there; t += SPAN) there = __ballot(pages_from(t) >= 0) != 0;
        if (there && sees_some) bad += 1.f;
      }
    }
    if (__ballot(bad != 0.f)) {
      float up[QB];                                     // 1 / down
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        m[q] = -INFINITY;
        l[q] = 0.f;
        up[q] = 1.f;
#pragma unroll
        for (int c = 0; c < CB; ++c) o[c][q] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll 1
      for (int t = k0; t < k1; t += BK) {
#pragma unroll 1
        for (int key = t + kw * TK; key < min(t + (kw + 1) * TK, k1); ++key) {
          const char *kp, *vp;
          if constexpr (PAGED) {
            const int id = table[min(key >> sh, a.c.max_pages - 1)];
            if ((unsigned)id >= (unsigned)a.c.n_pages) {
              key |= 15;                                // (the rest of the block has none either)
              continue;
            }
            const size_t at = (size_t)id * page_bytes + (size_t)(key & (slots - 1)) * RB;
            kp = Kp + at;
            vp = Vp + at;
          } else {
            kp = Kp + (size_t)key * ldb;
            vp = Vp + (size_t)key * ldb;
          }
#pragma unroll
          for (int q = 0; q < QB; ++q) {
            if (!__ballot(sees(q, key))) continue;
            float s = 0.f;
#pragma unroll 1
            for (int c = 0; c < CB; ++c) {
              float x[4], y[4];
              four_values<KV>(kp + (c * 16 + 4 * grp) * EC, x);
              four_values<T>(qrow[q] + (c * 16 + 4 * grp) * EB, y);
#pragma unroll
              for (int r = 0; r < 4; ++r) s = fmaf(x[r], a.q_and ? y[r] : y[r] * 0.f, s);
            }
            s += __shfl_xor(s, 16, kWave);
            s += __shfl_xor(s, 32, kWave);
            s *= a.scale_signed;
            asm("" : "+v"(s));                          // (rounded once, not fused with the difference below)
            if (sees(q, key)) {
              const float mn = fmaxf(m[q], s), ref = mn == -INFINITY ? 0.f : mn;
              const float alpha = __builtin_amdgcn_exp2f(m[q] - ref), p = __builtin_amdgcn_exp2f(s - ref);
              m[q] = mn;
              l[q] = l[q] * alpha + p;
              if (mn == -INFINITY && l[q] == 0.f) l[q] = 1.f;   // it sees a key
              const int e = __builtin_bit_cast(int, fmaxf(l[q], 1.f)) >> 23;   // (NaN counts as 1)
              const float down = __builtin_bit_cast(float, (252 - e) << 23), f = alpha * (down * up[q]);
              up[q] = __builtin_bit_cast(float, (e + 2) << 23);
#pragma unroll
              for (int c = 0; c < CB; ++c) {
                float v[4];
                four_values<KV>(vp + (c * 16 + 4 * grp) * EC, v);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[c][q][r] = fmaf(p, v[r] * down, o[c][q][r] * f);
              }
            }
          }
        }
      }
#pragma unroll
      for (int q = 0; q < QB; ++q) {
        inv[q] = l[q] == 0.f ? 0.f : up[q] / l[q];
        l[q] *= P1;                                     // to the scale of the others
      }
    }
  }

  // ---- the rows' outputs ----
  const bool whole_length = a.parts == 1 || part_keys(a, len) >= len;   // (else a part of it, for the join)
  auto out_row = [&](int r) -> T* {           // of the workgroup's row r
    if constexpr (PAGED) {
      const int i = (r0 + r) / a.group, h = hk * a.group + (r0 + r) - i * a.group;
      return static_cast<T*>(a.out) + (size_t)(row_first + i) * a.out_ld + (size_t)h * DH;
    } else {
      return static_cast<T*>(a.out) + (size_t)(r0 + r) * a.out_ld + (size_t)head * DH;
    }
  };
  auto part_row = [&](int r) -> size_t {
    const int i = (r0 + r) / a.group, h = hk * a.group + (r0 + r) - i * a.group;
    return ((size_t)part * a.n_rows + row_first + i) * a.n_heads + h;
  };
  auto store4 = [&](int r, int x, floatx4 s) {
    alignas(16) T t4[4] = {from_f32<T>(s.x), from_f32<T>(s.y), from_f32<T>(s.z), from_f32<T>(s.w)};
    T* p = out_row(r) + x;
    if constexpr (EB == 2) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(t4);
    else *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(t4);
  };
  if constexpr (KW == 1) {
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      const int r = (rw * QB + q) * 16 + ln;
      if (!live[q]) continue;
      if (!PAGED || whole_length) {
        if (no_average(m[q], l[q])) inv[q] = NAN;
#pragma unroll
        for (int c = 0; c < CB; ++c) store4(r, c * 16 + 4 * grp, o[c][q] * inv[q]);
      } else {
        const size_t pr = part_row(r);
#pragma unroll
        for (int c = 0; c < CB; ++c) *reinterpret_cast<floatx4*>(a.part_o + pr * DH + c * 16 + 4 * grp) = o[c][q] * inv[q];
        if (grp == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = make_float2(m[q], l[q]);
      }
    }
  } else {
    __syncthreads();                          // the tiles' LDS is free
    float* jo = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int q = 0; q < QB; ++q) {
      if (grp == 0) {
        jm[wave][q * 16 + ln] = m[q];
        jl[wave][q * 16 + ln] = l[q];
        if (kw == 0) jlive[(rw * QB + q) * 16 + ln] = live[q];
      }
#pragma unroll
      for (int c = 0; c < CB; ++c)
        *reinterpret_cast<floatx4*>(jo + ((wave * QB + q) * 16 + ln) * DH + (((c * 4 + grp) ^ (ln & 7)) << 2)) = o[c][q] * inv[q];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < BM * (DH / 4); e += 64 * W) {
      const int r = e / (DH / 4), x = e % (DH / 4);
      const int w0 = r / (QB * 16) * KW, i = r % (QB * 16);
      if (!jlive[r]) continue;
      float mm = jm[w0][i];
#pragma unroll
      for (int w = 1; w < KW; ++w) mm = fmaxf(mm, jm[w0 + w][i]);
      float f[KW], z = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        f[w] = share_of(jm[w0 + w][i], mm) * jl[w0 + w][i];
        z += f[w];
      }
      const float iz = z == 0.f ? 0.f : 1.0f / z;
      floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KW; ++w)
        s += f[w] * iz * *reinterpret_cast<const floatx4*>(jo + ((w0 + w) * QB * 16 + i) * DH + ((x ^ (i & 7)) << 2));
      if (!PAGED || whole_length) {
        if (no_average(mm, z)) s = floatx4{NAN, NAN, NAN, NAN};
        store4(r, x * 4, s);
      } else {
        const size_t pr = part_row(r);
        *reinterpret_cast<floatx4*>(a.part_o + pr * DH + x * 4) = s;
        if (x == 0) *reinterpret_cast<float2*>(a.part_ml + pr * 2) = make_float2(mm, z);
      }
    }
  }
}
// Merges the parts of ITEMS heads of a new row (averages of values and what weighs them): a wave, DH / 4 lanes four channels each of every
// (256 / DH)-th part, ITEMS * U parts' loads in flight.  Bound by HBM and a launch: 64 rows of 16 heads in 64
// parts (34 MB) 9 us, 4100 rows in 2..3 parts 14 us.
template <typename T, int DH, int ITEMS>
__global__ __launch_bounds__(256) void rows_join_kernel(RowsAttnArgs a) {
  constexpr int COLS = DH / 4, ROWS = kWave / COLS, U = 8 / ITEMS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const long long item = ((long long)blockIdx.x * 4 + wave) * ITEMS;
  const int row = (int)(item / a.n_heads), h0 = (int)(item - (long long)row * a.n_heads);
  if (row >= a.n_rows) return;
  int b = row;
  if (a.off) {
    int first, end;
    const Offsets offsets(a.off, a.n_seqs, row, lane);
    b = __builtin_amdgcn_readfirstlane(offsets.find(row, first, end));
    first = max(__builtin_amdgcn_readfirstlane(first), 0);
    if (b >= a.n_seqs || row < first || row - first >= a.max_new) return;   // a row of no sequence, or past max_new
  }
  const int len = max(0, min(a.lens[b], a.max_len));
  const int keys = part_keys(a, len);
  if (keys >= len) return;                      // one part, written where it belongs
  const int n = (len + keys - 1) / keys;
  const size_t stride = (size_t)a.n_rows * a.n_heads;
  const int p0 = lane / COLS, x = lane % COLS * 4;
  const float* ml = a.part_ml + (size_t)item * 2;
  const float* po = a.part_o + (size_t)item * DH + x;
  floatx4 s[ITEMS];
  float m[ITEMS], l[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    s[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  for (int p = p0; p < n; p += ROWS * U) {
    float2 w[ITEMS][U];
    floatx4 v[ITEMS][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)min(p + u * ROWS, n - 1) * stride;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        w[i][u] = *reinterpret_cast<const float2*>(ml + (at + i) * 2);
        v[i][u] = *reinterpret_cast<const floatx4*>(po + (at + i) * DH);
      }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float mn = m[i];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u * ROWS >= n) w[i][u] = make_float2(-INFINITY, 0.f);
        mn = fmaxf(mn, w[i][u].x);
      }
      const float l0 = l[i] * share_of(m[i], mn);
      float f[U];
      l[i] = l0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f[u] = share_of(w[i][u].x, mn) * w[i][u].y;
        l[i] += f[u];
      }
      const float inv = l[i] == 0.f ? 0.f : 1.0f / l[i];
      s[i] *= l0 * inv;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p + u * ROWS < n) s[i] += f[u] * inv * v[i][u];   // (a part past the last is the last one's again)
      m[i] = mn;
    }
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int d = COLS; d < kWave; d *= 2) {
      const float mo = __shfl_xor(m[i], d, kWave), lo = __shfl_xor(l[i], d, kWave);
      const float mn = fmaxf(m[i], mo), f = l[i] * share_of(m[i], mn), g = lo * share_of(mo, mn);
      l[i] = f + g;
      const float inv = l[i] == 0.f ? 0.f : 1.0f / l[i];
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] = s[i][r] * (f * inv) + __shfl_xor(s[i][r], d, kWave) * (g * inv);
      m[i] = mn;
    }
    if (lane >= COLS) continue;
    if (no_average(m[i], l[i])) s[i] = floatx4{NAN, NAN, NAN, NAN};
    alignas(16) T t4[4] = {from_f32<T>(s[i].x), from_f32<T>(s[i].y), from_f32<T>(s[i].z), from_f32<T>(s[i].w)};
    T* out = static_cast<T*>(a.out) + (size_t)row * a.out_ld + (size_t)(h0 + i) * DH + x;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(t4);
    else *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(t4);
  }
}

// ---- launches ----------------------------------------------------------------------------
// Keys of a wave's share of a tile (a load of each wave at least).
template <typename T, int DH, typename KV, int QB, int RW, int KW>
constexpr int rows_keys() {
  constexpr int least = 1024 * RW / (DH * (int)sizeof(KV));
  constexpr bool large = KW == 1 && QB == 2;
  return std::max(least, sizeof(T) == 4 ? (large ? 32 : 16) : large ? 64 : 32);
}

template <typename T, int DH, typename KV, bool PAGED, int QB, int RW, int KW>
hipError_t rows_launch(const RowsAttnArgs& a, unsigned grid, hipStream_t s) {
  constexpr int TK = rows_keys<T, DH, KV, QB, RW, KW>();
  NT_LAUNCH((attn_rows_kernel<T, DH, KV, PAGED, QB, RW, KW, TK>), dim3(grid), dim3(64 * RW * KW), 0, s, a);
  return hipGetLastError();
}

template <typename T, int DH, typename KV, bool PAGED>
hipError_t rows_tile(const RowsAttnArgs& a, hipStream_t s) {
  const unsigned grid = PAGED ? ((unsigned)(a.n_seqs * a.c.n_kv_heads * a.parts) + 7) / 8 * 8 * a.rblocks
                              : (unsigned)(a.rblocks * a.n_heads);
  hipError_t e = hipErrorInvalidValue;
  switch (a.tile) {
    case ROWS_128:
      if constexpr (PAGED || DH == 32 || sizeof(T) == 2) e = rows_launch<T, DH, KV, PAGED, 2, 4, 1>(a, grid, s);
      break;
    case ROWS_64: e = rows_launch<T, DH, KV, PAGED, 2, 2, 2>(a, grid, s); break;
    case ROWS_64_FINE:
      if constexpr (!PAGED && DH >= 64) e = rows_launch<T, DH, KV, PAGED, 1, 4, 1>(a, grid, s);
      break;
    case ROWS_32:
      if constexpr (!PAGED) e = rows_launch<T, DH, KV, PAGED, 2, 1, 4>(a, grid, s);
      break;
    case ROWS_16_PAIR:
      if constexpr (PAGED || DH * sizeof(T) >= 256) e = rows_launch<T, DH, KV, PAGED, 1, 1, 2>(a, grid, s);
      break;
    case ROWS_16: e = rows_launch<T, DH, KV, PAGED, 1, 1, 4>(a, grid, s); break;
  }
  if constexpr (PAGED) {
    if (e != hipSuccess || a.parts == 1) return e;
    // few parts: four heads of a row a wave
    const long long items = (long long)a.n_rows * a.n_heads;
    if (a.parts <= 8 && a.n_heads % 4 == 0)
      NT_LAUNCH((rows_join_kernel<T, DH, 4>), dim3((unsigned)((items / 4 + 3) / 4)), dim3(256), 0, s, a);
    else
      NT_LAUNCH((rows_join_kernel<T, DH, 1>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, typename KV, bool PAGED>
hipError_t rows_head(const RowsAttnArgs& a, hipStream_t s) {
  switch (a.c.d_head) {
    case 32: return rows_tile<T, 32, KV, PAGED>(a, s);
    case 64: return rows_tile<T, 64, KV, PAGED>(a, s);
    case 128: return rows_tile<T, 128, KV, PAGED>(a, s);
    default: return hipErrorInvalidValue;
  }
}
}  // namespace
}  // namespace nt
