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

// ---- append ----------------------------------------------------------------------------
// One wave a new row: the row's keys and values in 16-byte pieces, each to its head's page.
// A move of rows, so HBM and the launch bound it; the row's sequence is found by a search of
// 64 probes at a time (off is sorted), under way together with the row's own loads.
template <typename T, bool F8>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a) {
  constexpr int VN = Vec<T>::N, U = 4;   // pieces of keys and of values a lane has in flight
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int row = blockIdx.x * 4 + wave;
  if (row >= a.rows) return;
  const int width = a.c.n_kv_heads * a.c.d_head, pieces = width / VN;
  const T* k = static_cast<const T*>(a.k) + (size_t)row * a.ld;
  const T* v = static_cast<const T*>(a.v) + (size_t)row * a.ld;
  u32x4 kq[U], vq[U];
  auto load = [&](int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = min(p0 + u * kWave + lane, pieces - 1);   // (past the last: again, not stored)
      kq[u] = *reinterpret_cast<const u32x4*>(k + p * VN);
      vq[u] = *reinterpret_cast<const u32x4*>(v + p * VN);
    }
  };
  load(0);
  // the row's sequence b and its position: the sequence's last new row is its last position
  int b = row, behind = 1;
  if (a.off) {
    int lo = 0, hi = a.n_seqs;   // entries off[1..n_seqs] at or below the row: lo..hi of them
    while (lo < hi) {
      const int step = (hi - lo + kWave - 1) / kWave, at = lo + (lane + 1) * step;
      const int n = __popcll(__ballot(at <= hi && a.off[min(at, hi)] <= row));
      hi = min(hi, lo + (n + 1) * step - 1);
      lo += n * step;
      if (step == 1) break;
    }
    b = lo;
    if (b >= a.n_seqs || a.off[b] > row) return;   // not a row of any sequence
    behind = a.off[b + 1] - row;
  }
  const int pos = a.lens[b] - behind;
  if (pos < 0 || (pos >> a.c.page_shift) >= a.c.max_pages) return;
  const int page = a.c.table[(size_t)b * a.c.max_pages + (pos >> a.c.page_shift)];
  if ((unsigned)page >= (unsigned)a.c.n_pages) return;
  const int slot = pos & ((1 << a.c.page_shift) - 1);
  const size_t cell = ((size_t)page * a.c.n_kv_heads << a.c.page_shift) + slot;
  for (int p0 = 0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + u * kWave + lane;
      if (p >= pieces) continue;
      const int h = p * VN / a.c.d_head, x = p * VN - h * a.c.d_head;
      const size_t at = (cell + ((size_t)h << a.c.page_shift)) * a.c.d_head + x;
      if constexpr (F8) {
        static_assert(VN == 8, "E4M3 caches take 16-bit rows");
        auto codes = [](u32x4 q) {
          const half8 e = __builtin_bit_cast(half8, q);
          unsigned w[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i / 4] |= (unsigned)e4m3_rne((float)e[i]) << (i % 4 * 8);
          return make_uint2(w[0], w[1]);
        };
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.c.k) + at) = codes(kq[u]);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.c.v) + at) = codes(vq[u]);
      } else {
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.k) + at) = kq[u];
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.c.v) + at) = vq[u];
      }
    }
    p0 += U * kWave;
    if (p0 >= pieces) break;
    load(p0);
  }
}

// ---- attention -------------------------------------------------------------------------
// out_h = sum_j e^{s_j - m} V_j / sum_j e^{s_j - m},  s_j = scale q_h . K_j.
//
// A stream over the cache, bound by HBM once there are enough keys in flight: the key and
// value of a position are used once by each of the heads that share them.  Those heads (up
// to 16 a block) are the rows of the matrix products, which cost the same for one head as
// for 16 and stay far below the stream's time.  A wave takes 32 keys at a time: scores
// transposed, S^T = K.Q^T, straight from registers, so that lane l holds head l % 16's
// scores of four keys of each 16, which are the ones it supplies to P.V; the values go
// through LDS once, to be read key-major (16-bit: the transposing LDS read).  The softmax's
// running maximum and sum are fp32, in powers of two; P enters P.V in the model dtype (each
// p_j is off by at most half a step, as the values themselves are).
//
// SW waves share a task (sequence, key head, block of 16 heads, part of the length): they
// take its 32-key tiles in turn and join in LDS at the end.  A length is split into parts of
// `chunk` keys over workgroups when there are few tasks; the parts' (max, sum, unnormalised
// output) go to the workspace and paged_join_kernel merges them.
constexpr int TK = 32;          // keys of a tile
constexpr float LOG2E = 1.4426950408889634f;

typedef short short4v __attribute__((ext_vector_type(4)));
// Four 16-bit values of one column, rows r..r+3 of an LDS tile: each lane of 16 names the
// 8 bytes at row r + lane / 4, columns 4 (lane % 4).., and receives column lane.
__device__ __forceinline__ uint2 lds_column4(const unsigned char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) short4v*)(p)));
}

template <typename T, int DH, typename KV, int SW>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int EB = sizeof(T), EC = sizeof(KV);
  constexpr bool F8 = EC == 1;
  constexpr int QK = DH * EB / 64;                    // MFMA steps over the channels
  constexpr int KB = F8 && DH == 32 ? 8 : 16;         // bytes a lane loads at once of a key
  constexpr int NKL = DH * EC / (4 * KB);             // such loads a 16-key block
  constexpr int ROWP = DH * EC / 16;                  // 16-byte pieces of a value
  constexpr int VPL = TK * ROWP / kWave;              // pieces a lane takes of a tile's values
  constexpr int CB = DH / 16;                         // blocks of 16 channels of the output
  constexpr int VSTR = DH * EB / 4 + (EB == 2 ? 8 : 4);   // LDS row (dwords): no bank conflicts
  constexpr int VBYTES = TK * VSTR * 4;
  static_assert(TK * ROWP % kWave == 0, "a tile's values split evenly over the lanes");
  static_assert(SW * 16 * DH * 4 <= 4 * VBYTES || SW == 1, "the joined outputs fit in the values' LDS");
  __shared__ __attribute__((aligned(16))) unsigned char lds[4 * VBYTES];
  __shared__ float jm[4][16], jl[4][16];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int grp = lane >> 4, ln = lane & 15;
  const int n_tasks = a.n_seqs * a.c.n_kv_heads * a.qblocks;
  const int unit = SW == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  const int part = unit / n_tasks, task = unit - part * n_tasks;
  if (part >= a.parts) return;                        // (SW == 1: the grid's tail)
  const int qb = task % a.qblocks, bh = task / a.qblocks;
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
  const size_t head_bytes = (size_t)DH * EC << sh;    // a head's share of a page
  const char* Kp = static_cast<const char*>(a.c.k) + hk * head_bytes;
  const char* Vp = static_cast<const char*>(a.c.v) + hk * head_bytes;
  const size_t page_bytes = head_bytes * a.c.n_kv_heads;

  struct Pages { int id[2]; };                        // of a tile's two 16-key blocks; -1: none
  auto pages_of = [&](int t) {
    Pages p;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int key = t + 16 * j;
      const int id = table[min(key >> sh, a.c.max_pages - 1)];
      p.id[j] = key < len && (unsigned)id < (unsigned)a.c.n_pages ? id : -1;
    }
    return p;
  };
  u32x4 kr[2][NKL], vr[VPL];
  auto load_k = [&](int t, const Pages& p) {          // (of a hole: some page's, masked below)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const char* row = Kp + max(p.id[j], 0) * page_bytes + (size_t)(((t + 16 * j) & (slots - 1)) + ln) * (DH * EC);
#pragma unroll
      for (int i = 0; i < NKL; ++i) {
        if constexpr (KB == 16) {
          kr[j][i] = *reinterpret_cast<const u32x4*>(row + i * 64 + grp * 16);
        } else {
          const uint2 w = *reinterpret_cast<const uint2*>(row + i * 32 + grp * 8);
          kr[j][i] = u32x4{w.x, w.y, 0, 0};
        }
      }
    }
  };
  auto load_v = [&](int t, const Pages& p) {
    const char* at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) at[j] = Vp + max(p.id[j], 0) * page_bytes + (size_t)((t + 16 * j) & (slots - 1)) * (DH * EC);
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      const int pc = lane + u * kWave, row = pc / ROWP, col = pc % ROWP;
      vr[u] = *reinterpret_cast<const u32x4*>((row < 16 ? at[0] : at[1]) + (row & 15) * (DH * EC) + col * 16);
    }
    // what lies behind the length, or on no page, may be anything: no 0 * NaN from it
    if (t + TK > len || (p.id[0] | p.id[1]) < 0) {
#pragma unroll
      for (int u = 0; u < VPL; ++u) {
        const int row = (lane + u * kWave) / ROWP;
        if (t + row >= len || p.id[row >> 4] < 0) vr[u] = u32x4{0, 0, 0, 0};
      }
    }
  };

  float m = -INFINITY, lsum = 0.f;                    // of head ln; lsum: this lane's keys only
  floatx4 o[CB];                                      // O[head 4 * grp + r][c * 16 + ln]
#pragma unroll
  for (int c = 0; c < CB; ++c) o[c] = floatx4{0.f, 0.f, 0.f, 0.f};
  unsigned char* vs = lds + wave * VBYTES;

  const int step = SW * TK;
  int t = c0 + (SW == 1 ? 0 : wave * TK);
  if (t < c1) {
    Pages pg = pages_of(t);
    load_k(t, pg);
    load_v(t, pg);
    for (;;) {
      const int tn = t + step;
      const bool more = tn < c1;
      Pages pn = pg;
      if (more) pn = pages_of(tn);
      floatx4 sc[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        floatx4 acc = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < QK; ++st) {
          u32x4 kf;
          if constexpr (!F8) {
            kf = kr[j][st];
          } else if constexpr (DH == 32) {
            kf = f8_to_f16x8(kr[j][st].x, kr[j][st].y);
          } else {
            const u32x4 w = kr[j][st / 2];
            kf = st % 2 ? f8_to_f16x8(w.z, w.w) : f8_to_f16x8(w.x, w.y);
          }
          acc = Mfma<T>::step(kf, qf[st], acc);
        }
        sc[j] = acc;
      }
      if (more) load_k(tn, pn);
      // the tile's values to LDS, in the model dtype
#pragma unroll
      for (int u = 0; u < VPL; ++u) {
        const int pc = lane + u * kWave, row = pc / ROWP, col = pc % ROWP;
        unsigned char* d = vs + row * (VSTR * 4) + col * (F8 ? 32 : 16);
        if constexpr (F8) {
          *reinterpret_cast<u32x4*>(d) = f8_to_f16x8(vr[u].x, vr[u].y);
          *reinterpret_cast<u32x4*>(d + 16) = f8_to_f16x8(vr[u].z, vr[u].w);
        } else {
          *reinterpret_cast<u32x4*>(d) = vr[u];
        }
      }
      float cmax = -INFINITY;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = t + 16 * j + 4 * grp + r;
          sc[j][r] = key < len && pg.id[j] >= 0 ? sc[j][r] * a.scale_log2 : -INFINITY;
          cmax = fmaxf(cmax, sc[j][r]);
        }
      if (more) load_v(tn, pn);
      cmax = fmaxf(cmax, __shfl_xor(cmax, 16, kWave));
      cmax = fmaxf(cmax, __shfl_xor(cmax, 32, kWave));
      const float mn = fmaxf(m, cmax);
      const float ref = mn == -INFINITY ? 0.f : mn;   // nothing but masked keys so far
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      float ps = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j)
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
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      if constexpr (EB == 2) {
        T pe[8];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) pe[4 * j + r] = from_f32<T>(sc[j][r]);
        const u32x4 pf = __builtin_bit_cast(u32x4, pe);
        const unsigned char* col = vs + (4 * grp + (ln >> 2)) * (VSTR * 4) + (ln & 3) * 8;
#pragma unroll
        for (int c = 0; c < CB; ++c) {
          const uint2 lo = lds_column4(col + c * 32), hi = lds_column4(col + 16 * (VSTR * 4) + c * 32);
          o[c] = Mfma<T>::step(pf, u32x4{lo.x, lo.y, hi.x, hi.y}, o[c]);
        }
      } else {
        const unsigned* vw = reinterpret_cast<const unsigned*>(vs);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4 pf = __builtin_bit_cast(u32x4, sc[j]);
#pragma unroll
          for (int c = 0; c < CB; ++c) {
            u32x4 vf;
#pragma unroll
            for (int r = 0; r < 4; ++r) vf[r] = vw[(16 * j + 4 * grp + r) * VSTR + c * 16 + ln];
            o[c] = Mfma<T>::step(pf, vf, o[c]);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      if (!more) break;
      t = tn;
      pg = pn;
    }
  }
  lsum += __shfl_xor(lsum, 16, kWave);
  lsum += __shfl_xor(lsum, 32, kWave);

  T* out = static_cast<T*>(a.out) + (size_t)b * a.out_ld + (size_t)h0 * DH;
  const size_t prow = ((size_t)part * a.n_seqs + b) * a.n_heads + h0;   // of the workspace
  if constexpr (SW == 1) {
    const float inv = lsum == 0.f ? 0.f : 1.0f / lsum;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * grp + r;
      const float ir = __shfl(inv, i, kWave);
      if (i < nq)
#pragma unroll
        for (int c = 0; c < CB; ++c) out[i * DH + c * 16 + ln] = from_f32<T>(o[c][r] * ir);
    }
    return;
  } else {
    float* jo = reinterpret_cast<float*>(lds);
    __syncthreads();                                  // every wave is done with its values
    if (grp == 0) {
      jm[wave][ln] = m;
      jl[wave][ln] = lsum;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 4 * grp + r;
      if (i < nq)
#pragma unroll
        for (int c = 0; c < CB; ++c) jo[(wave * 16 + i) * DH + c * 16 + ln] = o[c][r];
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
        s += f * *reinterpret_cast<const floatx4*>(jo + (w * 16 + i) * DH + x);
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
// four channels each of every (1024 / DH)-th part.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int COLS = DH / 4, ROWS = 256 / COLS;
  __shared__ float sw[256 / kWave];
  __shared__ __attribute__((aligned(16))) float so[ROWS][DH];
  __shared__ float sl[ROWS];
  const int bh = blockIdx.x, b = bh / a.n_heads, h = bh - b * a.n_heads;
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int len = max(0, min(a.lens[b], a.max_len));
  const int n = max(1, (len + a.chunk - 1) / a.chunk);   // (part 0 is written for an empty row too)
  const size_t stride = (size_t)a.n_seqs * a.n_heads;
  const float* ml = a.part_ml + (size_t)bh * 2;
  float m = -INFINITY;
  for (int p = threadIdx.x; p < n; p += 256) m = fmaxf(m, ml[p * stride * 2]);
  m = wave_max(m);
  if (lane == 0) sw[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 256 / kWave; ++w) m = fmaxf(m, sw[w]);
  const float ref = m == -INFINITY ? 0.f : m;
  const int row = threadIdx.x / COLS, x = threadIdx.x % COLS * 4;
  floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
#pragma unroll 4
  for (int p = row; p < n; p += ROWS) {
    const float2 q = *reinterpret_cast<const float2*>(ml + p * stride * 2);
    const floatx4 v = *reinterpret_cast<const floatx4*>(a.part_o + (p * stride + bh) * DH + x);
    const float f = __builtin_amdgcn_exp2f(q.x - ref);
    l += f * q.y;
    s += f * v;
  }
  *reinterpret_cast<floatx4*>(&so[row][x]) = s;
  if (x == 0) sl[row] = l;
  __syncthreads();
  if (threadIdx.x < DH) {
    float sum = 0.f, z = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      sum += so[r][threadIdx.x];
      z += sl[r];
    }
    static_cast<T*>(a.out)[(size_t)b * a.out_ld + (size_t)h * DH + threadIdx.x] = from_f32<T>(z == 0.f ? 0.f : sum / z);
  }
}

template <typename T, int DH, typename KV>
hipError_t attn_launch(const PagedAttnArgs& a, hipStream_t s) {
  const unsigned units = (unsigned)(a.n_seqs * a.c.n_kv_heads * a.qblocks * a.parts);
  if (a.waves == 1) {
    NT_LAUNCH((paged_attn_kernel<T, DH, KV, 1>), dim3((units + 3) / 4), dim3(256), 0, s, a);
  } else {
    NT_LAUNCH((paged_attn_kernel<T, DH, KV, 4>), dim3(units), dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  NT_LAUNCH((paged_join_kernel<T, DH>), dim3((unsigned)(a.n_seqs * a.n_heads)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, typename KV>
hipError_t attn_dh(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.c.d_head) {
    case 32: return attn_launch<T, 32, KV>(a, s);
    case 64: return attn_launch<T, 64, KV>(a, s);
    case 128: return attn_launch<T, 128, KV>(a, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t kv_append(const KvAppendArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)((a.rows + 3) / 4));
  if (a.c.fp8 && a.c.dt != DT::F16) return hipErrorInvalidValue;   // the E4M3 cache pairs with fp16
  switch (a.c.dt) {
    case DT::F32: NT_LAUNCH((kv_append_kernel<float, false>), grid, dim3(256), 0, s, a); break;
    case DT::F16:
      if (a.c.fp8) NT_LAUNCH((kv_append_kernel<f16, true>), grid, dim3(256), 0, s, a);
      else NT_LAUNCH((kv_append_kernel<f16, false>), grid, dim3(256), 0, s, a);
      break;
    case DT::BF16: NT_LAUNCH((kv_append_kernel<bf16, false>), grid, dim3(256), 0, s, a); break;
  }
  return hipGetLastError();
}

// Parts are multiples of 128 keys (four waves' tiles).
void paged_attn_plan(PagedAttnArgs* a) {
  a->group = a->n_heads / a->c.n_kv_heads;
  a->qblocks = (a->group + 15) / 16;
  const int tasks = a->n_seqs * a->c.n_kv_heads * a->qblocks;
  const int tiles = (a->max_len + 4 * TK - 1) / (4 * TK);   // of 128 keys
  const int want = std::max(1, std::min(1024 / std::max(tasks, 1), tiles / 2));
  const int per = std::max(1, (tiles + want - 1) / want);
  a->chunk = per * 4 * TK;
  a->parts = std::max(1, (tiles + per - 1) / per);
  a->waves = 4;
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
