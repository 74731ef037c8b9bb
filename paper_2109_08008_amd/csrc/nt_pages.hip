// Pages of a paged key/value cache: block tables, positions and slots from the sequences' lengths
// (nt_op_kv_resize), and drafted tokens that stay (nt_op_kv_keep).
#include <algorithm>
#include <type_traits>

#include "nt_common.h"
#include "nt_kernels.h"

namespace nt {
namespace {

// ---- resize ----------------------------------------------------------------------------
// new_b = max(len_b + add_b, 0).  Pages taken, pages given up and new rows are numbered by sums over
// the sequences before a sequence: every workgroup forms the sums that it needs from the lengths,
// which nothing writes before all have read them.  A launch bounds a step (96 sequences 3.3 us), the
// stores of positions and slots a call with many new rows (4096 sequences, 1.8 million rows, 22 MB: 16 us and
// 4.8 for the lengths by a second launch); in between it is the chain of reads, sums and barriers.  Rows are divided
// by sequences: with more than 128 of them one workgroup writes all of a sequence's (256 sequences, 200000 rows, a
// growth and its return: 53 us alike, 111 with nearly all of them one sequence's).  The sums are
// fp64 (2^16 terms below 2^31: exact), which lanes add without LDS.
struct Need {
  double rows, take, give;                    // new rows; pages taken from and given to the ring
};
__device__ __forceinline__ int pages_of(int len, int shift) {
  return (int)(((unsigned)len + (1u << shift) - 1) >> shift);
}
// A sequence's new length; past 2^31 - 1 it is -1.
__device__ __forceinline__ int new_length(int len, int add) {
  if (add <= -len) return 0;
  return add > 0x7fffffff - len ? -1 : len + add;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d, kWave);
  return v;
}
// Sum over the lanes up to and with a lane.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // lane 15 of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // lane 31 to rows 2 and 3
  return v;
}

// Sums of Need over all sequences and over [0, first), and the most pages that a sequence has or is to
// have, in every thread of the workgroup (THREADS of them).  Where no thread's share is past 2^20 the
// threads' shares are added as 32-bit integers (4096 sequences, 256 workgroups: 9.8 us with fp64 throughout).
struct Sums {
  Need all, before;
  int most;
};
template <int THREADS>
__device__ Sums resize_sums(const KvResizeArgs& a, int first) {
  constexpr int WAVES = THREADS / kWave;
  __shared__ double part[WAVES][6];
  __shared__ int parti[WAVES][8];
  double v[6] = {0, 0, 0, 0, 0, 0};
  int most = 0;
#pragma unroll 4
  for (int b = threadIdx.x; b < a.n_seqs; b += THREADS) {
    const int len = max(a.lens[b], 0), add = a.add[b], now = new_length(len, add);
    const int p0 = pages_of(len, a.page_shift), p1 = pages_of(max(now, 0), a.page_shift);
    const double x[3] = {(double)max(add, 0), (double)max(p1 - p0, 0), (double)max(p0 - p1, 0)};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      v[i] += x[i];
      if (b < first) v[3 + i] += x[i];
    }
    most = max(most, now < 0 ? 0x7fffffff : max(p0, p1));
  }
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  most = max(most, dpp_mov_i<DPP_XOR1>(most));
  most = max(most, dpp_mov_i<DPP_XOR2>(most));
  most = max(most, dpp_mov_i<DPP_HALF_MIRROR>(most));
  most = max(most, dpp_mov_i<DPP_MIRROR>(most));
  most = max(max(readlane_i(most, 0), readlane_i(most, 16)), max(readlane_i(most, 32), readlane_i(most, 48)));
  const bool large = __ballot(v[0] > 1048576.0 || v[1] > 1048576.0 || v[2] > 1048576.0);
  int t[6];
#pragma unroll
  for (int i = 0; i < 6; ++i) t[i] = readlane_i(wave_scan(large ? 0 : (int)v[i]), kWave - 1);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < 6; ++i) parti[wave][i] = t[i];
    parti[wave][6] = most;
    parti[wave][7] = large;
  }
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int i = 0; i < 6; ++i) t[i] = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
#pragma unroll
    for (int i = 0; i < 6; ++i) t[i] += parti[w][i];
    most = max(most, parti[w][6]);
    any |= parti[w][7];
  }
  if (any) {
#pragma unroll 1
    for (int i = 0; i < 6; ++i) {
      const double s = wave_sum_f64(i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : i == 3 ? v[3] : i == 4 ? v[4] : v[5]);
      if (lane == 0) part[wave][i] = s;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      v[i] = 0;
      for (int w = 0; w < WAVES; ++w) v[i] += part[w][i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 6; ++i) v[i] = t[i];
  }
  return Sums{{v[0], v[1], v[2]}, {v[3], v[4], v[5]}, most};
}

__device__ __forceinline__ int ring_head(const KvResizeArgs& a) { return (int)((unsigned)a.state[0] % (unsigned)a.n_pages); }
__device__ __forceinline__ int ring_count(const KvResizeArgs& a) { return min(max(a.state[1], 0), a.n_pages); }

// 0: the call can be done; else what it reports.
__device__ __forceinline__ int resize_status(const KvResizeArgs& a, const Sums& s, int count) {
  if (s.most > a.max_pages || s.most == 0x7fffffff || count + s.all.give > a.n_pages) return RESIZE_TABLE;
  if (s.all.rows > (a.rows >= 0 ? a.rows : 0x7fffffff)) return RESIZE_ROWS;
  return s.all.take > count ? (int)fmin(s.all.take - count, 2147483647.0) : 0;
}

// The lengths and the ring's state, once every workgroup has read them.
template <int THREADS>
__device__ __forceinline__ void resize_finish(const KvResizeArgs& a, const Sums& sums, int status, int head, int count) {
  __syncthreads();                            // (all threads have read)
  if (threadIdx.x == 0) {
    if (status == 0) {
      const unsigned to = (unsigned)head + (unsigned)sums.all.take;
      a.state[0] = (int)(to >= (unsigned)a.n_pages ? to - a.n_pages : to);
      a.state[1] = count - (int)sums.all.take + (int)sums.all.give;
    }
    a.state[2] = status;
    a.state[3] = status ? 0 : (int)sums.all.rows;
  }
  if (status == 0)
    for (int b = threadIdx.x; b < a.n_seqs; b += THREADS) a.lens[b] = new_length(max(a.lens[b], 0), a.add[b]);
}

// Column x of the grid takes the sequences [x * a.seqs, (x + 1) * a.seqs), THREADS at a time: a
// thread each for the sums, then all threads write their pages (row 0 of the grid) and positions
// and slots (the rows of the grid in turn).
template <int THREADS>
__global__ __launch_bounds__(THREADS) void resize_fill_kernel(KvResizeArgs a) {
  constexpr int WAVES = THREADS / kWave, ROWS = 4;   // rows of a thread under way together
  __shared__ int scan[WAVES][3];
  __shared__ int row0[THREADS + 1], take0[THREADS + 1], give0[THREADS + 1], len0[THREADS];
  const int first = blockIdx.x * a.seqs, last = min(a.n_seqs, first + a.seqs);
  const int head = ring_head(a), count = ring_count(a);
  const Sums sums = resize_sums<THREADS>(a, first);
  const int status = resize_status(a, sums, count);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int mask = (1 << a.page_shift) - 1;
  const int total = status ? 0 : (int)sums.all.rows;
  auto ring = [&](unsigned i) -> int& {       // i < n_pages
    const unsigned at = (unsigned)head + i;
    return a.ring[at >= (unsigned)a.n_pages ? at - a.n_pages : at];
  };
  // For each of U numbers the last of the n sums that is at most it: which of the turn's sequences has
  // it.  The U searches go on together.
  auto find = [](const int* sum, int n, const auto& i, auto& q) {
    constexpr int U = sizeof(i) / sizeof(int);
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = 0;
    for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step; step >>= 1) {
      int x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = sum[min(q[u] + step, n)];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] += q[u] + step < n && x[u] <= i[u] ? step : 0;
    }
  };
  if (status == 0) {
    int before[3] = {(int)sums.before.rows, (int)sums.before.take, (int)sums.before.give};
    for (int s0 = first; s0 < last; s0 += THREADS) {
      const int b = s0 + threadIdx.x, n = min(THREADS, last - s0);
      int len = 0, x[3] = {0, 0, 0};
      if (b < last) {
        const int add = a.add[b];
        len = max(a.lens[b], 0);
        const int p0 = pages_of(len, a.page_shift), p1 = pages_of(new_length(len, add), a.page_shift);
        x[0] = max(add, 0);
        x[1] = max(p1 - p0, 0);
        x[2] = max(p0 - p1, 0);
      }
      int v[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) v[i] = wave_scan(x[i]);
      if (s0 > first) __syncthreads();        // (the last turn's readers are done)
      if (lane == kWave - 1)
#pragma unroll
        for (int i = 0; i < 3; ++i) scan[wave][i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        v[i] += before[i];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const int y = scan[w][i];
          v[i] += w < wave ? y : 0;
          before[i] += y;
        }
      }
      row0[threadIdx.x] = v[0] - x[0];
      take0[threadIdx.x] = v[1] - x[1];
      give0[threadIdx.x] = v[2] - x[2];
      len0[threadIdx.x] = len;
      if ((int)threadIdx.x == n - 1) {
        row0[n] = v[0];
        take0[n] = v[1];
        give0[n] = v[2];
      }
      if (a.off && b < last && blockIdx.y == 0) a.off[b] = v[0] - x[0];
      __syncthreads();
      if (blockIdx.y == 0) {
        for (unsigned i = take0[0] + threadIdx.x; i < (unsigned)take0[n]; i += THREADS) {   // (i may pass 2^31)
          const int at[1] = {(int)i};
          int to[1];
          find(take0, n, at, to);
          const int q = to[0];
          a.table[(size_t)(s0 + q) * a.max_pages + pages_of(len0[q], a.page_shift) + (int)i - take0[q]] = ring(i);
        }
        for (unsigned i = give0[0] + threadIdx.x; i < (unsigned)give0[n]; i += THREADS) {
          const int num[1] = {(int)i};
          int of[1];
          find(give0, n, num, of);
          const int q = of[0];
          const int p0 = pages_of(len0[q], a.page_shift) - (give0[q + 1] - give0[q]);
          int* entry = a.table + (size_t)(s0 + q) * a.max_pages + p0 + (int)i - give0[q];
          const int page = *entry;
          *entry = -1;
          const unsigned at = (unsigned)count + i;     // behind the tail, below n_pages
          ring(at) = page;
        }
      }
      if (a.pos || a.slot) {
        const unsigned rows = row0[n], step = gridDim.y * THREADS;      // (r0 may pass 2^31)
        for (unsigned r0 = row0[0] + blockIdx.y * THREADS + threadIdx.x; r0 < rows; r0 += ROWS * step) {
          int p[ROWS], page[ROWS], r[ROWS], qs[ROWS];
#pragma unroll
          for (int u = 0; u < ROWS; ++u) r[u] = (int)min(r0 + u * step, rows - 1);
          find(row0, n, r, qs);
#pragma unroll
          for (int u = 0; u < ROWS; ++u) {
            const int q = qs[u];
            p[u] = len0[q] + r[u] - row0[q];
            // a page of this call is read from the ring: another workgroup may be writing the table
            const int p0 = pages_of(len0[q], a.page_shift), pi = p[u] >> a.page_shift;
            const int* entry = pi >= p0 ? &ring(take0[q] + pi - p0) : a.table + (size_t)(s0 + q) * a.max_pages + pi;
            page[u] = *entry;
          }
#pragma unroll
          for (int u = 0; u < ROWS; ++u) {
            if (r0 + u * step >= rows) break;
            if (a.pos) a.pos[r[u]] = p[u];
            if (a.slot) a.slot[r[u]] = ((long long)page[u] << a.page_shift) + (p[u] & mask);
          }
        }
      }
    }
  }
  const int block = blockIdx.y * gridDim.x + blockIdx.x, blocks = gridDim.x * gridDim.y;
  if (a.off && block == 0 && threadIdx.x == 0) a.off[a.n_seqs] = total;
  if (a.off && status && blockIdx.y == 0)
    for (int b = first + threadIdx.x; b < last; b += THREADS) a.off[b] = 0;
  // rows of no sequence
  for (long long r = total + (long long)block * THREADS + threadIdx.x; r < a.rows; r += (long long)blocks * THREADS) {
    if (a.pos) a.pos[r] = -1;
    if (a.slot) a.slot[r] = -1;
  }
  if (blocks == 1) resize_finish<THREADS>(a, sums, status, head, count);
}

// What resize_fill_kernel leaves where it has more than one workgroup.
constexpr int RESIZE_MANY = 1024, RESIZE_FEW = 256;
__global__ __launch_bounds__(RESIZE_MANY) void resize_end_kernel(KvResizeArgs a) {
  const int head = ring_head(a), count = ring_count(a);
  const Sums sums = resize_sums<RESIZE_MANY>(a, 0);
  resize_finish<RESIZE_MANY>(a, sums, resize_status(a, sums, count), head, count);
}

// ---- keep ------------------------------------------------------------------------------
// A wave moves 64 16-byte pieces of a sequence's rows, of keys and values, U entries of the path at a
// time.  An entry that is moved lies behind its place, so what is read was not written before.  Short
// chains bound it: the sequence's numbers, its path and pages (a lane an entry, handed round as
// scalars), the cells.  64 sequences of up to 24 new tokens 4.4 us; 900 of 48..64, 8 heads of 128 bf16
// channels, 13 us, 53 MB at 4.1 TB/s (a large copy reaches 4.9).
__global__ __launch_bounds__(256) void kv_keep_kernel(KvKeepArgs a) {
  constexpr int U = 16;
  const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int b = wave / a.waves;
  if (b >= a.n_seqs) return;
  const int cell = a.c.d_head * a.eb;         // bytes of a head's row
  const int pieces = a.c.n_kv_heads * (cell / 16);
  const int part = wave - b * a.waves;
  const int first = max(a.off[b], 0), n_new = max(a.off[b + 1] - first, 0);
  const int n = min(min(max(a.n_path[b], 0), a.max_path), n_new);
  const long long base = (long long)a.lens[b] - n_new;
  if (part == 0 && lane == 0) a.add[b] = n - n_new;
  // the lane's piece: keys' first, then values'
  int p = part * kWave + lane;
  const bool live = p < 2 * pieces;
  char* pool = static_cast<char*>(p < pieces ? a.c.k : a.c.v);
  if (p >= pieces) p -= pieces;
  p = live ? p : 0;
  const int sh = a.c.page_shift, h = p / (cell / 16);
  const size_t head_bytes = (size_t)cell << sh, page_bytes = head_bytes * a.c.n_kv_heads;
  pool += h * head_bytes + (size_t)(p * 16 - h * cell);
  const int* path = a.path + (size_t)b * a.max_path;
  const int* table = a.c.table + (size_t)b * a.c.max_pages;
  const long long page0 = base >> sh;         // lane l has page page0 + l of the sequence, -1 for none
  int pages = -1;
  if (page0 + lane >= 0 && page0 + lane < a.c.max_pages) pages = table[page0 + lane];
  // Offset of a position from the piece's place in the pool's first page; -1: it has none.
  auto cell_of = [&](long long pos) -> long long {
    const long long i = (pos >> sh) - page0;
    int page = __shfl(pages, (int)(i & (kWave - 1)), kWave);
    if (i >= kWave) page = page0 + i >= 0 && page0 + i < a.c.max_pages ? table[page0 + i] : -1;
    if (pos < 0 || (unsigned)page >= (unsigned)a.c.n_pages) return -1;
    return (long long)((size_t)page * page_bytes + (size_t)(pos & ((1 << sh) - 1)) * cell);
  };
  for (int i1 = 0; i1 < n; i1 += kWave) {
    const int i = i1 + lane, src = i < n ? path[i] : -1;   // a lane an entry
    const long long to = cell_of(base + i), from = cell_of(base + src);
    unsigned long long left = __ballot(src > i && src < n_new && to >= 0 && from >= 0);   // (else there, or none)
    while (left) {
      u32x4 v[U];
      char* dst[U];
      bool more[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        more[u] = left != 0;
        const int e = more[u] ? __builtin_ctzll(left) : 0;
        left &= left - 1;
        const long long f = (long long)(unsigned)__builtin_amdgcn_readlane((int)from, e) |
                            (long long)__builtin_amdgcn_readlane((int)(from >> 32), e) << 32;
        const long long t = (long long)(unsigned)__builtin_amdgcn_readlane((int)to, e) |
                            (long long)__builtin_amdgcn_readlane((int)(to >> 32), e) << 32;
        dst[u] = pool + t;
        if (more[u]) v[u] = *reinterpret_cast<const u32x4*>(pool + f);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (more[u] && live) *reinterpret_cast<u32x4*>(dst[u]) = v[u];
    }
  }
}

}  // namespace

hipError_t kv_resize(const KvResizeArgs& args, hipStream_t s) {
  KvResizeArgs a = args;
  // one workgroup does all of a small call; else up to 256, columns of sequences by rows of new tokens
  const bool small = a.n_seqs <= RESIZE_MANY && a.rows <= 8 * RESIZE_MANY;
  a.seqs = small ? RESIZE_MANY : std::max(1, (a.n_seqs + 255) / 256);
  const int x = std::max(1, (a.n_seqs + a.seqs - 1) / a.seqs);
  const int y = small ? 1 : std::max(1, std::min(256 / x, a.rows / RESIZE_MANY));
  if (small && a.n_seqs <= RESIZE_FEW && a.rows <= 4 * RESIZE_FEW)
    NT_LAUNCH((resize_fill_kernel<RESIZE_FEW>), dim3(1), dim3(RESIZE_FEW), 0, s, a);
  else
    NT_LAUNCH((resize_fill_kernel<RESIZE_MANY>), dim3((unsigned)x, (unsigned)y), dim3(RESIZE_MANY), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || x * y == 1) return e;
  NT_LAUNCH(resize_end_kernel, dim3(1), dim3(RESIZE_MANY), 0, s, a);
  return hipGetLastError();
}

hipError_t kv_keep(const KvKeepArgs& args, hipStream_t s) {
  if (args.n_seqs <= 0) return hipSuccess;
  KvKeepArgs a = args;
  a.waves = (2 * a.c.n_kv_heads * (a.c.d_head * a.eb / 16) + kWave - 1) / kWave;
  NT_LAUNCH(kv_keep_kernel, dim3((unsigned)(((long long)a.n_seqs * a.waves + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace nt
