// Pages of a paged key/value cache: block tables, positions and slots from the sequences' lengths
// (nt_op_kv_resize), and drafted tokens that stay (nt_op_kv_keep).
#include <algorithm>

#include "nt_common.h"
#include "nt_kernels.h"

namespace nt {
namespace {

// ---- resize ----------------------------------------------------------------------------
// new_b = max(len_b + add_b, 0).  Pages taken, pages given up and new rows are numbered by sums over
// the sequences before a sequence: every workgroup forms the sums that it needs from the lengths,
// which nothing writes before resize_end_kernel.
struct Need {
  long long rows, take, give;                 // new rows; pages taken from and given to the ring
};
__device__ __forceinline__ Need need_of(int len, int add, int shift) {
  const long long have = max(len, 0), now = max(have + add, 0ll);
  const long long p0 = (have + (1 << shift) - 1) >> shift, p1 = (now + (1 << shift) - 1) >> shift;
  return Need{max(now - have, 0ll), max(p1 - p0, 0ll), max(p0 - p1, 0ll)};
}

__device__ __forceinline__ long long wave_sum_ll(long long v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v += __shfl_xor(v, d, kWave);
  return v;
}

constexpr int RESIZE_THREADS = 1024, RESIZE_WAVES = RESIZE_THREADS / kWave;

// Sums of Need over sequences [0, n) and over [0, first), and the most pages that a sequence is to
// have, in every thread of the workgroup.
struct Sums {
  Need all, before;
  long long most;
};
__device__ Sums resize_sums(const KvResizeArgs& a, int first) {
  __shared__ long long part[RESIZE_WAVES][7];
  Need all{0, 0, 0}, before{0, 0, 0};
  long long most = 0;
  for (int b = threadIdx.x; b < a.n_seqs; b += RESIZE_THREADS) {
    const int len = a.lens[b], add = a.add[b];
    const Need x = need_of(len, add, a.page_shift);
    all.rows += x.rows;
    all.take += x.take;
    all.give += x.give;
    if (b < first) {
      before.rows += x.rows;
      before.take += x.take;
      before.give += x.give;
    }
    const long long have = max(len, 0), now = max(have, have + add);
    // (lengths stay below 2^31)
    most = max(most, now > 0x7fffffffll ? 1ll << 40 : (now + (1 << a.page_shift) - 1) >> a.page_shift);
  }
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  long long v[7] = {all.rows, all.take, all.give, before.rows, before.take, before.give, most};
#pragma unroll
  for (int i = 0; i < 6; ++i) v[i] = wave_sum_ll(v[i]);
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v[6] = max(v[6], __shfl_xor(v[6], d, kWave));
  __syncthreads();
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < 7; ++i) part[wave][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 7; ++i) {
    v[i] = part[0][i];
    for (int w = 1; w < RESIZE_WAVES; ++w) v[i] = i == 6 ? max(v[i], part[w][i]) : v[i] + part[w][i];
  }
  return Sums{{v[0], v[1], v[2]}, {v[3], v[4], v[5]}, v[6]};
}

__device__ __forceinline__ int ring_head(const KvResizeArgs& a) { return (int)((unsigned)a.state[0] % (unsigned)a.n_pages); }
__device__ __forceinline__ int ring_count(const KvResizeArgs& a) { return min(max(a.state[1], 0), a.n_pages); }

// 0: the call can be done; else what it reports.
__device__ __forceinline__ int resize_status(const KvResizeArgs& a, const Sums& s) {
  if (s.most > a.max_pages) return RESIZE_TABLE;
  if (s.all.rows > (a.rows >= 0 ? a.rows : 0x7fffffff)) return RESIZE_ROWS;
  return (int)min(max(s.all.take - ring_count(a), 0ll), 0x7fffffffll);
}

// The lengths and the ring's state, once every workgroup has read them.
__device__ __forceinline__ void resize_finish(const KvResizeArgs& a, const Sums& sums, int status) {
  const int head = ring_head(a), free = ring_count(a);
  __syncthreads();                            // (all threads have read)
  if (threadIdx.x == 0) {
    if (status == 0) {
      a.state[0] = (int)((head + sums.all.take) % a.n_pages);
      a.state[1] = (int)min(free - sums.all.take + sums.all.give, (long long)a.n_pages);
    }
    a.state[2] = status;
    a.state[3] = status ? 0 : (int)sums.all.rows;
  }
  if (status == 0)
    for (int b = threadIdx.x; b < a.n_seqs; b += RESIZE_THREADS) {
      const int len = max(a.lens[b], 0);
      a.lens[b] = len + max(a.add[b], -len);
    }
}

// Column x of the grid takes the sequences [x * a.seqs, (x + 1) * a.seqs), RESIZE_THREADS at a time: a
// thread each for the sums, then all threads write their pages (row 0 of the grid) and positions
// and slots (the rows of the grid in turn).
__global__ __launch_bounds__(RESIZE_THREADS) void resize_fill_kernel(KvResizeArgs a) {
  __shared__ long long scan[RESIZE_WAVES][3];
  __shared__ int row0[RESIZE_THREADS + 1], take0[RESIZE_THREADS + 1], give0[RESIZE_THREADS + 1], len0[RESIZE_THREADS];
  const int first = blockIdx.x * a.seqs, last = min(a.n_seqs, first + a.seqs);
  const Sums sums = resize_sums(a, first);
  const int status = resize_status(a, sums);
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int head = ring_head(a), free = ring_count(a), mask = (1 << a.page_shift) - 1;
  const int total = status ? 0 : (int)sums.all.rows;
  auto ring = [&](long long i) -> int& { return a.ring[(head + i) % a.n_pages]; };
  // The last of the n sums that is at most i: which of the turn's sequences has the i-th.
  auto find = [](const int* sum, int n, int i) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sum[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  Need before = sums.before;
  for (int s0 = first; s0 < last; s0 += RESIZE_THREADS) {
    const int b = s0 + threadIdx.x, n = min(RESIZE_THREADS, last - s0);
    Need x{0, 0, 0};
    int len = 0;
    if (b < last && status == 0) {
      len = max(a.lens[b], 0);
      x = need_of(len, a.add[b], a.page_shift);
    }
    long long v[3] = {x.rows, x.take, x.give};   // inclusive sums over the threads
#pragma unroll
    for (int d = 1; d < kWave; d *= 2)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const long long y = __shfl_up(v[i], d, kWave);
        if (lane >= d) v[i] += y;
      }
    __syncthreads();                          // (the last turn's readers are done)
    if (lane == kWave - 1)
#pragma unroll
      for (int i = 0; i < 3; ++i) scan[wave][i] = v[i];
    __syncthreads();
    v[0] += before.rows;
    v[1] += before.take;
    v[2] += before.give;
    for (int w = 0; w < RESIZE_WAVES; ++w) {
      if (w < wave)
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] += scan[w][i];
      before.rows += scan[w][0];
      before.take += scan[w][1];
      before.give += scan[w][2];
    }
    row0[threadIdx.x] = (int)(v[0] - x.rows);
    take0[threadIdx.x] = (int)(v[1] - x.take);
    give0[threadIdx.x] = (int)(v[2] - x.give);
    len0[threadIdx.x] = len;
    if (threadIdx.x == n - 1) {
      row0[n] = (int)v[0];
      take0[n] = (int)v[1];
      give0[n] = (int)v[2];
    }
    if (a.off && b < last && blockIdx.y == 0) a.off[b] = (int)(v[0] - x.rows);
    __syncthreads();
    if (blockIdx.y == 0) {
      for (int i = take0[0] + (int)threadIdx.x; i < take0[n]; i += RESIZE_THREADS) {
        const int q = find(take0, n, i);
        const int p0 = (int)(((long long)len0[q] + mask) >> a.page_shift);
        a.table[(size_t)(s0 + q) * a.max_pages + p0 + i - take0[q]] = ring(i);
      }
      for (int i = give0[0] + (int)threadIdx.x; i < give0[n]; i += RESIZE_THREADS) {
        const int q = find(give0, n, i);
        const int p0 = (int)(((long long)len0[q] + mask) >> a.page_shift) - (give0[q + 1] - give0[q]);
        int* entry = a.table + (size_t)(s0 + q) * a.max_pages + p0 + i - give0[q];
        ring((long long)free + i) = *entry;
        *entry = -1;
      }
    }
    if (a.pos || a.slot)
      for (int r = row0[0] + (int)(blockIdx.y * RESIZE_THREADS + threadIdx.x); r < row0[n]; r += (int)gridDim.y * RESIZE_THREADS) {
        const int q = find(row0, n, r);
        const int p = len0[q] + r - row0[q];
        if (a.pos) a.pos[r] = p;
        if (a.slot) {
          // a page of this call is read from the ring: another workgroup may be writing the table
          const int p0 = (int)(((long long)len0[q] + mask) >> a.page_shift), pi = p >> a.page_shift;
          const int page = pi >= p0 ? ring((long long)take0[q] + pi - p0) : a.table[(size_t)(s0 + q) * a.max_pages + pi];
          a.slot[r] = ((long long)page << a.page_shift) + (p & mask);
        }
      }
  }
  const int block = blockIdx.y * gridDim.x + blockIdx.x, blocks = gridDim.x * gridDim.y;
  if (a.off && block == 0 && threadIdx.x == 0) a.off[a.n_seqs] = total;
  // rows of no sequence
  for (long long r = total + (long long)block * RESIZE_THREADS + threadIdx.x; r < a.rows; r += (long long)blocks * RESIZE_THREADS) {
    if (a.pos) a.pos[r] = -1;
    if (a.slot) a.slot[r] = -1;
  }
  if (blocks == 1) resize_finish(a, sums, status);
}

// What resize_fill_kernel leaves where it has more than one workgroup.
__global__ __launch_bounds__(RESIZE_THREADS) void resize_end_kernel(KvResizeArgs a) {
  const Sums sums = resize_sums(a, 0);
  resize_finish(a, sums, resize_status(a, sums));
}

// ---- keep ------------------------------------------------------------------------------
// A lane moves a 16-byte piece of a sequence's rows, of keys or values, U entries of the path at a
// time.  An entry that is moved lies behind its place, so what is read was not written before.
__global__ __launch_bounds__(256) void kv_keep_kernel(KvKeepArgs a) {
  constexpr int U = 8;
  const long long item = (long long)blockIdx.x * 256 + threadIdx.x;
  const int cell = a.c.d_head * a.eb;         // bytes of a head's row
  const int pieces = a.c.n_kv_heads * (cell / 16);
  const int b = (int)(item / (2 * pieces));
  if (b >= a.n_seqs) return;
  int p = (int)(item - (long long)b * 2 * pieces);
  const int first = max(a.off[b], 0), n_new = max(a.off[b + 1] - first, 0);
  const int n = min(min(max(a.n_path[b], 0), a.max_path), n_new);
  if (p == 0) a.add[b] = n - n_new;
  char* pool = static_cast<char*>(p < pieces ? a.c.k : a.c.v);
  if (p >= pieces) p -= pieces;
  const int h = p / (cell / 16), x = p * 16 - h * cell;
  const int* path = a.path + (size_t)b * a.max_path;
  const int* table = a.c.table + (size_t)b * a.c.max_pages;
  const long long base = (long long)a.lens[b] - n_new;
  auto at = [&](long long pos) -> char* {     // null: no such position
    if (pos < 0 || (pos >> a.c.page_shift) >= a.c.max_pages) return nullptr;
    const int page = table[pos >> a.c.page_shift];
    if ((unsigned)page >= (unsigned)a.c.n_pages) return nullptr;
    const size_t slot = (((size_t)page * a.c.n_kv_heads + h) << a.c.page_shift) + (pos & ((1 << a.c.page_shift) - 1));
    return pool + slot * cell + x;
  };
  for (int i0 = 0; i0 < n; i0 += U) {
    u32x4 v[U];
    char* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      to[u] = nullptr;
      const int i = i0 + u, src = i < n ? path[i] : 0;
      if (src <= i || src >= n_new) continue;   // there already, or no new token
      const char* from = at(base + src);
      char* dst = at(base + i);
      if (!from || !dst) continue;
      to[u] = dst;
      v[u] = *reinterpret_cast<const u32x4*>(from);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *reinterpret_cast<u32x4*>(to[u]) = v[u];
  }
}

}  // namespace

hipError_t kv_resize(const KvResizeArgs& args, hipStream_t s) {
  KvResizeArgs a = args;
  // one workgroup does all of a small call; else up to 256, columns of sequences by rows of new tokens
  const bool small = a.n_seqs <= RESIZE_THREADS && a.rows <= 8 * RESIZE_THREADS;
  a.seqs = small ? RESIZE_THREADS : std::max(1, (a.n_seqs + 255) / 256);
  const int x = std::max(1, (a.n_seqs + a.seqs - 1) / a.seqs);
  const int y = small ? 1 : std::max(1, std::min(256 / x, a.rows / RESIZE_THREADS));
  NT_LAUNCH(resize_fill_kernel, dim3((unsigned)x, (unsigned)y), dim3(RESIZE_THREADS), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || x * y == 1) return e;
  NT_LAUNCH(resize_end_kernel, dim3(1), dim3(RESIZE_THREADS), 0, s, a);
  return hipGetLastError();
}

hipError_t kv_keep(const KvKeepArgs& a, hipStream_t s) {
  if (a.n_seqs <= 0) return hipSuccess;
  const long long pieces = 2ll * a.c.n_kv_heads * (a.c.d_head * a.eb / 16) * a.n_seqs;
  NT_LAUNCH(kv_keep_kernel, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace nt
