// What a model says about given tokens: from each row of logits, in one pass, the
// log-sum-exp, the entropy, the log-probabilities of given tokens and the k best
// alternatives with theirs.
//
// With m the row's maximum, s = sum e^{x - m} and t = sum e^{x - m} (x - m):
//   lse = m + log s,   H = log s - t / s,   log p(w) = (x_w - m) - log s.
// A thread keeps (m, s, t) of what it has read, all in fp32, and rescales once a batch of
// loads: with the maximum moving from m to m', t becomes e^{m - m'} (t + s (m - m')).
//
// HBM bounds it (V values a row, read once, non-temporal), closely followed in 16 bits by
// the vector units: ten slots an element, four of them the exponential's.
//
// The alternatives are found as in the beam selection (nt_search.hip): the maxima of 64
// groups of threads give a threshold that the row's k best reach, only the threads whose
// maximum reaches it look at their values again, and each value found counts the ones
// before it under (value desc, index asc).  A row with more than SCORE_CAP values at the
// threshold (ties, above all 16-bit ones) raises it to the k-th best of some of those
// collected and collects again, until what is above it fits; then the lowest indices at the
// threshold fill up.  So the result never depends on the order of arrival.
//
// Few long rows are cut into parts over workgroups; a part leaves (m, s, t) and its k best, and
// logp_join_kernel merges them.  Short rows are a wave's each (short_logp_kernel).
//
// Measured, us (GB/s): 4000 rows of 32000 fp32 values, k = 8, 84 (6080; k = 0 82); 8192 of 32001
// bf16, k = 5, 90 (5830; k = 0 84); 1300 of 32000 fp32 32.5 (5120: every row is in flight at once, and
// nothing covers their ends); 8192 of 1000 bf16 14; 2 of 131072 fp32, k = 20, 12.7 in two launches.
// Reads alone reach 6200 GB/s on this card, 7000 non-temporal.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "nt_common.h"
#include "nt_kernels.h"

namespace nt {
namespace {

constexpr int SCORE_THREADS = 256;
constexpr int SCORE_CAP = 528;    // as many as a join keeps at most (32 parts, k = 32)
constexpr int SCORE_BATCH = 4;    // 16-byte loads of a batch; the next batch's are in flight with it
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Stats {
  float m, s, t;
};
// (m, s, t) as seen from another reference `to`.  A part without a finite value (m = -inf) has
// s = t = 0, or NaN where it held a NaN, and keeps them.  (Bounded, so that what the type's lowest
// value has summed up leaves with 0 and not with -inf * 0.)
__device__ __forceinline__ Stats rescale(Stats a, float to) {
  if (a.m == -INFINITY) return {to, a.s, a.t};
  const float d = fmaxf(a.m - to, -1e30f), f = __builtin_amdgcn_exp2f(d * LOG2E);
  return {to, a.s * f, (a.t + a.s * d) * f};
}
// The wave's, seen from the largest `best`, which is at least each lane's a.m.
__device__ __forceinline__ Stats wave_stats(Stats a, float best) {
  const float m = wave_max(best);
  a = rescale(a, m);
  return {m, wave_sum(a.s), wave_sum(a.t)};
}

__device__ __forceinline__ void wave_fence() {   // orders a wave's own LDS accesses
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
}
// (value desc, index asc)
__device__ __forceinline__ bool before(float v1, int i1, float v2, int i2) { return v1 > v2 || (v1 == v2 && i1 < i2); }

// The candidates of a workgroup: `n` (value, index) pairs, and how many come before one.
struct Candidates {
  __attribute__((aligned(16))) float v[SCORE_CAP + 8];   // (-inf, INT_MAX) behind the last
  __attribute__((aligned(16))) int i[SCORE_CAP + 8];
  int count;
};
template <int NT>
__device__ __forceinline__ void clear(Candidates& c) {   // by NT threads; a barrier before the first put
  for (int e = threadIdx.x; e < SCORE_CAP + 8; e += NT) {
    c.v[e] = -INFINITY;
    c.i[e] = INT_MAX;
  }
  if (threadIdx.x == 0) c.count = 0;
}
__device__ __forceinline__ void put(Candidates& c, float x, int i) {
  const int at = atomicAdd(&c.count, 1);
  if (at < SCORE_CAP) {
    c.v[at] = x;
    c.i[at] = i;
  }
}
// How many of the first n come before entry e (what lies behind them, up to a multiple of eight, is
// before none).
__device__ __forceinline__ int rank_of(const float* cv, const int* ci, int n, int e) {
  const float x = cv[e];
  const int i = ci[e];
  int at = 0;
#pragma unroll 1
  for (int j = 0; j < n; j += 8) {
    const float4 v0 = *reinterpret_cast<const float4*>(cv + j), v1 = *reinterpret_cast<const float4*>(cv + j + 4);
    const int4 w0 = *reinterpret_cast<const int4*>(ci + j), w1 = *reinterpret_cast<const int4*>(ci + j + 4);
    at += before(v0.x, w0.x, x, i) + before(v0.y, w0.y, x, i) + before(v0.z, w0.z, x, i) + before(v0.w, w0.w, x, i) +
          before(v1.x, w1.x, x, i) + before(v1.y, w1.y, x, i) + before(v1.z, w1.z, x, i) + before(v1.w, w1.w, x, i);
  }
  return at;
}

// The values of a 16-byte vector.
template <typename T>
__device__ __forceinline__ void widen(u32x4 q, float (&x)[Vec<T>::N]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 4) {
      x[w] = __uint_as_float(q[w]);
    } else if constexpr (std::is_same<T, bf16>::value) {
      x[2 * w] = __uint_as_float(q[w] << 16);
      x[2 * w + 1] = __uint_as_float(q[w] & 0xffff0000u);
    } else {
      const unsigned u = q[w];
      typedef _Float16 half2v __attribute__((ext_vector_type(2)));
      const half2v h = __builtin_bit_cast(half2v, u);
      x[2 * w] = (float)h[0];
      x[2 * w + 1] = (float)h[1];
    }
  }
}
template <typename T>
__device__ __forceinline__ u32x4 minus_infinity() {   // a vector of them
  const unsigned u = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
  return u32x4{u, u, u, u};
}

// The maximum of a thread's vectors.
template <typename T>
__device__ __forceinline__ float best_of(const u32x4 (&q)[SCORE_BATCH]) {
  if constexpr (std::is_same<T, f16>::value) {   // two at a time
    half8 best = __builtin_bit_cast(half8, q[0]);
#pragma unroll
    for (int u = 1; u < SCORE_BATCH; ++u) best = __builtin_elementwise_max(best, __builtin_bit_cast(half8, q[u]));
    float m = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, (float)best[e]);
    return m;
  } else {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < SCORE_BATCH; ++u) {
      float v[Vec<T>::N];
      widen<T>(q[u], v);
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) m = fmaxf(m, v[e]);
    }
    return m;
  }
}

// Takes a thread's vectors q[0 .. count - 1] (of SCORE_BATCH; the others hold -inf) into acc and
// returns their maximum.  acc is kept relative to a reference acc.m near the maximum so far, so that
// one turn over the values is enough; where a batch rises more than 2^64 above it, and in the first
// batch, the reference moves first.
// With c = ref log2(e) as rounded and r its rounding error, x log2(e) - c is one operation and
// equals (x - ref) log2(e) + r: the sums are put right by r once a batch.  That form cannot take an r
// past 1 (|ref| past 1.1e7: t and r s cancel in ever more places, and near |ref| = 2e9, where r reaches
// 128, 2^r or 2^-r leaves fp32's range) nor -inf (0 * -inf), NaN and values past 2e38, which show as a
// NaN in t; the batch is then done by differences, p max(x - ref, -1e30) (a logit of -inf adds nothing, a
// NaN stays one), and `careful` sends the wave's next batches there at once.
template <typename T, bool WHOLE>
__device__ __forceinline__ float take_batch(const u32x4 (&q)[SCORE_BATCH], int count, Stats& acc, bool& careful) {
  constexpr int VN = Vec<T>::N;
  if (!careful) {
    if (__ballot(acc.m == -INFINITY)) {
      const float m = best_of<T>(q);
      if (acc.m == -INFINITY) acc.m = m;
    }
    const float ref = acc.m == -INFINITY ? 0.f : acc.m;
    const float c = ref * LOG2E, r = fmaf(ref, LOG2E, -c);
    float s[2] = {0.f, 0.f}, t[2] = {0.f, 0.f}, best = -INFINITY;
#pragma unroll
    for (int u = 0; u < SCORE_BATCH; ++u) {
      if (!WHOLE && u >= count) break;
      float v[VN];
      widen<T>(q[u], v);
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float d = fmaf(v[e], LOG2E, -c), p = __builtin_amdgcn_exp2f(d);
        best = fmaxf(best, v[e]);
        s[e & 1] += p;
        t[e & 1] = fmaf(p, d, t[e & 1]);
      }
    }
    const float f = __builtin_amdgcn_exp2f(-r);
    const float sb = s[0] + s[1], tb = (t[0] + t[1] - r * sb) * (LN2 * f);
    careful = __ballot(tb != tb || fabsf(r) > 1.f) != 0;
    if (!careful && !__ballot((best - ref) * LOG2E > 64.f)) {
      acc.s += sb * f;
      acc.t += tb;
      return best;
    }
  }
  const float best = best_of<T>(q), mx = fmaxf(acc.m, best);
  acc = rescale(acc, mx);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sb = 0.f, tb = 0.f;
#pragma unroll
  for (int u = 0; u < SCORE_BATCH; ++u) {
    if (!WHOLE && u >= count) break;
    float v[VN];
    widen<T>(q[u], v);
#pragma unroll
    for (int e = 0; e < VN; ++e) {
      const float d = v[e] - ref, p = __builtin_amdgcn_exp2f(d * LOG2E);
      sb += p;
      tb = fmaf(p, fmaxf(d, -1e30f), tb);
    }
  }
  acc.s += sb;
  acc.t += tb;
  return best;
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void token_logp_kernel(TokenLogpArgs a) {
  constexpr int NW = NT / kWave, VN = Vec<T>::N;
  static_assert(NT == 2 * 64 || NT == 4 * 64 || NT == 16 * 64, "64 groups of NW threads");
  __shared__ float sm[NW], ss[NW], st[NW], kth[NW];
  __shared__ float4 gmax[16];
  __shared__ Candidates cand;
  __shared__ float raised;
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts;
  const int c0 = part * a.part_len, n = min(a.part_len, a.V - c0);
  const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.ld + c0;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  int token = -1;
  if (a.parts == 1 && a.n_tok > 0) token = a.tokens[(size_t)row * a.n_tok + min(tid, a.n_tok - 1)];
  if (a.k > 0) clear<NT>(cand);
  // `head` single values up to a 128-byte line (a load that straddles lines fetches both: 8192 rows
  // of 32001 bf16 values 98 us from 16-byte boundaries, of 32000 89), nv vectors and a tail; threads
  // 0 .. HEAD - 1 take the head's, the next ones the tail's
  constexpr int HEAD = 128 / (int)sizeof(T);
  const int head = (int)((128 - (reinterpret_cast<uintptr_t>(x) & 127)) & 127) / (int)sizeof(T);
  const int nv = (n - head) / VN, tail = head + nv * VN;
  // (there are some: a row here has more than SHORT values, a part 8 KB, and the last one at most a
  // value less for each other part)
  const u32x4* xv = reinterpret_cast<const u32x4*>(x + head);
  const int single = tid < HEAD ? (tid < head ? tid : -1) : tail + tid - HEAD < n ? tail + tid - HEAD : -1;
  const T single_raw = x[max(single, 0)];
  // (Past the last vector: that one again.  Of loads that only some lanes or turns issue, the compiler
  // would wait for every one under way; those of one address cost little.)
  const int last = nv - 1;
  auto load = [&](u32x4 (&q)[SCORE_BATCH], int batch) {
#pragma unroll
    for (int u = 0; u < SCORE_BATCH; ++u)
      q[u] = __builtin_nontemporal_load(xv + min(tid + (batch * SCORE_BATCH + u) * NT, last));
  };
  u32x4 q0[SCORE_BATCH], q1[SCORE_BATCH];
  load(q0, 0);
  Stats acc{-INFINITY, 0.f, 0.f};
  float single_value = -INFINITY;
  if (single >= 0) {
    const float c = to_f32(single_raw);
    single_value = acc.m = fmaxf(c, -INFINITY);
    acc.s = c == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(c - c);   // 1; NaN of an infinity or a NaN
    acc.t = c == -INFINITY ? 0.f : c - c;
  }
  // the best batch's maximum, which one it is, and the best of all others
  float first = -INFINITY, second = -INFINITY;
  int first_batch = 0;
  bool careful = false;
  auto note = [&](float best, int batch) {
    second = fmaxf(second, fminf(first, best));
    first_batch = best > first ? batch : first_batch;
    first = fmaxf(first, best);
  };
  auto take = [&](u32x4 (&q)[SCORE_BATCH], int batch) { note(take_batch<T, true>(q, SCORE_BATCH, acc, careful), batch); };
  auto take_rest = [&](u32x4 (&q)[SCORE_BATCH], int batch) {   // behind the whole batches
    if (batch * SCORE_BATCH * NT >= nv) return;
    const int count = (nv - tid + NT - 1) / NT - batch * SCORE_BATCH;
#pragma unroll
    for (int u = 0; u < SCORE_BATCH; ++u)
      if (u >= count) q[u] = minus_infinity<T>();
    note(take_batch<T, false>(q, count, acc, careful), batch);
  };
  for (int b = 0, whole = nv / (NT * SCORE_BATCH);;) {
    if (b >= whole) {
      take_rest(q0, b);
      break;
    }
    load(q1, b + 1);
    take(q0, b++);
    if (b >= whole) {
      take_rest(q1, b);
      break;
    }
    load(q0, b + 1);
    take(q1, b++);
  }
  // the given tokens' logits, under way until the end
  T given_raw{};
  if (a.parts == 1 && a.n_tok > 0) given_raw = x[(unsigned)token < (unsigned)a.V ? token : 0];
  const float mine = fmaxf(first, single_value);   // acc.m is a reference near it
  {
    const Stats w = wave_stats(acc, mine);
    if (lane == 0) {
      sm[wave] = w.m;
      ss[wave] = w.s;
      st[wave] = w.t;
    }
  }
  if (a.k > 0) {
    float g = fmaxf(mine, dpp_mov<DPP_XOR1>(mine));
    if constexpr (NW >= 4) g = fmaxf(g, dpp_mov<DPP_XOR2>(g));
#pragma unroll
    for (int o = 4; o < NW; o <<= 1) g = fmaxf(g, __shfl_xor(g, o, kWave));
    if (tid % NW == 0) reinterpret_cast<float*>(gmax)[tid / NW] = g;
  }
  __syncthreads();
  Stats all{-INFINITY, 0.f, 0.f};
  if constexpr (NW > 4) {   // a wave of the workgroup's a lane
    if (lane < NW) all = Stats{sm[lane], ss[lane], st[lane]};
    all = wave_stats(all, all.m);
  } else {
#pragma unroll
    for (int w = 0; w < NW; ++w) all.m = fmaxf(all.m, sm[w]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const Stats r = rescale(Stats{sm[w], ss[w], st[w]}, all.m);
      all.s += r.s;
      all.t += r.t;
    }
  }
  const float log_s = logf(all.s);
  if (a.parts == 1) {
    if (tid == 0) {
      const bool none = all.s == 0.f;      // no logit above -inf
      if (a.lse) a.lse[row] = none ? -INFINITY : all.m + log_s;
      if (a.entropy) a.entropy[row] = none ? 0.f : log_s - all.t / all.s;
    }
  } else if (tid == 0) {
    *reinterpret_cast<float4*>(a.part_stats + ((size_t)row * a.parts + part) * 4) = make_float4(all.m, all.s, all.t, 0.f);
  }
  auto put_given = [&] {
    if (a.parts > 1) return;   // (the join's)
    float given = to_f32(given_raw);
    for (int j = tid; j < a.n_tok; j += NT) {
      if (j >= NT) {
        token = a.tokens[(size_t)row * a.n_tok + j];
        if ((unsigned)token < (unsigned)a.V) given = to_f32(x[token]);
      }
      const float lp = given == -INFINITY && all.s == all.s ? -INFINITY : (given - all.m) - log_s;
      a.logp[(size_t)row * a.n_tok + j] = (unsigned)token < (unsigned)a.V ? lp : 0.f;
    }
  };
  if (a.k == 0) {
    put_given();
    return;
  }

  // The k-th largest group maximum: each wave counts the maxima above GW groups' ones (lane l group
  // GW wave + l % GW against GW others), the smallest with fewer than k above it is it.
  float thr;
  {
    constexpr int GW = 64 / NW;
    const float g = reinterpret_cast<const float*>(gmax)[GW * wave + lane % GW];
    float above = 0.f;
#pragma unroll
    for (int j = 0; j < GW / 4; ++j) {
      const float4 o = gmax[lane / GW * (GW / 4) + j];
      above += (o.x > g ? 1.f : 0.f) + (o.y > g ? 1.f : 0.f) + (o.z > g ? 1.f : 0.f) + (o.w > g ? 1.f : 0.f);
    }
#pragma unroll
    for (int o = GW; o < kWave; o <<= 1) above += __shfl_xor(above, o, kWave);
    const float low = -wave_max(above < (float)a.k ? -g : -INFINITY);
    if (lane == 0) kth[wave] = low;
  }
  __syncthreads();
  thr = kth[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) thr = fminf(thr, kth[w]);
  auto take_values = [&](u32x4 q, int i) {
    float v[VN];
    widen<T>(q, v);
#pragma unroll
    for (int e = 0; e < VN; ++e)
      if (v[e] >= thr && v[e] != -INFINITY) put(cand, v[e], head + VN * i + e);
  };
  if (single >= 0) {
    const float c = to_f32(single_raw);
    if (c >= thr && c != -INFINITY) put(cand, c, single);
  }
  // The wave's candidate threads, G at a time: a lane for each value of their best batches.  (Each
  // thread going through its own values took 350 instructions of every wave for the few that have
  // any: a third of what a row of 32000 16-bit values takes in all.)
  unsigned long long who = __ballot(first >= thr && first != -INFINITY);
  constexpr int PER = SCORE_BATCH * VN, G = kWave / PER;
  auto gather = [&](auto turns_c) {   // so many turns' values under way together
    constexpr int U = decltype(turns_c)::value;
    int at[U];
    float c[U];
#pragma unroll
    for (int t = 0; t < U; ++t) {
      int l = -1, batch = 0;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int next = who ? __builtin_ctzll(who) : -1;
        who &= who - 1;   // (0 stays 0)
        if (lane / PER == g) {
          l = next;
          batch = readlane_i(first_batch, max(next, 0));
        }
      }
      const int e = lane % PER, i = wave * kWave + l + (batch * SCORE_BATCH + e / VN) * NT;
      at[t] = l >= 0 && i < nv ? head + VN * i + e % VN : -1;
      c[t] = to_f32(x[max(at[t], 0)]);
    }
    unsigned long long hits[U];
    int total = 0;
#pragma unroll
    for (int t = 0; t < U; ++t) {
      hits[t] = __ballot(at[t] >= 0 && c[t] >= thr && c[t] != -INFINITY);
      total += __popcll(hits[t]);
    }
    int place = 0;
    if (lane == 0) place = atomicAdd(&cand.count, total);
    place = __builtin_amdgcn_readfirstlane(place);
#pragma unroll
    for (int t = 0; t < U; ++t) {
      const int own = place + __builtin_amdgcn_mbcnt_hi((unsigned)(hits[t] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)hits[t], 0));
      if ((hits[t] >> lane & 1) && own < SCORE_CAP) {
        cand.v[own] = c[t];
        cand.i[own] = at[t];
      }
      place += __popcll(hits[t]);
    }
  };
  while (who && *(volatile int*)&cand.count <= SCORE_CAP) {
    if (__popcll(who) <= G) gather(std::integral_constant<int, 1>{});
    else gather(std::integral_constant<int, 4>{});
  }
  // The few threads with a second batch that reaches it: the wave goes through their other vectors,
  // lane u reading u, u + 64, .. (Reading all of every candidate thread's again, a 128-byte line for
  // each 16 bytes, took a quarter of a long call: 4000 rows of 32000 fp32 values, k = 8, 102 us
  // against 82 with k = 0.)
  who = __ballot(second >= thr && second != -INFINITY);
  while (who && *(volatile int*)&cand.count <= SCORE_CAP) {
    const int l = __builtin_ctzll(who), skip = readlane_i(first_batch, l);
    who &= who - 1;
    for (int u = lane; u * NT < nv; u += kWave) {
      const int i = wave * kWave + l + u * NT;
      if (i < nv && u / SCORE_BATCH != skip) take_values(xv[i], i);
    }
  }
  __syncthreads();
  int found = cand.count;
  if (found > SCORE_CAP) {
    do {
      // raise the threshold to the k-th best of some of those collected: k values reach it
      constexpr int SAMPLE = 128;
      static_assert(SAMPLE <= SCORE_CAP && SAMPLE <= NT, "an entry a thread");
      if (tid < SAMPLE && rank_of(cand.v, cand.i, SAMPLE, tid) == a.k - 1) raised = cand.v[tid];
      __syncthreads();
      thr = raised;
      __syncthreads();
      clear<NT>(cand);
      __syncthreads();
      for (int i0 = tid; i0 < n; i0 += 16 * NT) {
        T c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = x[min(i0 + u * NT, n - 1)];
#pragma unroll
        for (int u = 0; u < 16; ++u)
          if (i0 + u * NT < n && to_f32(c[u]) > thr) put(cand, to_f32(c[u]), i0 + u * NT);
      }
      __syncthreads();
      found = cand.count;
    } while (found > SCORE_CAP);
    // fewer than k above it: the lowest indices at it, in order
    for (int i0 = 0; i0 < n && found < a.k; i0 += NT) {
      const unsigned long long at = __ballot(i0 + tid < n && to_f32(x[min(i0 + tid, n - 1)]) == thr);
      if (lane == 0) reinterpret_cast<int*>(sm)[wave] = __popcll(at);
      __syncthreads();
      int place = found, total = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int c = reinterpret_cast<const int*>(sm)[w];
        if (w < wave) place += c;
        total += c;
      }
      place += __popcll(at & ((1ull << lane) - 1));
      if ((at >> lane & 1) && place < a.k) {
        cand.v[place] = thr;
        cand.i[place] = i0 + tid;
      }
      found = min(a.k, found + total);
      __syncthreads();
    }
  }
  // each candidate's place is the number of candidates before it
  const size_t out = ((size_t)row * a.parts + part) * a.k;
  for (int e = tid; e < found; e += NT) {
    const int at = rank_of(cand.v, cand.i, found, e);
    if (at >= a.k) continue;
    if (a.parts == 1) {
      a.topi[out + at] = cand.i[e];
      a.toplp[out + at] = (cand.v[e] - all.m) - log_s;
    } else {
      a.part_v[out + at] = cand.v[e];
      a.part_i[out + at] = c0 + cand.i[e];
    }
  }
  for (int e = found + tid; e < a.k; e += NT) {   // fewer logits above -inf than k
    if (a.parts == 1) {
      a.topi[out + e] = INT_MAX;
      a.toplp[out + e] = -INFINITY;
    } else {
      a.part_v[out + e] = -INFINITY;
      a.part_i[out + e] = INT_MAX;
    }
  }
  put_given();
}

// Rows of up to SHORT values: a wave a row, its values in registers, and everything within the wave.
// The threshold is the k-th largest of the lanes' maxima.  Past SHORT_CAP values at it (ties), k turns
// of a wave-wide search for the next one.
// (A workgroup a row has most of its threads idle and half its groups empty: 8192 rows of 1000 bf16
// values, k = 5, took 38 us, with k = 32, where no threshold came of them, 566.)
// From VEC_FROM values on, a lane reads 16 bytes at a time, at whatever alignment the row has (the last
// ones end with the row and hold some of their neighbour's); shorter rows a value at a time, so that no
// lane is without (1000 rows of 2001 bf16 values, k = 8, 8.1 us by single values, 6.7 by vectors; but
// 8192 of 300, k = 32, 15 / 29: too few maxima for the threshold).
constexpr int SHORT = 2048, SHORT_CAP = 192, VEC_FROM = 1024;
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void short_logp_kernel(TokenLogpArgs a) {
  constexpr int VN = VEC ? Vec<T>::N : 1, NV = (VEC ? SHORT : VEC_FROM) / (kWave * VN);
  __shared__ __attribute__((aligned(16))) float cv[4][SHORT_CAP + 8];
  __shared__ __attribute__((aligned(16))) int ci[4][SHORT_CAP + 8];
  __shared__ __attribute__((aligned(16))) float best[4][kWave];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int row = blockIdx.x * 4 + wave;
  if (row >= a.rows) return;            // whole wave; no workgroup barrier below
  const T* x = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
  auto first = [&](int j) { return min((j * kWave + lane) * VN, a.V - VN); };   // of vector j
  struct Values { T t[VN]; };
  Values raw[NV];                       // (all under way together: nothing looks at one before)
#pragma unroll
  for (int j = 0; j < NV; ++j) __builtin_memcpy(&raw[j], x + first(j), sizeof(Values));
  int token = -1;
  float given = 0.f;
  if (lane < a.n_tok) {
    token = a.tokens[(size_t)row * a.n_tok + lane];
    if ((unsigned)token < (unsigned)a.V) given = to_f32(x[token]);
  }
  float v[NV * VN], mine = -INFINITY;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (VEC) {
      float w[VN];
      widen<T>(__builtin_bit_cast(u32x4, raw[j]), w);
#pragma unroll
      for (int e = 0; e < VN; ++e) v[j * VN + e] = w[e];
    } else {
      v[j] = to_f32(raw[j].t[0]);
    }
    if ((j + 1) * kWave * VN > a.V) {   // values of an earlier lane
      const int skip = (j * kWave + lane) * VN - first(j);
#pragma unroll
      for (int e = 0; e < VN; ++e) v[j * VN + e] = e < skip ? -INFINITY : v[j * VN + e];
    }
#pragma unroll
    for (int e = 0; e < VN; ++e) mine = fmaxf(mine, v[j * VN + e]);
  }
  const float m = wave_max(mine), ref = m == -INFINITY ? 0.f : m;
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (j * kWave * VN >= a.V) break;
#pragma unroll
    for (int e = 0; e < VN; ++e) {
      const float d = v[j * VN + e] - ref, p = __builtin_amdgcn_exp2f(d * LOG2E);
      s += p;
      t = fmaf(p, fmaxf(d, -1e30f), t);   // 0, not NaN, of a logit of -inf
    }
  }
  s = wave_sum(s);
  t = wave_sum(t);
  const float log_s = logf(s);
  if (lane == 0) {
    const bool none = s == 0.f;           // no logit above -inf
    if (a.lse) a.lse[row] = none ? -INFINITY : m + log_s;
    if (a.entropy) a.entropy[row] = none ? 0.f : log_s - t / s;
  }
  for (int j = lane; j < a.n_tok; j += kWave) {
    if (j >= kWave) {
      token = a.tokens[(size_t)row * a.n_tok + j];
      if ((unsigned)token < (unsigned)a.V) given = to_f32(x[token]);
    }
    const float lp = given == -INFINITY && s == s ? -INFINITY : (given - m) - log_s;
    a.logp[(size_t)row * a.n_tok + j] = (unsigned)token < (unsigned)a.V ? lp : 0.f;
  }
  if (a.k == 0) return;
  best[wave][lane] = mine;
  wave_fence();
  int above = 0;
#pragma unroll
  for (int j = 0; j < kWave; j += 4) {
    const float4 o = *reinterpret_cast<const float4*>(&best[wave][j]);
    above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
  }
  const float thr = -wave_max(above < a.k ? -mine : -INFINITY);
  int found = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if (j * kWave * VN >= a.V) break;
#pragma unroll
    for (int e = 0; e < VN; ++e) {
      const float c = v[j * VN + e];
      const unsigned long long hits = __ballot(c >= thr && c != -INFINITY);
      if (!hits) continue;
      const int place = found + __builtin_amdgcn_mbcnt_hi((unsigned)(hits >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)hits, 0));
      if ((hits >> lane & 1) && place < SHORT_CAP) {
        cv[wave][place] = c;
        ci[wave][place] = first(j) + e;
      }
      found += __popcll(hits);
    }
  }
  const size_t out = (size_t)row * a.k;
  if (found <= SHORT_CAP) {
    if (lane < 8) {
      cv[wave][found + lane] = -INFINITY;
      ci[wave][found + lane] = INT_MAX;
    }
    wave_fence();
    for (int e = lane; e < found; e += kWave) {
      const int at = rank_of(cv[wave], ci[wave], found, e);
      if (at < a.k) {
        a.topi[out + at] = ci[wave][e];
        a.toplp[out + at] = (cv[wave][e] - m) - log_s;
      }
    }
  } else {
    float pv = INFINITY;
    int pi = -1;
    for (found = 0; found < a.k; ++found) {   // the best behind (pv, pi)
      float bv = -INFINITY;
      int bi = INT_MAX;
#pragma unroll
      for (int j = NV * VN - 1; j >= 0; --j) {
        const int i = first(j / VN) + j % VN;
        if (before(pv, pi, v[j], i) && v[j] >= bv && v[j] != -INFINITY) {
          bv = v[j];
          bi = i;
        }
      }
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const float ov = __shfl_xor(bv, o, kWave);
        const int oi = __shfl_xor(bi, o, kWave);
        if (before(ov, oi, bv, bi)) {
          bv = ov;
          bi = oi;
        }
      }
      if (bi == INT_MAX) break;
      if (lane == 0) {
        a.topi[out + found] = bi;
        a.toplp[out + found] = (bv - m) - log_s;
      }
      pv = bv;
      pi = bi;
    }
  }
  for (int e = found + lane; e < a.k; e += kWave) {   // fewer logits above -inf than k
    a.topi[out + e] = INT_MAX;
    a.toplp[out + e] = -INFINITY;
  }
}

// Merges a row's parts: their statistics, and of their k best each the row's.
template <typename T>
__global__ __launch_bounds__(SCORE_THREADS) void logp_join_kernel(TokenLogpArgs a) {
  constexpr int NT = SCORE_THREADS;
  static_assert(SCORE_PARTS <= kWave && SCORE_PARTS % 4 == 0, "a part a lane");
  static_assert(SCORE_PARTS == 32 && SCORE_CAP >= 32 * 33 / 2, "what is left of the entries fits");
  // the parts' best, second, fourth, .. 32nd best values (-inf: none)
  __shared__ __attribute__((aligned(16))) float hv[6][SCORE_PARTS];
  __shared__ float least[6];
  __shared__ Candidates cand;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid % kWave;
  const int n = a.parts * a.k;
  const T* logits = static_cast<const T*>(a.logits) + (size_t)row * a.ld;
  int token = -1;
  T given{};
  if (tid < a.n_tok) token = a.tokens[(size_t)row * a.n_tok + tid];
  // thread t takes places t % 8, t % 8 + 8, .. of part t / 8
  static_assert(NT == 8 * SCORE_PARTS, "eight threads a part");
  const int own = tid / 8;
  float ev[4];
  int ei[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int place = tid % 8 + 8 * u;
    const bool in = own < a.parts && place < a.k;
    const size_t e = (size_t)row * n + (in ? own * a.k + place : 0);
    ev[u] = a.k > 8 * u ? a.part_v[e] : 0.f;
    ei[u] = a.k > 8 * u ? a.part_i[e] : INT_MAX;
    if (!in) ei[u] = INT_MAX;
  }
  // (levels but the first are of use where k (k + 1) / 2 entries are more than there are threads)
  const int level = tid / SCORE_PARTS, of = tid % SCORE_PARTS, levels = a.k * (a.k + 1) / 2 > NT ? 6 : 1;
  if (a.k > 0 && level < levels)
    hv[level][of] = of < a.parts && 1 << level <= a.k ? a.part_v[(size_t)row * n + of * a.k + (1 << level) - 1] : -INFINITY;
  if (a.k > 0) clear<NT>(cand);
  if ((unsigned)token < (unsigned)a.V) given = logits[token];   // looked at at the end
  Stats all{-INFINITY, 0.f, 0.f};
  if (lane < a.parts) {
    const float4 q = *reinterpret_cast<const float4*>(a.part_stats + ((size_t)row * a.parts + lane) * 4);
    all = Stats{q.x, q.y, q.z};
  }
  all = wave_stats(all, all.m);
  const float log_s = logf(all.s);
  if (tid == 0) {
    const bool none = all.s == 0.f;
    if (a.lse) a.lse[row] = none ? -INFINITY : all.m + log_s;
    if (a.entropy) a.entropy[row] = none ? 0.f : log_s - all.t / all.s;
  }
  auto put_given = [&] {
    for (int j = tid; j < a.n_tok; j += NT) {
      if (j >= NT) {
        token = a.tokens[(size_t)row * a.n_tok + j];
        if ((unsigned)token < (unsigned)a.V) given = logits[token];
      }
      const float x = to_f32(given), lp = x == -INFINITY && all.s == all.s ? -INFINITY : (x - all.m) - log_s;
      a.logp[(size_t)row * a.n_tok + j] = (unsigned)token < (unsigned)a.V ? lp : 0.f;
    }
  };
  if (a.k == 0) {
    put_given();
    return;
  }
  __syncthreads();
  // Where r parts' l-th best reach a value, r l entries do: the ceil(k / l)-th largest of the l-th bests
  // is no more than the k-th entry of all, for l = 1, 2, 4, ..  (64 rows of 50000, k = 32, in parts: 37 us
  // without it, 21 with.)
  float thr = -INFINITY;
  if (levels > 1) {
    if (level < levels) {
      const float own_v = hv[level][of];
      int above = 0;
#pragma unroll
      for (int j = 0; j < SCORE_PARTS; j += 4) {
        const float4 v = *reinterpret_cast<const float4*>(&hv[level][j]);
        above += (v.x > own_v) + (v.y > own_v) + (v.z > own_v) + (v.w > own_v);
      }
      float low = above << level < a.k ? -own_v : -INFINITY;   // (fewer than ceil(k / l) above it)
#pragma unroll
      for (int o = 1; o < SCORE_PARTS; o <<= 1) low = fmaxf(low, __shfl_xor(low, o, kWave));
      if (of == 0) least[level] = -low;
    }
    __syncthreads();
#pragma unroll
    for (int l = 0; l < 6; ++l) thr = fmaxf(thr, least[l]);
  }
  // An entry behind `place` of its own part and behind the best of h other parts (of equal values the
  // earlier part's) is behind place + h.  What reaches the threshold and is left of all parts' entries
  // where that is below k is a list of little more than k, with many equal values of a few k.
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (8 * u >= a.k) break;
    const int place = tid % 8 + 8 * u;
    int heads = 0;
#pragma unroll
    for (int j = 0; j < SCORE_PARTS; j += 4) {
      const float4 v = *reinterpret_cast<const float4*>(&hv[0][j]);
      heads += (j < own ? v.x >= ev[u] : v.x > ev[u]) + (j + 1 < own ? v.y >= ev[u] : v.y > ev[u]) +
               (j + 2 < own ? v.z >= ev[u] : v.z > ev[u]) + (j + 3 < own ? v.w >= ev[u] : v.w > ev[u]);
    }
    // (its own part's best, where that is above it, is one of the `place` already)
    if (ev[u] < hv[0][own]) --heads;
    if (ei[u] != INT_MAX && ev[u] >= thr && place + heads < a.k) put(cand, ev[u], ei[u]);
  }
  __syncthreads();
  const int found = cand.count;   // at most k + (k - 1) + .. + 1 of them
  for (int e = tid; e < found; e += NT) {
    const int at = rank_of(cand.v, cand.i, found, e);
    if (at < a.k) {
      a.topi[(size_t)row * a.k + at] = cand.i[e];
      a.toplp[(size_t)row * a.k + at] = (cand.v[e] - all.m) - log_s;
    }
  }
  for (int e = found + tid; e < a.k; e += NT) {   // fewer logits above -inf than k
    a.topi[(size_t)row * a.k + e] = INT_MAX;
    a.toplp[(size_t)row * a.k + e] = -INFINITY;
  }
  put_given();
}

// Many rows that are not long take two waves each instead of four: what a wave does besides its values
// is a third to a half of its work.  us four / two waves, k = 8: 8192 rows of 2100 bf16 values 40 / 26,
// of 8200 49 / 38, of 12000 57 / 47, of 20000 75 / 64 (k = 32: 94 / 95); of 4100 fp32 38 / 32, of 8200
// 52 / 52 (k = 32: 71 / 78); 1000 of 4100 bf16 8.5 / 7.6, of 8200 9.6 / 9.8; 100 of 4100 6.1 / 6.4.
template <typename T>
bool two_waves(const TokenLogpArgs& a) {
  const long long bytes = (long long)a.V * sizeof(T);
  return a.parts == 1 && a.rows >= 512 && bytes <= (a.rows >= 4096 ? 24 << 10 : 9 << 10);
}

// No more rows than CUs take sixteen each: more of a row under way, and more threads to share out the
// alternatives (us four / sixteen waves, fp32, k = 8: 1 row of 32000 8.0 / 7.7, 128 of 32000 10.0 / 9.2,
// 64 of 70000 13.7 / 11.9; k = 32: 128 of 32000 12.8 / 11.6; but 64 of 4100 6.3 / 6.8, 400 of 32000
// 14.0 / 17.7).
bool sixteen_waves(const TokenLogpArgs& a) { return a.parts == 1 && a.rows <= 256 && a.V >= 12000; }

template <typename T>
hipError_t logp_launch(const TokenLogpArgs& a, hipStream_t s) {
  if (a.V <= SHORT) {
    const dim3 grid((unsigned)((a.rows + 3) / 4));
    if (a.V >= VEC_FROM) NT_LAUNCH((short_logp_kernel<T, true>), grid, dim3(256), 0, s, a);
    else NT_LAUNCH((short_logp_kernel<T, false>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (two_waves<T>(a)) {
    NT_LAUNCH((token_logp_kernel<T, 128>), dim3((unsigned)a.rows), dim3(128), 0, s, a);
    return hipGetLastError();
  }
  if (sixteen_waves(a)) {
    NT_LAUNCH((token_logp_kernel<T, 1024>), dim3((unsigned)a.rows), dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  NT_LAUNCH((token_logp_kernel<T, SCORE_THREADS>), dim3((unsigned)(a.rows * a.parts)), dim3(SCORE_THREADS), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  NT_LAUNCH((logp_join_kernel<T>), dim3((unsigned)a.rows), dim3(SCORE_THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace

// Whether a row is one workgroup's or cut into parts, which cost a second launch and a selection each: cut
// where its time (as of 7 bytes a fp32 value and 5 a 16-bit one) is past a bound that grows
// with the rows, which occupy the GPU too, and doubles with the largest k.  Measured, us whole / cut:
// fp32, k = 8: 1 row of 32000 7.7 / 9.5, of 70000 9.8 / 9.2, of 131072 12.6 / 9.3; 64 of 70000
// 11.9 / 14.2, of 131072 16.9 / 15.2; 128 of 131072 19.5 / 20.4, of 300000 35.6 / 33.5; 256 of 300000
// 53 / 57; bf16: 2 of 70000 9.9 / 9.6, 64 of 131072 13.8 / 13.5; k = 32, fp32: 1 of 131072 14.8 / 15.2,
// 64 of 131072 19.0 / 24.2, of 300000 33.6 / 31.6.
// No more than 1024 workgroups come of it.
void token_logp_plan(DT dt, TokenLogpArgs* a) {
  const long long row_bytes = (long long)a->V * dt_bytes(dt), rows = a->rows;
  const long long bound = (444 + 5 * rows + rows * rows / 128) << (a->k > 20 ? 11 : 10);
  long long parts = 1;
  if (rows > 0 && row_bytes + 3ll * a->V >= bound)
    parts = std::max(1ll, std::min<long long>({1024 / rows, row_bytes / 8192, SCORE_PARTS}));
  a->part_len = (int)((a->V + parts - 1) / parts);
  a->parts = (a->V + a->part_len - 1) / a->part_len;
}

hipError_t token_logp(DT dt, const TokenLogpArgs& a, hipStream_t s) {
  if (a.rows <= 0) return hipSuccess;
  switch (dt) {
    case DT::F32: return logp_launch<float>(a, s);
    case DT::F16: return logp_launch<f16>(a, s);
    case DT::BF16: return logp_launch<bf16>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace nt
