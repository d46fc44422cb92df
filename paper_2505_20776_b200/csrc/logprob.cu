// Log probabilities under rows of logits: of given tokens, of the k best words, and the row's entropy.  With x = logits /
// temperature, m its maximum, Z = sum e^(x - m) and E = sum e^(x - m) (x - m):
//   lse = m + log Z,  log p(w) = (x_w - m) - log Z,  entropy = -sum p log p = log Z - E / Z.
// One pass over the logits with running m, Z and E in fp32 (a thread's 16 or 32 words of a turn share one rescaling); a row is
// split over the CTAs of a cluster where rows are few, and joined in the first CTA's shared memory.
//
// Where one word has nearly all of the probability, what is left to the others decides the results: with r = Z - 1, the sum of all
// words but the best, log Z = log1p(r), the best word's log probability is -log1p(r), the entropy log1p(r) - E / (1 + r), all terms of
// one sign, so that nothing cancels and no log probability is above 0, no entropy below.  So partial results are joined without their
// best word (1 and 0 to Z and E, exactly).  Only the thread that has the row's best word gets its part of r by a difference,
// Z - 1, which is off by some 2^-22; where r is below 1/2 the CTA sums that thread's words again without the best one.  (us per call,
// replayed, before / with it: one row of 32000 bf16 5.3 / 5.6, 60 of 128256 10.6 / 11.1, 2047 of 32000 fp32 53.0 / 53.9; the sum out of line,
// in a function of its own, 55.6 for the last.)
//
// The best words are found without sorting: a word's key is (logit, lower index first).  Every thread knows its own best key
// after the pass (up to its place in a vector); the k-th best of the warps' j best thread keys (j times the number of warps >= k)
// bounds the k-th best key of the CTA from below, so only threads with a key that good are looked at again: the turn of the
// loop that had their best, or all their vectors where another turn has a logit that good.  All of it is dealt to all threads (when
// each such thread looked through its own, with the rest of its warp waiting, that took longer than the pass), and the few
// words above the bound are put in order by counting.  Words that are too many for the list (values
// arranged so that one thread has them all) are taken out one by one.
//
// What bounds it: reading the logits (HBM), the exponentials (16 a cycle and SM) close behind for bf16; for few rows the chain of
// latencies: load, reduction, second look, join.
#include "common.cuh"
#include "pair.cuh"

using namespace sm100;
using namespace pair;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kNextRow = 32768;
constexpr int kMaxBest = 32, kMaxSlices = 8, kList = 512;
constexpr float kLn2 = 0.693147180559945309417f;
typedef unsigned long long Key;                 // 0: none

struct LogprobArgs {
  const void* logits;
  const int32_t* tokens;
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t *top_ids, *status;
  long long stride;
  int V, given, best, slices, resident;
  float inv_temperature, c;                     // c = log2 e / temperature, rounded once
};

__device__ __forceinline__ uint32_t ordered(float x) {         // no NaN; -0 counts as 0
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ Key make_key(float x, int idx) { return ((Key)ordered(x) << 32) | (uint32_t)~idx; }

// A row as 16-byte vectors: vector v holds words v * kWords - skew + (0 .. kWords - 1); the first and last one may reach outside.
template <bool F32>
struct Row {
  static constexpr int kWords = F32 ? 4 : 8;
  const char* base;                             // of the row, at most 15 bytes below its first word
  int skew, V, n_vec;
  __device__ __forceinline__ Row(const LogprobArgs& a, int row) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.logits) + (unsigned long long)(row * a.stride) * (F32 ? 4 : 2);
    base = reinterpret_cast<const char*>(at & ~(uintptr_t)15);
    skew = (int)(at & 15) / (F32 ? 4 : 2);
    V = a.V;
    n_vec = (int)(((long long)V + skew + kWords - 1) / kWords);
  }
  __device__ __forceinline__ float word(int idx) const {
    const char* at = base + (long long)(idx + skew) * (F32 ? 4 : 2);
    return F32 ? *reinterpret_cast<const float*>(at) : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16);
  }
  __device__ __forceinline__ int first_word(int v) const { return v * kWords - skew; }
  __device__ __forceinline__ int whole() const { return (V + skew) / kWords; }           // vectors up to the last whole one
};

// Vector v of the row; words outside are -inf.
template <bool F32>
__device__ __forceinline__ uint4 load_vec(const Row<F32>& row, int v) {
  constexpr int W = Row<F32>::kWords;
  const int w0 = row.first_word(v);
  if (w0 >= 0 && w0 <= row.V - W) return *reinterpret_cast<const uint4*>(row.base + (long long)v * 16);
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      q[i] = w0 + i >= 0 && w0 + i < row.V ? __float_as_uint(row.word(w0 + i)) : 0xff800000u;
    } else {
      const int w = w0 + 2 * i;
      q[i] = (w >= 0 && w < row.V ? __float_as_uint(row.word(w)) >> 16 : 0xff80u) |
             (w + 1 >= 0 && w + 1 < row.V ? __float_as_uint(row.word(w + 1)) & 0xffff0000u : 0xff800000u);
    }
  }
  return make_uint4(q[0], q[1], q[2], q[3]);
}
template <bool F32>
__device__ __forceinline__ void unpack(uint4 r, float (&x)[Row<F32>::kWords]) {
  const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < Row<F32>::kWords; ++j)
    x[j] = F32 ? __uint_as_float(q[j % 4]) : __uint_as_float(j & 1 ? q[j / 2 % 4] & 0xffff0000u : q[j / 2 % 4] << 16);
}

template <bool F32>
__device__ __forceinline__ uint4 none() {                       // words of -inf
  constexpr uint32_t q = F32 ? 0xff800000u : 0xff80ff80u;
  return make_uint4(q, q, q, q);
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {           // (of a number and NaN: the number)
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// The largest word of a vector.
template <bool F32>
__device__ __forceinline__ float largest(uint4 r) {
  if constexpr (F32) {
    return fmaxf(fmax3(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z)), __uint_as_float(r.w));
  } else {
    const uint32_t m = max_bf16x2(max_bf16x2(r.x, r.y), max_bf16x2(r.z, r.w));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
}
// bf16 words below about -1e30 become that (NaN stays).
__device__ __forceinline__ uint4 at_least_lowest(uint4 r) {
  auto lift = [](uint32_t w) {
    uint32_t q;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(q) : "r"(w), "r"(0xf14af14au));
    return q;
  };
  return make_uint4(lift(r.x), lift(r.y), lift(r.z), lift(r.w));
}

// Statistics of some words relative to m, their largest logit or one at most kSlack below it: with t(x) = x c - m c (c: log2 e /
// temperature), z the sum of 2^t, e that of 2^t t.  m c is rounded once, and every use rounds it alike, so that it takes no part in
// the error.  Where that rounding itself would be large (a row of nothing but masks, which may be the type's lowest value),
// t is (x - m) c.
struct Stat {
  float m, z, e;
};
struct Scale {
  float c, plain, slack;                        // log2 e / temperature; m below this in magnitude: t is x c - m c; kSlack in logits
};
constexpr float kSlack = 4.f;                   // in powers of two
constexpr float kLarge = 1048576.f;             // of m c: its rounding is 2^-5 and less
// (temperatures far from any use have every word taken as (x - m) c)
__device__ __forceinline__ Scale scale_of(float c) {
  const bool usual = c > 1e-20f && c < 1e6f;
  return {c, usual ? kLarge / c : 0.f, usual ? kSlack / c : 0.f};
}
// `s` relative to a new reference m >= s.m (of one thread, in the pass).
__device__ __forceinline__ Stat at_maximum(Stat s, float m, const Scale& sc) {
  const bool plain = fabsf(m) < sc.plain, was = fabsf(s.m) < sc.plain;
  const float to = __fmul_rn(m, sc.c), from = __fmul_rn(s.m, sc.c);
  const float d = plain ? (was ? __fsub_rn(from, to) : fmaf(s.m, sc.c, -to)) : was ? -fmaf(m, sc.c, -from) : (s.m - m) * sc.c;
  const float f = ex2_approx(d);
  // (z = 0: no word, or none but -inf; f = 0: nothing is left of it, whatever d is)
  if (s.z == 0.f) return {m, 0.f, 0.f};
  return {m, s.z * f, f == 0.f ? 0.f : f * fmaf(d, s.z, s.e)};
}
// ... and relative to the logit m itself: t is (x - m) c from here on, without the rounding of m c.
__device__ __forceinline__ Stat relative_to(Stat s, float m, const Scale& sc) {
  const float d = fabsf(s.m) < sc.plain ? -fmaf(m, sc.c, -__fmul_rn(s.m, sc.c)) : (s.m - m) * sc.c;
  const float f = ex2_approx(d);
  if (s.z == 0.f) return {m, 0.f, 0.f};
  return {m, s.z * f, f == 0.f ? 0.f : f * fmaf(d, s.z, s.e)};
}
// (x - m) c, for any words x <= m.
struct Difference {
  float m, c, to, off;                          // m c, and what it was rounded by
  bool plain;
  __device__ __forceinline__ float operator()(float x) const { return plain ? fmaf(x, c, -to) - off : (x - m) * c; }
};
__device__ __forceinline__ Difference difference_to(float m, const Scale& sc) {
  const float to = __fmul_rn(m, sc.c);
  return {m, sc.c, to, fmaf(m, sc.c, -to), fabsf(m) < sc.plain};
}
// What the thread with a warp's best word has beside that word, and which thread it is (-1: none but -inf and NaN).
struct Own {
  float z, e;
  int tid;
};
// The joint statistics of stats[0 .. n), n <= 8, by every warp for itself: a lane has one of them.  z and e are without the best
// word, of what goes in and of what comes out; of stats with parts of their own, `own` is that of the best, which the result leaves out.
template <bool OWN>
__device__ __forceinline__ Stat join(const Stat* stats, int n, const Scale& sc, const Own* owns, Own* own) {
  const int i = threadIdx.x & 7;
  Stat s = {-INFINITY, 0.f, 0.f};
  Own mine = {0.f, 0.f, -1};
  if (i < n) {
    s = stats[i];
    if (OWN) mine = owns[i];
  }
  float m = s.m;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bool some = s.m > -INFINITY;
  const int best = __ffs(__ballot_sync(0xffffffffu, some && s.m == m)) - 1;
  if (i != best) {
    s.z += mine.z;
    s.e += mine.e;
    if (some) {
      const float d = difference_to(m, sc)(s.m), f = ex2_approx(d), z = s.z + 1.f;
      s.z = z * f;
      s.e = f == 0.f ? 0.f : f * fmaf(d, z, s.e);
    }
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    s.z += __shfl_xor_sync(0xffffffffu, s.z, o);
    s.e += __shfl_xor_sync(0xffffffffu, s.e, o);
  }
  s.m = m;
  if (OWN) *own = best >= 0 ? owns[best] : Own{0.f, 0.f, -1};
  return s;
}
static_assert(kWarps <= 8 && kMaxSlices <= 8, "join has 8 lanes");

struct Shared {
  Stat warp_stat[kWarps];
  Own warp_own[kWarps];
  float2 again_sum;                             // z and e of the best word's thread, summed again
  Key bounds[kWarps * kMaxBest];                // the warps' best thread keys
  Key list[kList];
  Key top[kMaxBest];
  int n_list, n_again;
  int again[kThreads];                          // what is looked at again: a turn's first vector, or -1 - thread: all its vectors
  // in the first CTA of a cluster, from all of it
  Stat stat[kMaxSlices];
  Key keys[kMaxSlices * kMaxBest];
  uint64_t arrived;
  int abort_flag;
};

__device__ __forceinline__ Key warp_max_key(Key k) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  return ((Key)hi << 32) | lo;
}

// Places of keys[i], i < n, in descending order, counted by the threads of the CTA: put(place, key).  Zero keys are left out.
template <class Put>
__device__ __forceinline__ void in_order(const Key* keys, int n, Put&& put) {
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const Key mine = keys[i];
    int place = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) place += keys[j] > mine ? 1 : 0;
    if (mine != 0) put(place, mine);
  }
}

// `n` vectors from v on to L2, as far as they lie before `end`.
template <bool F32>
__device__ __forceinline__ void prefetch_l2(const Row<F32>& row, int v, int n, int end) {
  n = min(n, end - v);
  if (n > 0)
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row.base + (long long)v * 16), "r"(n * 16) : "memory");
}

// use(key) for every word of vector v (NaN has none).
template <bool F32, class Use>
__device__ __forceinline__ void each_key(const Row<F32>& row, int v, Use&& use) {
  constexpr int W = Row<F32>::kWords;
  float x[W];
  unpack<F32>(load_vec(row, v), x);
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const int idx = row.first_word(v) + j;
    if (x[j] == x[j] && idx >= 0 && idx < row.V) use(make_key(x[j], idx));
  }
}

// The `best` best keys of the words in vectors [lo, hi) to sh.top, in order (zeros where there are no more words).  `mine`: no word
// of the thread has a better key; `full` warps had a vector for every thread, and their best thread keys are in sh.bounds.
// `meanwhile`: done beside the second look, which the first warps have.
template <bool F32, class Meanwhile>
__device__ __forceinline__ void best_words(Shared& sh, const Row<F32>& row, int lo, int hi, int best, Key mine, int turn, int n_turn, Key rest, int full,
                                           Meanwhile&& meanwhile) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // The bound: of the warps' best thread keys (j of each, at least k in all) the k-th best; or the lowest, where they are too many
  // for a warp to look at.
  const int j = full > 0 ? (best + full - 1) / full : 0, n_bounds = j * full;
  Key bound = 0;
  if (n_bounds > 0 && n_bounds <= 32) {
    const Key k = lane < n_bounds ? sh.bounds[lane] : 0;
    int place = 0;
#pragma unroll 4
    for (int i = 0; i < n_bounds; ++i) place += sh.bounds[i] > k ? 1 : 0;
    // (a zero key: a thread that has none but NaN; then the bound is none)
    const unsigned who = __ballot_sync(0xffffffffu, lane < n_bounds && place == best - 1);
    bound = who ? __shfl_sync(0xffffffffu, k, __ffs(who) - 1) : 0;
  } else if (n_bounds > 0) {
    bound = sh.bounds[j - 1];
    for (int i = 1; i < full; ++i) bound = min(bound, sh.bounds[i * j + j - 1]);
  }
  if (mine != 0 && mine >= bound) sh.again[atomicAdd(&sh.n_again, 1)] = rest >= bound ? -1 - tid : turn;
  __syncthreads();
  const int n_again = sh.n_again, member = tid & 7;        // 8 threads to each
  for (int q = tid >> 3; q < n_again; q += kThreads >> 3) {
    const int what = sh.again[q], first = what < 0 ? lo - 1 - what : what, end = what < 0 ? hi : min(hi, first + n_turn);
    for (int v = first + member * kThreads; v < end; v += 8 * kThreads)
      each_key(row, v, [&](Key k) {
        if (k >= bound) {
          const int at = atomicAdd(&sh.n_list, 1);
          if (at < kList) sh.list[at] = k;
        }
      });
  }
  meanwhile();
  __syncthreads();
  const int n = sh.n_list;
  if (n <= kList) {
    in_order(sh.list, n, [&](int place, Key k) {
      if (place < best) sh.top[place] = k;
    });
  } else {
    Key before = ~0ull;
#pragma unroll 1
    for (int r = 0; r < best; ++r) {
      Key k = 0;
      for (int v = lo + tid; v < hi; v += kThreads)
        each_key(row, v, [&](Key q) {
          if (q < before && q > k) k = q;
        });
      k = warp_max_key(k);
      __syncthreads();                          // (the round before has been read)
      if (lane == 0) sh.list[warp] = k;
      __syncthreads();
      for (int i = 0; i < kWarps; ++i) k = max(k, sh.list[i]);
      if (tid == 0) sh.top[r] = k;
      before = k;
    }
  }
  __syncthreads();
}

// AHEAD: more rows than CTAs at once, so that reading is what counts: two turns ahead go to L2, and the next row's beginning while this
// one's words are put in order.  us per call, replayed, with / without: 2047 rows of 32000 fp32 52.4 / 57.4, bf16 40.2 / 44.7, 1500 of
// 128256 bf16 84.5 / 94; before rows that one word dominates were summed again, 200 of 32000 fp32 13.2 / 11.2, 500 of 128256 bf16 38 / 36.9 (128
// threads and twice the CTAs: 56.9 and 39.4 where it was 53.3 and 38).
template <bool F32, bool AHEAD>
__global__ void __launch_bounds__(kThreads, 4) logprob_kernel(const __grid_constant__ LogprobArgs a) {
  constexpr int W = Row<F32>::kWords;
  constexpr int kVecs = F32 || AHEAD ? 4 : 2;   // 16-byte loads of a thread at once, and as many for the next turn
  constexpr int kTurn = kVecs * kThreads;
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_slices = a.slices, r = (int)blockIdx.x / n_slices, rank = (int)blockIdx.x - r * n_slices;
  if (tid < kMaxBest) sh.top[tid] = 0;
  if (tid == 0) {
    sh.n_list = sh.n_again = 0;
    if (n_slices > 1) {
      sh.abort_flag = 0;
      mbar_init(&sh.arrived, 1);
      fence_mbar_init();
      if (rank == 0) mbar_arrive_expect_tx(&sh.arrived, n_slices * (a.best * 8 + 12));
    }
  }
  if (n_slices > 1) {
    __syncwarp();
    cluster_arrive();                           // (waited for before the first write to another CTA)
  }
  pdl_launch_dependents();
  const Row<F32> row(a, r);
  const int per = (row.n_vec + n_slices - 1) / n_slices;
  const int lo = min(row.n_vec, rank * per), hi = min(row.n_vec, lo + per);
  const Scale sc = scale_of(a.c);
  pdl_wait();
  // the first given tokens' logits, ahead of the pass
  int token = -1;
  float given = -INFINITY;
  if (rank == 0 && tid < a.given) {
    token = a.tokens[(long long)r * a.given + tid];
    if (token >= 0 && token < a.V) given = row.word(token);
  }

  // Of a thread: its best logit, the first vector that has it, and the best logit of the other turns of its loop.
  Stat s = {-INFINITY, 0.f, 0.f};
  float top_value = -INFINITY, other = -INFINITY;
  int top_v = lo + tid;
  uint4 next[kVecs];
  const int in_lo = max(lo, row.skew > 0 ? 1 : 0), in_hi = min(hi, row.whole());        // vectors without words outside
  auto fetch = [&](int v) {
    if (v >= in_lo && v + (kVecs - 1) * kThreads < in_hi) {
      const uint4* at = reinterpret_cast<const uint4*>(row.base) + v;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) next[i] = at[i * kThreads];
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        next[i] = v + i * kThreads < hi ? load_vec(row, v + i * kThreads) : none<F32>();
    }
  };
  fetch(lo + tid);
  if (AHEAD && tid == 0) prefetch_l2(row, lo + kTurn, kTurn, in_hi);
  const uint64_t c2 = pack_f32x2(sc.c, sc.c);
  for (int v = lo + tid; v < hi; v += kTurn) {
    uint4 raw[kVecs];
    float x[kVecs][W], vm[kVecs], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) raw[i] = next[i];
    if (v + kTurn < hi) fetch(v + kTurn);
    if (AHEAD && tid == 0) prefetch_l2(row, v + 2 * kTurn, kTurn, in_hi);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      vm[i] = largest<F32>(raw[i]);
      m = fmaxf(m, vm[i]);
    }
    other = fmaxf(other, fminf(m, top_value));
    if (m > top_value) {
      top_value = m;
      top_v = v;
#pragma unroll
      for (int i = kVecs - 1; i > 0; --i)
        if (vm[i] == m && vm[0] != m) top_v = v + i * kThreads;
    }
    // a new reference only where the sums would grow large: a maximum that only just rises is most turns' case for some thread of a warp
    if (m > s.m + sc.slack) s = at_maximum(s, m, sc);
    const float ref = s.m == -INFINITY ? 0.f : s.m;       // (nothing but -inf and NaN so far)
    if (fabsf(ref) < sc.plain) {
      const float neg = -__fmul_rn(ref, sc.c);
      const uint64_t neg2 = pack_f32x2(neg, neg);
      uint64_t z = 0ull, e = 0ull;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        // (a word masked out: 0 times a large number, not times infinity)
        unpack<F32>(F32 ? raw[i] : at_least_lowest(raw[i]), x[i]);
#pragma unroll
        for (int j = 0; j < W; j += 2) {
          float t0, t1;
          unpack_f32x2(fma_f32x2(pack_f32x2(x[i][j], x[i][j + 1]), c2, neg2), t0, t1);
          const uint64_t q = pack_f32x2(ex2_approx(t0), ex2_approx(t1));
          z = add_f32x2(z, q);
          e = fma_f32x2(q, F32 ? pack_f32x2(fmaxf(t0, -1e30f), fmaxf(t1, -1e30f)) : pack_f32x2(t0, t1), e);
        }
      }
      float z0, z1, e0, e1;
      unpack_f32x2(z, z0, z1);
      unpack_f32x2(e, e0, e1);
      s.z += z0 + z1;
      s.e += e0 + e1;
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        unpack<F32>(raw[i], x[i]);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float t = (x[i][j] - ref) * sc.c, q = ex2_approx(t);
          s.z += q;
          s.e = fmaf(q, fmaxf(t, -1e30f), s.e);
        }
      }
    }
  }

  // the beginning of the row that this place on the SM will most likely have next, while nothing else is read
  if (AHEAD && tid == 0 && blockIdx.x + a.resident < gridDim.x) {
    const Row<F32> later(a, blockIdx.x + a.resident);
    prefetch_l2(later, 0, kNextRow / 16, later.whole());
  }
  // warp: statistics, and the j-th best of its threads' best keys
  float m = top_value;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  s = relative_to(s, m, sc);
  const int best_lane = __ffs(__ballot_sync(0xffffffffu, top_value == m && m > -INFINITY)) - 1;
  if (lane == best_lane) sh.warp_own[warp] = {s.z - 1.f, s.e, tid};
  if (best_lane < 0 && lane == 0) sh.warp_own[warp] = {0.f, 0.f, -1};
  if (lane == best_lane) s.z = s.e = 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s.z += __shfl_xor_sync(0xffffffffu, s.z, o);
    s.e += __shfl_xor_sync(0xffffffffu, s.e, o);
  }
  if (lane == 0) sh.warp_stat[warp] = s;
  const int full = min(kWarps, (hi - lo) / 32);           // warps with a vector for every thread
  Key mine = 0;
  if (a.best > 0) {
    // its best word is one of vector top_v: at least as good as `k` below, at most as good as `mine`
    if (top_v < hi) mine = make_key(top_value, max(row.first_word(top_v), 0));
    if (warp < full) {
      Key k = top_v < hi ? make_key(top_value, row.first_word(top_v) + W - 1) : 0;
      const int j = (a.best + full - 1) / full;
#pragma unroll 1
      for (int i = 0; i < j; ++i) {
        const Key top = warp_max_key(k);
        if (lane == 0) sh.bounds[warp * j + i] = top;
        if (k == top) k = 0;
      }
    }
  }
  __syncthreads();
  Own own;
  s = join<true>(sh.warp_stat, kWarps, sc, sh.warp_own, &own);
  // The best word is nearly all there is: its thread's other words (an equal word would weigh 1, so none is there), by the last warp.
  const bool again = own.tid >= 0 && s.z + own.z < 0.5f;
  const bool summing = again && warp == kWarps - 1;
  int v_again = lo + own.tid + lane * kThreads;
  uint4 raw_again = none<F32>();
  if (summing && v_again < hi) raw_again = load_vec(row, v_again);            // (on its way while the best words are looked for)
  auto sum_again = [&]() {
    if (!summing) return;
    const Difference diff = difference_to(s.m, sc);
    float z = 0.f, e = 0.f;
#pragma unroll 1
    while (true) {
      float x[W];
      unpack<F32>(raw_again, x);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float t = diff(x[j]), q = x[j] == s.m ? 0.f : ex2_approx(t);
        z += q;
        e = fmaf(q, fmaxf(t, -1e30f), e);
      }
      v_again += 32 * kThreads;
      if (v_again >= hi) break;
      raw_again = load_vec(row, v_again);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      z += __shfl_xor_sync(0xffffffffu, z, o);
      e += __shfl_xor_sync(0xffffffffu, e, o);
    }
    if (lane == 0) sh.again_sum = make_float2(z, e);
  };
  if (a.best > 0) {
    const int turn = lo + tid + (top_v - lo - tid) / kTurn * kTurn;
    best_words(sh, row, lo, hi, a.best, mine, turn, kTurn, make_key(other, 0), full, sum_again);
  } else {
    sum_again();
    __syncthreads();
  }
  if (again) {
    own.z = sh.again_sum.x;
    own.e = sh.again_sum.y;
  }
  s.z += own.z;
  s.e += own.e;

  const Key* keys = sh.top;
  int n_keys = a.best;
  if (n_slices > 1) {
    cluster_wait();                             // every CTA of the cluster has started
    const uint32_t bar = map_to_cta(smem_u32(&sh.arrived), 0);
    if (tid < a.best) {
      const uint32_t at = map_to_cta(smem_u32(&sh.keys[rank * a.best + tid]), 0);
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(at), "l"(sh.top[tid]), "r"(bar)
                   : "memory");
    }
    if (tid >= kThreads - 3) {
      const int i = tid - (kThreads - 3);
      const uint32_t at = map_to_cta(smem_u32(&sh.stat[rank]) + 4 * i, 0);
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(at),
                   "r"(__float_as_uint(i == 0 ? s.m : i == 1 ? s.z : s.e)), "r"(bar)
                   : "memory");
    }
    if (rank != 0) return;
    if (!mbar_wait(&sh.arrived, 0, &sh.abort_flag)) {
      if (lane == 0) spx_raise(a.status, SPECEXT_ERR_TIMEOUT);
      settle();
      return;
    }
    s = join<false>(sh.stat, n_slices, sc, nullptr, nullptr);
    keys = sh.keys;
    n_keys = n_slices * a.best;
  }

  // a row without a finite logit: all its log probabilities are -inf, and its entropy is 0
  const bool empty = s.m == -INFINITY && s.z == 0.f;
  const float log_z = log1pf(s.z), lse = empty ? -INFINITY : fmaf(s.m, a.inv_temperature, log_z);
  // (the difference to the maximum first: x - lse would lose log Z where the maximum is huge, as in a row of the type's lowest value)
  auto log_p = [&](float raw) { return empty ? -INFINITY : fmaf(raw - s.m, a.inv_temperature, -log_z); };
  if (tid == 0) {
    a.lse[r] = lse;
    a.entropy[r] = empty ? 0.f : log_z - s.e / (1.f + s.z) * kLn2;
  }
  for (int i = tid; i < a.given; i += kThreads) {
    const long long at = (long long)r * a.given + i;
    if (i >= kThreads) {
      token = a.tokens[at];
      given = token >= 0 && token < a.V ? row.word(token) : -INFINITY;
    }
    const bool known = token >= 0 && token < a.V;
    a.logprob[at] = known ? log_p(given) : -INFINITY;                          // -1: no token
    if (!known && token != -1) spx_raise(a.status, SPECEXT_ERR_INVALID_ARG);
  }
  const bool bad = !(s.z == s.z);               // a NaN or +inf among the logits: no order
  in_order(keys, n_keys, [&](int place, Key k) {
    if (place < a.best && !bad) {
      const long long at = (long long)r * a.best + place;
      a.top_ids[at] = (int32_t)~(uint32_t)k;
      a.top_logprob[at] = log_p(unordered((uint32_t)(k >> 32)));
    }
  });
  if (bad && tid < a.best) {
    const long long at = (long long)r * a.best + tid;
    a.top_ids[at] = -1;
    a.top_logprob[at] = __uint_as_float(0x7fc00000u);
  }
}

template <bool F32, bool AHEAD>
cudaError_t launch(const LogprobArgs& a, int rows, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * (unsigned)a.slices);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.slices;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.slices > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<F32, AHEAD>, a);
}

}  // namespace

cudaError_t spx_launch_logprobs(const void* logits, bool f32, int rows, int V, long long stride, float temperature,
                                const int32_t* tokens, int given, int best, float* logprob, float* entropy, float* lse,
                                int32_t* top_ids, float* top_logprob, int n_sm, int32_t* status, cudaStream_t st) {
  LogprobArgs a;
  a.logits = logits; a.tokens = tokens;
  a.logprob = logprob; a.entropy = entropy; a.lse = lse; a.top_ids = top_ids; a.top_logprob = top_logprob; a.status = status;
  a.stride = stride; a.V = V; a.given = given; a.best = best;
  a.inv_temperature = 1.f / temperature;
  a.c = (float)(1.4426950408889634074 / (double)temperature);
  // CTAs per row: as many as are resident at once (four per SM), as long as a thread has two vectors and more.  us per call, 1 / 2 /
  // 4 / 8, replayed: one row of 32000 bf16 6.9 / 6.1 / 5.6 / 5.5 (at most 4 by this rule), 16 of 128256 27.2 / 16.0 / 10.6 / 9.0, 60 of
  // 128256 27.9 / 16.8 / 13.9 / 11.2, 200 of 32000 fp32 12.3 / 11.0 (2 by this rule; 4 and 8 were 15.3 and 22.9)
  const int words = f32 ? 4 : 8;
  int slices = 1;
  while (slices < kMaxSlices && 2ll * rows * slices <= 4ll * n_sm && V / words >= 2 * slices * 2 * kThreads) slices *= 2;
  a.slices = slices;
  a.resident = 4 * n_sm;
  if (slices == 1 && rows > a.resident) return f32 ? launch<true, true>(a, rows, st) : launch<false, true>(a, rows, st);
  return f32 ? launch<true, false>(a, rows, st) : launch<false, false>(a, rows, st);
}
