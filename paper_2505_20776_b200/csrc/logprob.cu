// Log probabilities under rows of logits: of given tokens, of the k best words, and the row's entropy.  With x = logits /
// temperature, m its maximum, Z = sum e^(x - m) and E = sum e^(x - m) (x - m):
//   lse = m + log Z,  log p(w) = (x_w - m) - log Z,  entropy = -sum p log p = log Z - E / Z.
// One pass over the logits with running m, Z and E in fp32 (32 words share one rescaling); a row is split over the CTAs of a
// cluster where rows are few, and joined in the first CTA's shared memory.
//
// The best words are found without sorting: a word's key is (logit, lower index first).  Every thread knows its own best key
// after the pass; the lowest of the j-th best thread keys of the warps, with j times the number of warps >= k, bounds the k-th
// best key of the CTA from below, so only threads with a key that good look at their words again (from L2), and the few words
// above the bound are put in order by counting.  Words that are too many for the list (values arranged so that one thread has
// them all) are taken out one by one.
//
// What bounds it: reading the logits (HBM), the exponentials (16 a cycle and SM) close behind for bf16; for few rows the chain of
// latencies: load, reduction, second look, join.
#include "common.cuh"
#include "pair.cuh"

using namespace sm100;
using namespace pair;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kVecs = 4;                        // 16-byte loads of a thread in flight
constexpr int kMaxBest = 32, kMaxSlices = 8, kList = 512;
constexpr float kLn2 = 0.693147180559945309417f, kLog2e = 1.44269504088896340736f;
typedef unsigned long long Key;                 // 0: none

struct LogprobArgs {
  const void* logits;
  const int32_t* tokens;
  float *logprob, *entropy, *lse, *top_logprob;
  int32_t *top_ids, *status;
  long long stride;
  int V, given, best, slices;
  float inv_temperature;
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
};

// kVecs vectors v, v + kThreads, ... below `end` as floats; words outside are -inf.
template <bool F32>
__device__ __forceinline__ void load_chunk(const Row<F32>& row, int v, int end, float (&x)[kVecs][Row<F32>::kWords]) {
  constexpr int W = Row<F32>::kWords;
  uint4 r[kVecs];
  bool whole[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int u = v + i * kThreads, w0 = row.first_word(u);
    whole[i] = u < end && w0 >= 0 && w0 <= row.V - W;
    if (whole[i]) r[i] = *reinterpret_cast<const uint4*>(row.base + (long long)u * 16);
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int u = v + i * kThreads, w0 = row.first_word(u);
    if (whole[i]) {
      const uint32_t q[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
      for (int j = 0; j < W; ++j)
        x[i][j] = F32 ? __uint_as_float(q[j % 4]) : __uint_as_float(j & 1 ? q[j / 2 % 4] & 0xffff0000u : q[j / 2 % 4] << 16);
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) x[i][j] = u < end && w0 + j >= 0 && w0 + j < row.V ? row.word(w0 + j) : -INFINITY;
    }
  }
}

struct Stat {
  float m, z, e;                                // of raw logits: e is the sum of e^((raw - m) / temperature) (raw - m)
};
__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float m = fmaxf(a.m, b.m);
  Stat r = {m, 0.f, 0.f};
  if (a.z != 0.f) {                             // (also a NaN)
    const float d = a.m - m, f = ex2_approx(d * c);
    r.z = a.z * f;
    r.e = f == 0.f ? 0.f : f * fmaf(d, a.z, a.e);
  }
  if (b.z != 0.f) {
    const float d = b.m - m, f = ex2_approx(d * c);
    r.z = fmaf(b.z, f, r.z);
    r.e += f == 0.f ? 0.f : f * fmaf(d, b.z, b.e);
  }
  return r;
}

struct Shared {
  Stat warp_stat[kWarps];
  Key warp_bound[kWarps];
  Key list[kList];
  Key top[kMaxBest];
  int n_list;
  Stat stat[kMaxSlices];                        // in the first CTA, from all of the cluster
  Key keys[kMaxSlices][kMaxBest];
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
    for (int j = 0; j < n; ++j) place += keys[j] > mine ? 1 : 0;
    if (mine != 0) put(place, mine);
  }
}

// The `best` best keys of the words in vectors [lo, hi) to sh.top, in order (zeros where there are no more words).
template <bool F32>
__device__ __forceinline__ void best_words(Shared& sh, const Row<F32>& row, int lo, int hi, int best, float top_value, int top_v) {
  constexpr int W = Row<F32>::kWords;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  Key mine = 0;
  if (top_v >= 0) {
    float x[kVecs][W];
    load_chunk(row, top_v, hi, x);
#pragma unroll
    for (int i = kVecs - 1; i >= 0; --i)
#pragma unroll
      for (int j = W - 1; j >= 0; --j) {
        const int idx = row.first_word(top_v + i * kThreads) + j;
        if (x[i][j] == top_value && top_v + i * kThreads < hi && idx >= 0 && idx < row.V) mine = make_key(x[i][j], idx);
      }
  }
  // the bound: whole warps of threads with a key, j-th best of each
  const int full = min(kWarps, (hi - lo) / 32);
  Key bound = 0;
  if (full > 0 && warp < full) {
    const int j = (best + full - 1) / full;
    if (j <= 32) {
      Key k = mine;
      for (int i = 0; i < j; ++i) {
        bound = warp_max_key(k);
        if (k == bound) k = 0;
      }
    }
  }
  if (lane == 0) sh.warp_bound[warp] = bound;
  if (tid < kMaxBest) sh.top[tid] = 0;
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  bound = full > 0 ? sh.warp_bound[0] : 0;
  for (int i = 1; i < full; ++i) bound = min(bound, sh.warp_bound[i]);
  if (mine >= bound && mine != 0) {
    for (int v = lo + tid; v < hi; v += kVecs * kThreads) {
      float x[kVecs][W];
      load_chunk(row, v, hi, x);
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const int u = v + i * kThreads, idx = row.first_word(u) + j;
          if (x[i][j] == x[i][j] && u < hi && idx >= 0 && idx < row.V) {
            const Key k = make_key(x[i][j], idx);
            if (k >= bound) {
              const int at = atomicAdd(&sh.n_list, 1);
              if (at < kList) sh.list[at] = k;
            }
          }
        }
    }
  }
  __syncthreads();
  const int n = sh.n_list;
  if (n <= kList) {
    in_order(sh.list, n, [&](int place, Key k) {
      if (place < best) sh.top[place] = k;
    });
  } else {
    Key before = ~0ull;
    for (int r = 0; r < best; ++r) {
      Key k = 0;
      for (int v = lo + tid; v < hi; v += kVecs * kThreads) {
        float x[kVecs][W];
        load_chunk(row, v, hi, x);
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const int u = v + i * kThreads, idx = row.first_word(u) + j;
            if (x[i][j] == x[i][j] && u < hi && idx >= 0 && idx < row.V) {
              const Key q = make_key(x[i][j], idx);
              if (q < before && q > k) k = q;
            }
          }
      }
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

template <bool F32>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const __grid_constant__ LogprobArgs a) {
  constexpr int W = Row<F32>::kWords;
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_slices = a.slices, r = (int)blockIdx.x / n_slices, rank = (int)blockIdx.x - r * n_slices;
  if (n_slices > 1) cluster_arrive_relaxed();   // (waited for before the first write to another CTA)
  pdl_launch_dependents();
  const Row<F32> row(a, r);
  const int per = (row.n_vec + n_slices - 1) / n_slices;
  const int lo = min(row.n_vec, rank * per), hi = min(row.n_vec, lo + per);
  const float c = a.inv_temperature * kLog2e;
  pdl_wait();

  Stat s = {-INFINITY, 0.f, 0.f};
  float top_value = -INFINITY;
  int top_v = -1;
  for (int v = lo + tid; v < hi; v += kVecs * kThreads) {
    float x[kVecs][W];
    load_chunk(row, v, hi, x);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int j = 0; j < W; j += 2) m = fmax3(m, x[i][j], x[i][j + 1]);
    if (m > top_value || top_v < 0) {
      top_value = m;
      top_v = v;
    }
    if (m > s.m) {
      if (s.z != 0.f) {                         // (s.m is finite then)
        const float d = s.m - m, f = ex2_approx(d * c);
        s.e = f == 0.f ? 0.f : f * fmaf(d, s.z, s.e);
        s.z *= f;
      }
      s.m = m;
    }
    const float m0 = s.m == -INFINITY ? 0.f : s.m;
    float z = 0.f, e = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float d = x[i][j] - m0, q = ex2_approx(d * c);
        z += q;
        e = fmaf(q, fmaxf(d, -1e30f), e);       // (a word masked out: 0 times a large number, not times infinity)
      }
    s.z += z;
    s.e += e;
  }
  if (a.best > 0) best_words(sh, row, lo, hi, a.best, top_value, top_v);

#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Stat b = {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o), __shfl_xor_sync(0xffffffffu, s.e, o)};
    s = join(s, b, c);
  }
  if (lane == 0) sh.warp_stat[warp] = s;
  __syncthreads();
  s = sh.warp_stat[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) s = join(s, sh.warp_stat[i], c);

  const Key* keys = sh.top;
  int n_keys = a.best;
  if (n_slices > 1) {
    cluster_wait();                             // every CTA of the cluster has started
    if (tid < a.best) {
      const uint32_t at = map_to_cta(smem_u32(&sh.keys[0][0] + rank * a.best + tid), 0);
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(sh.top[tid]) : "memory");
    }
    if (tid == 0) {
      const uint32_t at = map_to_cta(smem_u32(&sh.stat[rank]), 0);
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(s.m) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(s.z) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(s.e) : "memory");
    }
    cluster_sync();
    if (rank != 0) return;
    s = sh.stat[0];
    for (int i = 1; i < n_slices; ++i) s = join(s, sh.stat[i], c);
    keys = &sh.keys[0][0];
    n_keys = n_slices * a.best;
  }

  // log(z) of a row without a finite logit is -inf: all its log probabilities are, and its entropy is 0
  const bool empty = s.z == 0.f;
  const float log_z = log2f(s.z) * kLn2, lse = empty ? -INFINITY : fmaf(s.m, a.inv_temperature, log_z);
  // (the difference to the maximum first: x - lse would lose log Z where the maximum is huge, as in a row of the type's lowest value)
  auto log_p = [&](float raw) { return empty ? -INFINITY : fmaf(raw - s.m, a.inv_temperature, -log_z); };
  if (tid == 0) {
    a.lse[r] = lse;
    a.entropy[r] = empty ? 0.f : log_z - s.e * a.inv_temperature / s.z;
  }
  for (int i = tid; i < a.given; i += kThreads) {
    const long long at = (long long)r * a.given + i;
    const int t = a.tokens[at];
    float lp = -INFINITY;                       // -1: no token
    if (t >= 0 && t < a.V) lp = log_p(row.word(t));
    else if (t != -1) spx_raise(a.status, SPECEXT_ERR_INVALID_ARG);
    a.logprob[at] = lp;
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

template <bool F32>
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
  return cudaLaunchKernelEx(&cfg, logprob_kernel<F32>, a);
}

}  // namespace

cudaError_t spx_launch_logprobs(const void* logits, bool f32, int rows, int V, long long stride, float inv_temperature,
                                const int32_t* tokens, int given, int best, float* logprob, float* entropy, float* lse,
                                int32_t* top_ids, float* top_logprob, int n_sm, int32_t* status, cudaStream_t st) {
  LogprobArgs a;
  a.logits = logits; a.tokens = tokens;
  a.logprob = logprob; a.entropy = entropy; a.lse = lse; a.top_ids = top_ids; a.top_logprob = top_logprob; a.status = status;
  a.stride = stride; a.V = V; a.given = given; a.best = best; a.inv_temperature = inv_temperature;
  // CTAs per row: as many as fill the chip three times, as long as a thread still has a load of its own in every slice
  const int words = f32 ? 4 : 8;
  int slices = 1;
  while (slices < kMaxSlices && (long long)rows * slices < 3ll * n_sm && V / words >= 2 * slices * 2 * kThreads) slices *= 2;
  a.slices = slices;
  return f32 ? launch<true>(a, rows, st) : launch<false>(a, rows, st);
}
