// Attention over the 8-bit prefix cache (q8.cuh) for few stacked (query head x node) rows of a KV head, single-token decoding first
// of all, and for more where the prefix is short, in blocks of 8 or 16 (rows_instead in api.cu draws the line).  Here a key costs its
// bytes and next to nothing else, so the kernel is laid out to keep loads in flight and to have no meeting points: keys are dealt
// in groups of 16, every warp has groups of its own (every eighth of its CTA's) and a ring of its own in shared memory, which it
// fills by asynchronous copies five groups ahead, 160 KB in flight per SM.  Nothing waits on a barrier before the end, there are
// no tensor maps to encode and to fetch, and the keys are dealt to the SMs almost evenly.
//
// What bounds it: HBM for long prefixes (one node of 32 query / 8 KV heads at 128K 48.4 us, 5.5 TB/s), else latency (1K 5.1 us).
//
// Keys are the M side of the (warp-level) products, query rows the N side in groups of 8:
//   S^T = K Q^T (16 keys x 8 rows),  O^T += V^T P^T (16 columns x 8 rows, 16 keys deep),
// so four or eight rows are padded to 8 and not to the 128 of a tcgen05 product, and the codes go from shared memory through one
// conversion per two codes straight into the A operands: a lane reads whole 16-byte pieces of a key, the order of the summed
// dimension being free, and pairs the values of two keys by one byte permutation per two pairs.  (128 keys are 32768 codes: 512
// cycles of conversions a scheduler, 256 of products for 8 rows, against 1460 for their bytes at an SM's share of the copy rate.)
// Scales and arithmetic are those of verify_q8.cu; every warp has a reference maximum of its own.
//
// The CTAs of a KV head (problem) are one cluster that merges through shared memory, each CTA receiving its share of the rows
// from all; or, without clusters, they leave partial results to the merge kernel.
#include <atomic>

#include "pair.cuh"
#include "q8.cuh"

using namespace sm100;
using namespace pair;

namespace {

constexpr int kGroupKeys = 16;
constexpr int kMaxCluster = 16, kParts = 30;             // parts a CTA receives: CTAs x rows of its share (16 rows over 1 to 16)
constexpr float kHeadroom = 6.0f, kSlack = 8.0f;         // log2, see verify_q8.cu
constexpr float kLn2 = 0.693147180559945309417f;

// Shared memory: a ring per warp (a stage: 16 keys, then their values), whose room later holds the warps' O | parts received
// from the cluster.
template <int D, int NR>
struct Geo {
  static constexpr int kWarps = 8, kThreads = kWarps * 32;
  static constexpr int kHalf = kGroupKeys * D, kStage = 2 * kHalf;
  static constexpr int kStages = D == 128 ? 6 : 8;
  static constexpr int kRing = kStages * kStage;
  static constexpr int kParts0 = kWarps * kRing;
  static constexpr int kBytes = kParts0 + kParts * (D * 4 + 8) + 128;
  static_assert(kRing >= NR * 8 * D * 4, "the rings later hold the warps' O");
  static_assert(kBytes + kWarps * 32 * 8 <= 232448, "more shared memory than a CTA can have");
};

__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, uint32_t bytes, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(bytes), "l"(policy) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// 16 or 8 bytes into the shared memory of a CTA of the cluster, counted on a barrier there: data and signal go one way, where
// plain stores and a meeting of the cluster wait for the stores to arrive first.
__device__ __forceinline__ void send_v4(uint32_t dst, uint32_t bar, float4 x) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst),
               "r"(__float_as_uint(x.x)), "r"(__float_as_uint(x.y)), "r"(__float_as_uint(x.z)), "r"(__float_as_uint(x.w)), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void send_v2(uint32_t dst, uint32_t bar, float x, float y) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(dst),
               "r"(__float_as_uint(x)), "r"(__float_as_uint(y)), "r"(bar)
               : "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// What a warp has of its rows: lane (g, t) = (lane / 4, lane % 4).  S^T of a step: keys g and g + 8, rows 2t and 2t + 1 of a group.
template <int D, int NR>
struct WarpState {
  uint32_t q[NR][D / 16][2];                    // B operands: row g, elements (D/4) t + 4 j + {0, 1}, + {2, 3}
  float mult[NR][2];                            // of rows 2t, 2t + 1: softmax scale, log2 e, the query row's power of two
  float m[NR][2], l[NR][2];
  float o[D / 16][NR][4];                       // O^T: see store_o
};

// One step: 16 keys.  k_frag(j, a): A operand of the j-th 16 elements of the keys; v_frag(w, a): those of output columns 4w .. 4w + 3
// of each lane's share, two products' worth.  visible(n, row, key): whether a row sees the key (only asked when `masked`).
template <int D, int NR, class KFrag, class VFrag, class Visible>
__device__ __forceinline__ void step(WarpState<D, NR>& st, float k_scale, float v_log2, float v_inv, bool masked, KFrag&& k_frag,
                                     VFrag&& v_frag, Visible&& visible) {
  float s[NR][4], s2[NR][4];                    // two chains: the products' latency is what a step waits for
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] = s2[n][i] = 0.f;
#pragma unroll
  for (int j = 0; j < D / 16; ++j) {
    uint32_t a[4];
    k_frag(j, a);
#pragma unroll
    for (int n = 0; n < NR; ++n) mma16816(j & 1 ? s2[n] : s[n], a, st.q[n][j][0], st.q[n][j][1]);
  }
  bool high = false;
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z = fmaf(s[n][i] + s2[n][i], st.mult[n][i & 1] * k_scale, v_log2);
      if (masked && !visible(n, i & 1, i >> 1)) z = -INFINITY;
      s[n][i] = z;
      high |= z > st.m[n][i & 1] + (kHeadroom + kSlack);
    }
  if (__any_sync(0xffffffffu, high)) {
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float z = fmaxf(s[n][c], s[n][c + 2]);
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, x));
        z -= kHeadroom;
        if (z > st.m[n][c] + kSlack) {          // (-inf in the beginning)
          const float f = ex2_approx(st.m[n][c] - z);
          st.m[n][c] = z;
          st.l[n][c] *= f;
#pragma unroll
          for (int mt = 0; mt < D / 16; ++mt) {
            st.o[mt][n][c] *= f;
            st.o[mt][n][c + 2] *= f;
          }
        }
      }
  }
  uint32_t p[NR][2];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const float m0 = st.m[n][0] == -INFINITY ? 0.f : st.m[n][0], m1 = st.m[n][1] == -INFINITY ? 0.f : st.m[n][1];
    const float e0 = ex2_approx(s[n][0] - m0), e1 = ex2_approx(s[n][1] - m1), e2 = ex2_approx(s[n][2] - m0), e3 = ex2_approx(s[n][3] - m1);
    st.l[n][0] = fmaf(e0 + e2, v_inv, st.l[n][0]);
    st.l[n][1] = fmaf(e1 + e3, v_inv, st.l[n][1]);
    p[n][0] = transpose8x8(pack_f16x2(e0, e1));
    p[n][1] = transpose8x8(pack_f16x2(e2, e3));
  }
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    uint32_t a[2][4];
    v_frag(w, a);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NR; ++n) mma16816(st.o[2 * w + i][n], a[i], p[n][0], p[n][1]);
  }
}

// Place of 16-byte piece c of a staged key, moved about so that the lanes' reads (of keys, and of one piece of several keys) and
// the copies use all banks.
template <int D>
__device__ __forceinline__ int piece(int key, int c) {
  return key * D + ((D == 128 ? c ^ (key & 7) : c ^ ((key >> 1) & 3)) << 4);
}

// `then`: what to do between the reads of the stage and their use.
template <int D, int NR, class Then>
__device__ __forceinline__ void staged_step(WarpState<D, NR>& st, const unsigned char* stage, int nkeys, float ks, float ev, float iv,
                                            int lane, Then&& then) {
  const int g = lane >> 2, t = lane & 3;
  constexpr int P = D / 64;                     // 16-byte pieces of a lane's quarter of a key
  uint32_t kw[2][P * 4], vw[4][D / 32];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint4 x = *reinterpret_cast<const uint4*>(stage + piece<D>(g + 8 * h, P * t + i));
      kw[h][4 * i] = x.x; kw[h][4 * i + 1] = x.y; kw[h][4 * i + 2] = x.z; kw[h][4 * i + 3] = x.w;
    }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = 2 * t + (i & 1) + 8 * (i >> 1);
    const unsigned char* v = stage + kGroupKeys * D;
    if constexpr (D == 128) {
      const uint4 x = *reinterpret_cast<const uint4*>(v + piece<D>(key, g));
      vw[i][0] = x.x; vw[i][1] = x.y; vw[i][2 % (D / 32)] = x.z; vw[i][3 % (D / 32)] = x.w;
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(v + piece<D>(key, g >> 1) + (g & 1) * 8);
      vw[i][0] = x.x; vw[i][1] = x.y;
    }
  }
  then();
  step<D, NR>(
      st, ks, ev, iv, nkeys < kGroupKeys,
      [&](int j, uint32_t (&a)[4]) {
        a[0] = e4m3x2_to_f16x2(kw[0][j]);
        a[1] = e4m3x2_to_f16x2(kw[1][j]);
        a[2] = e4m3x2_to_f16x2(kw[0][j] >> 16);
        a[3] = e4m3x2_to_f16x2(kw[1][j] >> 16);
      },
      [&](int w, uint32_t (&a)[2][4]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t lo = __byte_perm(vw[0][w], vw[1][w], i ? 0x7362 : 0x5140);       // keys 2t, 2t + 1
          const uint32_t hi = __byte_perm(vw[2][w], vw[3][w], i ? 0x7362 : 0x5140);       // keys 2t + 8, 2t + 9
          a[i][0] = e4m3x2_to_f16x2(lo);
          a[i][1] = e4m3x2_to_f16x2(lo >> 16);
          a[i][2] = e4m3x2_to_f16x2(hi);
          a[i][3] = e4m3x2_to_f16x2(hi >> 16);
        }
      },
      [&](int, int, int h) { return g + 8 * h < nkeys; });
}

// 16 tree nodes from `node0` on, bf16 from global memory; lane i has in `row_seen` which of them row i sees.
template <int D, int NR>
__device__ __forceinline__ void tree_step(WarpState<D, NR>& st, const AttnArgs& a, int head, int node0, uint32_t row_seen, int lane) {
  const int g = lane >> 2, t = lane & 3, T = a.plan.T;
  uint32_t kw[2][D / 8], vw[4][D / 16];         // bf16 pairs
  uint32_t km = 0u, vm = 0u;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int u = node0 + g + 8 * h;
    const uint4* src = reinterpret_cast<const uint4*>(a.Kt + (long long)u * a.tkv_st + (long long)head * a.tkv_sh + (D / 4) * t);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 x = u < T ? src[i] : none;
      kw[h][4 * i] = x.x; kw[h][4 * i + 1] = x.y; kw[h][4 * i + 2] = x.z; kw[h][4 * i + 3] = x.w;
      km = amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(km, x.x), x.y), x.z), x.w);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = node0 + 2 * t + (i & 1) + 8 * (i >> 1);
    const uint4* src = reinterpret_cast<const uint4*>(a.Vt + (long long)u * a.tkv_st + (long long)head * a.tkv_sh + (D / 8) * g);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const uint4 x = u < T ? src[c] : none;
      vw[i][4 * c] = x.x; vw[i][4 * c + 1] = x.y; vw[i][4 * c + 2] = x.z; vw[i][4 * c + 3] = x.w;
      vm = amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(vm, x.x), x.y), x.z), x.w);
    }
  }
  const int ke = f16_exponent(__reduce_max_sync(0xffffffffu, km)), ve = f16_exponent(__reduce_max_sync(0xffffffffu, vm));
  const float kf = exp2_int(-ke), vf = exp2_int(-ve);
  uint32_t seen[NR][2];
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) seen[n][c] = __shfl_sync(0xffffffffu, row_seen, n * 8 + 2 * t + c);
  step<D, NR>(
      st, exp2_int(ke), (float)ve, exp2_int(-ve), true,
      [&](int j, uint32_t (&x)[4]) {
        x[0] = bf16x2_to_f16x2(kw[0][2 * j], kf);
        x[1] = bf16x2_to_f16x2(kw[1][2 * j], kf);
        x[2] = bf16x2_to_f16x2(kw[0][2 * j + 1], kf);
        x[3] = bf16x2_to_f16x2(kw[1][2 * j + 1], kf);
      },
      [&](int w, uint32_t (&x)[2][4]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int c = 2 * w + i;              // a pair of columns, of four keys
          const uint32_t e0 = __byte_perm(vw[0][c], vw[1][c], 0x5410), o0 = __byte_perm(vw[0][c], vw[1][c], 0x7632);
          const uint32_t e1 = __byte_perm(vw[2][c], vw[3][c], 0x5410), o1 = __byte_perm(vw[2][c], vw[3][c], 0x7632);
          x[i][0] = bf16x2_to_f16x2(e0, vf);
          x[i][1] = bf16x2_to_f16x2(o0, vf);
          x[i][2] = bf16x2_to_f16x2(e1, vf);
          x[i][3] = bf16x2_to_f16x2(o1, vf);
        }
      },
      [&](int n, int c, int h) { return ((seen[n][c] >> (g + 8 * h)) & 1u) != 0; });
}

// The warps' results of one row's four columns: reference maximum, row sum, O.
template <int D, int ROWS, int kWarps>
__device__ __forceinline__ float4 join_warps(const float* o, const float2 (&ml)[kWarps][32], int row, int col, float& m, float& l) {
  float w[kWarps];
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    w[i] = ml[i][row].x;
    m = fmaxf(m, w[i]);
  }
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    // (none: no key of the warp is seen by the row, nor of any other where m is none too, as in a worker that has later tree keys only)
    const float f = w[i] == -INFINITY ? 0.f : ex2_approx(w[i] - m);
    const float4 x = *reinterpret_cast<const float4*>(o + (i * ROWS + row) * D + ((col ^ (row >> 1 & 3)) << 2));
    l = fmaf(ml[i][row].y, f, l);
    acc.x = fmaf(f, x.x, acc.x);
    acc.y = fmaf(f, x.y, acc.y);
    acc.z = fmaf(f, x.z, acc.z);
    acc.w = fmaf(f, x.w, acc.w);
  }
  return acc;
}

// NR: groups of 8 rows.  CLUSTER: the workers of a problem merge among themselves.
template <int D, int NR, bool CLUSTER>
__global__ void __launch_bounds__(Geo<D, NR>::kThreads, 1)
rows_q8_kernel(const __grid_constant__ Q8Args args) {
  using G = Geo<D, NR>;
  constexpr int kWarps = G::kWarps, kThreads = G::kThreads, kRows = NR * 8, kCols = D / 4;
  const AttnArgs& a = args.a;
  const AttnPlan& p = a.plan;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~static_cast<uintptr_t>(127));
  __shared__ float2 warp_ml[kWarps][32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int worker = blockIdx.x, prob = worker / p.cpp, head = prob / p.n_rblk;
  const int row0 = (prob - head * p.n_rblk) * kRows;     // the problem's rows (with one row block: all)
  // units are groups of 16 keys; those from p.TPH on are the tree's
  const int unit_lo = spx_unit_start(p, worker), unit_hi = spx_unit_start(p, worker + 1);
  const int first = unit_lo - prob * p.UPP + warp, end = unit_hi - prob * p.UPP, staged_end = min(end, p.TPH);
  const int log_g = 31 - __clz(p.G);
  const uint32_t ring = smem_u32(base) + warp * G::kRing;
  const unsigned char* ring_ptr = base + warp * G::kRing;
  // CTAs of the cluster, rows of a CTA's share, and this one's
  const int n_rows = min(kRows, p.rows - row0), cs = CLUSTER ? p.cluster : 1, rank = CLUSTER ? (int)cluster_rank() : 0;
  const int run = (n_rows + cs - 1) / cs, n_mine = min(run, n_rows - rank * run);
  __shared__ uint64_t arrived;                           // the parts of this CTA's rows, from all CTAs
  __shared__ int abort_flag;
  if constexpr (CLUSTER) {
    if (tid == 0) {
      abort_flag = 0;
      mbar_init(&arrived, 1);
      fence_mbar_init();
      if (n_mine > 0) mbar_arrive_expect_tx(&arrived, cs * n_mine * (D * 4 + 8));
    }
    __syncwarp();
    cluster_arrive();                                    // (waited for before the first write to another CTA)
  }
  pdl_launch_dependents();

  // A lane copies the same piece of every 4th (8th for D = 64) key.  Requests and scales go by running pointers: a step is 128 keys
  // further on, which is a whole number of blocks.
  constexpr int kPieces = D / 16, kStep = 32 / kPieces, kCopies = kGroupKeys / kStep;
  const int c_row = lane / kPieces, c_col = lane % kPieces;
  const long long at0 = (long long)(first * kGroupKeys + c_row) * a.kv_sl + (long long)head * a.kv_sh + c_col * 16;
  const long long row_step = kStep * a.kv_sl, unit_step = kWarps * kGroupKeys * a.kv_sl;
  const uint8_t *k_src = args.Kc + at0, *v_src = args.Vc + at0;
  const uint64_t stream_once = policy_evict_first();
  auto request = [&](int unit, int stage) {
    const uint32_t dst = ring + stage * G::kStage;
    if (unit < p.L / kGroupKeys && unit < staged_end) {
      const uint8_t *k = k_src, *v = v_src;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        copy_async(dst + piece<D>(c_row + i * kStep, c_col), k, 16u, stream_once);
        copy_async(dst + G::kHalf + piece<D>(c_row + i * kStep, c_col), v, 16u, stream_once);
        k += row_step;
        v += row_step;
      }
    } else if (unit < staged_end) {
      // the last, ragged group: nothing behind the prefix is read, zeros stand there
#pragma unroll 1
      for (int i = 0; i < kCopies; ++i) {
        const int row = c_row + i * kStep;
        const bool in = unit * kGroupKeys + row < p.L;
        const long long off = in ? i * row_step : 0;
        copy_async(dst + piece<D>(row, c_col), in ? k_src + off : args.Kc, in ? 16u : 0u, stream_once);
        copy_async(dst + G::kHalf + piece<D>(row, c_col), in ? v_src + off : args.Vc, in ? 16u : 0u, stream_once);
      }
    }
    k_src += unit_step;
    v_src += unit_step;
    copies_commit();
  };
  const long long s_at = (long long)((first * kGroupKeys) >> args.log_block) * args.s_sb + (long long)head * args.s_sh;
  const long long s_step = (long long)((kWarps * kGroupKeys) >> args.log_block) * args.s_sb;
  static_assert(kWarps * kGroupKeys == 128, "a step is a whole number of blocks");
  const uint8_t *ks_src = args.Ks + s_at, *vs_src = args.Vs + s_at;
  // The first keys are asked for in L2 ahead of the wait for the kernel before (what it may still write to them goes through L2
  // as well).
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (first + i * kWarps < min(staged_end, p.L / kGroupKeys)) {
#pragma unroll
      for (int j = 0; j < kCopies; ++j) {
        asm volatile("prefetch.global.L2 [%0];" ::"l"(k_src + i * unit_step + j * row_step));
        asm volatile("prefetch.global.L2 [%0];" ::"l"(v_src + i * unit_step + j * row_step));
      }
    }
  }
  pdl_wait();
  // (queries and scales first: behind the copies they would come after 160 KB of keys and values)
  uint32_t ks = 127u, vs = 127u;
  if (first < staged_end) {
    ks = *ks_src;
    vs = *vs_src;
  }
  uint4 q_raw[NR][D / 32];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int r = row0 + n * 8 + g;
    const uint4* src = reinterpret_cast<const uint4*>(a.Q + (long long)(r >> log_g) * a.q_st +
                                                      (long long)(head * p.G + (r & (p.G - 1))) * a.q_sh + (D / 4) * t);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) q_raw[n][i] = r < p.rows ? src[i] : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int i = 0; i < G::kStages - 1; ++i) request(first + i * kWarps, i);

  WarpState<D, NR> st;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      st.m[n][c] = -INFINITY;
      st.l[n][c] = 0.f;
    }
#pragma unroll
    for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.o[mt][n][i] = 0.f;
  }
  // query rows: f16 with the row's own power of two
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    uint32_t w[D / 8];
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 x = q_raw[n][i];
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
      m = amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(m, x.x), x.y), x.z), x.w);
    }
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const int e = f16_exponent(m);
    const float f = exp2_int(-e);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      st.q[n][j][0] = bf16x2_to_f16x2(w[2 * j], f);
      st.q[n][j][1] = bf16x2_to_f16x2(w[2 * j + 1], f);
    }
    const float mult = p.scale2 * exp2_int(e);
    st.mult[n][0] = __shfl_sync(0xffffffffu, mult, 8 * t);
    st.mult[n][1] = __shfl_sync(0xffffffffu, mult, 8 * t + 4);
  }

  // Tree nodes come first: their keys and values are fetched while the first copies are on their way.  (The warp's units are
  // first, first + kWarps, ..; those behind the prefix are the tree's.)
#pragma unroll 1
  for (int unit = first + (max(p.TPH - first, 0) + kWarps - 1) / kWarps * kWarps; unit < end; unit += kWarps) {
    const int node0 = (unit - p.TPH) * kGroupKeys;
    // which of the unit's 16 nodes the node of row `lane` sees: itself and its ancestors
    uint32_t seen = 0u;
    bool bad = false;
    int u = row0 + lane < p.rows ? (row0 + lane) >> log_g : -1;
#pragma unroll 1
    for (int i = 0; i < p.T && u >= 0; ++i) {
      if ((unsigned)(u - node0) < (unsigned)kGroupKeys) seen |= 1u << (u - node0);
      const int pu = a.parent[u];
      u = pu < u ? pu : -1;
    }
    for (int v = lane; v < p.T; v += 32) bad |= a.parent[v] < -1 || a.parent[v] >= v;
    if (bad) spx_raise(a.status, SPECEXT_ERR_BAD_TREE);
    __syncwarp();
    tree_step<D, NR>(st, a, head, node0, seen, lane);
  }
  int stage = 0;
#pragma unroll 1
  for (int unit = first; unit < staged_end; unit += kWarps) {
    if (unit + kWarps < staged_end) {
      ks_src += s_step;
      vs_src += s_step;
    }
    const uint32_t ks_next = *ks_src, vs_next = *vs_src;
    copies_wait<G::kStages - 2>();
    __syncwarp();
    staged_step<D, NR>(st, ring_ptr + stage * G::kStage, p.L - unit * kGroupKeys, e8m0_value(ks), e8m0_log2(vs),
                       e8m0_value(vs == 255u ? 255u : 254u - vs), lane, [&]() {
                         // into the stage that the step before has read
                         request(unit + (G::kStages - 1) * kWarps, stage == 0 ? G::kStages - 1 : stage - 1);
                       });
    stage = stage == G::kStages - 1 ? 0 : stage + 1;
    ks = ks_next;
    vs = vs_next;
  }
  copies_wait<0>();                                      // (none left that holds anything)

  // every warp is done with its ring: the room holds the warps' O, [warp][row][D], the 16-byte columns of a row moved by its pair
  // so that a warp's stores use all banks
  __syncthreads();
  float* room = reinterpret_cast<float*>(base);
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = n * 8 + 2 * t + c;
      float l = st.l[n][c];
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      if (g == 0) warp_ml[warp][row] = make_float2(st.m[n][c], l);
      float* dst = room + (warp * kRows + row) * D;
#pragma unroll
      for (int w = 0; w < D / 32; ++w)
        *reinterpret_cast<float4*>(dst + (((D / 32) * g + w) ^ t) * 4) =
            make_float4(st.o[2 * w][n][c], st.o[2 * w][n][c + 2], st.o[2 * w + 1][n][c], st.o[2 * w + 1][n][c + 2]);
    }
  __syncthreads();
  if constexpr (!CLUSTER) {
    const int slot = worker + prob;                      // (one row block: the merge kernel's blocks have 32 rows)
    float* po = a.ws + p.off_part_o + (long long)slot * kCols * p.RB * 4;
    for (int i = tid; i < n_rows * kCols; i += kThreads) {
      const int col = i / n_rows, row = i - col * n_rows;
      float m, l;
      const float4 x = join_warps<D, kRows, kWarps>(room, warp_ml, row, col, m, l);
      *reinterpret_cast<float4*>(po + ((long long)col * p.RB + row) * 4) = x;
      if (col == 0) {
        a.ws[p.off_part_m + (long long)slot * p.RB + row] = m;
        a.ws[p.off_part_l + (long long)slot * p.RB + row] = l;
      }
    }
  } else {
    float4* part = reinterpret_cast<float4*>(base + G::kParts0);               // [source CTA][row of the share][column]
    float2* ml = reinterpret_cast<float2*>(base + G::kParts0 + kParts * D * 4);
    cluster_wait();                                      // every CTA of the cluster has started
    for (int i = tid; i < n_rows * kCols; i += kThreads) {
      const int row = i / kCols, col = i - row * kCols, owner = row / run, slot = rank * min(run, n_rows - owner * run) + row - owner * run;
      float m, l;
      const float4 x = join_warps<D, kRows, kWarps>(room, warp_ml, row, col, m, l);
      const uint32_t bar = map_to_cta(smem_u32(&arrived), owner);
      send_v4(map_to_cta(smem_u32(part + slot * kCols + col), owner), bar, x);
      if (col == 0) send_v2(map_to_cta(smem_u32(ml + slot), owner), bar, m, l);
    }
    if (n_mine <= 0) return;
    if (!mbar_wait(&arrived, 0, &abort_flag)) {
      if (lane == 0) spx_raise(a.status, SPECEXT_ERR_TIMEOUT);
      settle();
      return;
    }
    for (int i = tid; i < n_mine * kCols; i += kThreads) {
      const int mine = i / kCols, col = i - mine * kCols, row = rank * run + mine;
      // (loops as they are: unrolled to 16 parts, code that runs once takes 1300 cycles to fetch and run, this 640)
      float M = -INFINITY, Z = 0.f;
#pragma unroll 4
      for (int c = 0; c < cs; ++c) M = fmaxf(M, ml[c * n_mine + mine].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
      for (int c = 0; c < cs; ++c) {
        const float2 s = ml[c * n_mine + mine];
        const float4 x = part[(c * n_mine + mine) * kCols + col];
        const float f = ex2_approx(s.x - M);
        Z = fmaf(s.y, f, Z);
        acc.x = fmaf(f, x.x, acc.x);
        acc.y = fmaf(f, x.y, acc.y);
        acc.z = fmaf(f, x.z, acc.z);
        acc.w = fmaf(f, x.w, acc.w);
      }
      const float inv = 1.f / Z;
      const int node = (row0 + row) >> log_g, h = head * p.G + ((row0 + row) & (p.G - 1));
      *reinterpret_cast<uint2*>(a.O + (long long)node * a.o_st + (long long)h * a.o_sh + col * 4) =
          make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
      if (col == 0) a.lse[(long long)h * p.T + node] = (M + log2f(Z)) * kLn2;
    }
  }
}

template <int D, int NR, bool CLUSTER>
cudaError_t launch(const Q8Args& q, cudaStream_t st) {
  static SpxOncePerDevice once;
  const cudaError_t ec = spx_opt_in_smem(rows_q8_kernel<D, NR, CLUSTER>, Geo<D, NR>::kBytes, &once, CLUSTER);
  if (ec != cudaSuccess) return ec;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(q.a.plan.n_cta);
  cfg.blockDim = dim3(Geo<D, NR>::kThreads);
  cfg.dynamicSmemBytes = Geo<D, NR>::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = q.a.plan.cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CLUSTER ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, rows_q8_kernel<D, NR, CLUSTER>, q);
}

template <int D, bool CLUSTER>
cudaError_t launch_rows(const Q8Args& q, cudaStream_t st) {
  return q.a.plan.q_rows == 8 ? launch<D, 1, CLUSTER>(q, st) : launch<D, 2, CLUSTER>(q, st);
}

}  // namespace

// How many clusters of `size` CTAs of this kernel device `dev` (the current one) holds at once, looked up once per device and
// size; 0 when there is no device.
int spx_rows_q8_max_clusters(int dev, int size) {
  static std::atomic<int> known[kSpxMaxDevices][kMaxCluster + 1];
  if (dev < 0 || dev >= kSpxMaxDevices || size < 1 || size > kMaxCluster) return 0;
  int n = known[dev][size].load();
  if (n > 0) return n - 1;
  auto* kernel = rows_q8_kernel<128, 2, true>;
  static SpxOncePerDevice once;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(size);
  cfg.blockDim = dim3(Geo<128, 2>::kThreads);
  cfg.dynamicSmemBytes = Geo<128, 2>::kBytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (spx_opt_in_smem(kernel, Geo<128, 2>::kBytes, &once, true) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  known[dev][size].store(n + 1);
  return n;
}

cudaError_t spx_launch_rows_q8(const Q8Args& q, cudaStream_t st, int* n_launches) {
  const bool cluster = q.a.plan.cluster > 0;
  *n_launches += 1;
  if (q.a.plan.D == 128) return cluster ? launch_rows<128, true>(q, st) : launch_rows<128, false>(q, st);
  return cluster ? launch_rows<64, true>(q, st) : launch_rows<64, false>(q, st);
}
