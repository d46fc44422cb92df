// Hybrid Tree Attention over a prefix cache in 8 bits (codes e4m3, scales e8m0, see q8.cuh), on the pipeline of core.cuh: partial
// attention of 128 stacked (query head x tree node) rows of one KV head by a CTA, or of 256 by a pair of CTAs (tcgen05
// cta_group::2, each staging half of every key tile), against a run of 128-key tiles.
//
// S = Q K^T is a product of e4m3 by e4m3, twice: a bf16 value has 8 significant bits and is the sum of two e4m3 values of 4, so
// with the query row taken to [2^7, 2^8) by a power of two its high and low parts, multiplied with the codes as they lie in
// memory, give S as exactly as bf16 products would, in the time of the bf16 products and without touching K.  (e4m3's smallest step is
// 2^-9: elements below 2^-9 of the row's largest are kept to half of it, 2^-17 of the largest.)  The tree's bf16 keys are two such tiles, high parts
// and low parts, with a power of two per 32 nodes.
// For O += P V the codes of V become f16 (every e4m3 value is one: one conversion per two codes) by four warps, and P is f16.
// The scales stay outside the products:
//   z = S * (scale log2(e) 2^e k_scale) + log2(v_scale)          e: the query row's own power of two
//   P = 2^(z - M) rounded to f16,  O += P v_code,  l += 2^(z - M) / v_scale
// with M the reference maximum of z: the V scale rides on the exponent, at no cost per element, and P stays in f16's range
// whatever the scales are.  M is 2^6 below the maximum it was taken from and may fall 2^8 more behind, so P is at most 2^14;
// f16 keeps 11 bits down to 2^-20 of the row's largest weight and reaches 2^-30.
// (First both K and V were expanded to f16, by the same four warps: 2.7 us a tile of 128 keys against 0.75 for its bytes.)
//
// Warps: 0-7 the queries' parts, then softmax; 8 TMA producer of the codes, 9 issuer of the S MMAs, 10 of the PV MMAs, 11
// ancestor masks, TMA producer of Q, and the tree's keys; 12-15 the tree's scales, expansion of V (a thread has a key), and the
// tree's values.  Every wait is bounded; all threads reach the final barrier before tensor memory is freed.
//
// What bounds it: the chain of a tile, not memory.  256 rows on a pair take 0.96 us a tile (128 keys: products 0.55, as much for the
// exponentials), 128 rows on a CTA 0.95, on top of 12.5 us of launch, queries, last tile, stores and merge: 60 nodes of 32 query / 8
// KV heads 27.0 us at 16K (1.2 TB/s of codes), 32 KV heads 28.4 at 8K (2.4).
#include "core.cuh"
#include "q8.cuh"
#include "tmap.h"

using namespace core;

namespace {

constexpr int kThreadsQ8 = 512;
constexpr int kExpandWarp = 12;                // first of four
constexpr int kRegsLaunchQ8 = 128, kRegsOtherQ8 = 48, kRegsSoftmaxQ8 = 208;
static_assert(256 * (kRegsLaunchQ8 - kRegsOtherQ8) >= 256 * (kRegsSoftmaxQ8 - kRegsLaunchQ8),
              "setmaxnreg.inc would wait for registers that are never released");
constexpr float kHeadroom = 6.0f;              // log2: how far the reference lies below the maximum it was taken from
constexpr int kMaxUnits = 8;
constexpr int kTreeAhead = 4;                  // tiles ahead of its turn that the tree's K is begun with

struct Q8Maps {
  CUtensorMap q, k, v;
};

// Shared memory: Q (high parts, low parts) | V stages (f16) | ring of K codes | ring of V codes | control.  A unit of K is what
// this CTA has of a tile's keys, whole; one of V its columns of all 128 keys.
template <int PAIR, int D>
struct GeoQ8 {
  static constexpr int kQ = 128 * D;                                   // one part
  static constexpr int kVRow = PAIR == 2 ? 64 : D;                     // bytes of a key in a unit of V
  static constexpr int kVBlk = SPX_TILE_KEYS * 128, kVStage = kVBlk * (kVRow / 64);
  static constexpr int kKUnit = SPX_TILE_KEYS / PAIR * D, kVUnit = SPX_TILE_KEYS * kVRow;
  static constexpr int nv = kVStage == 32768 ? 2 : 3;
  static constexpr int kKUnits = kKUnit == 16384 ? 4 : 6, kVUnits = kVUnit == 16384 ? 3 : 6;
  static constexpr uint32_t v_off = 2 * kQ, k8_off = v_off + nv * kVStage, v8_off = k8_off + kKUnits * kKUnit;
  static constexpr int kCtrl = v8_off + kVUnits * kVUnit;
  static_assert(kTreeAhead + nv <= 2 * kKUnits - 1, "the wait for a unit could take an earlier phase for its own");
  static_assert(nv * kVStage >= 2 * kQ, "the V stages hold the bf16 queries in the beginning");
};

// Scales of a tile, per group of 32 keys.  Those of all tiles of a run are made when it begins and lie behind the control block:
// fetched by the softmax warps tile by tile they cost 600 cycles of every 3800, most of it for code that is out of the
// instruction cache by the time it is needed again.
struct alignas(16) Q8Scales {
  float4 k, v_log2, v_inv;
};
struct CtrlQ8 {
  Ctrl c;                                      // (its K ring is not used; v_full, v_empty: the f16 stages)
  uint64_t k_full[kMaxUnits];                  // leader: one arrival per CTA (the producer's with its bytes, or the tree's)
  uint64_t k_empty[kMaxUnits];                 // each CTA: MMA completion
  uint64_t vc_full[kMaxUnits], vc_empty[kMaxUnits];      // this CTA: codes of V, between the producer and the expansion
  uint64_t q_land, q_read;                     // this CTA: the bf16 queries have landed; 8 warps have read them
  uint64_t q_ready;                            // leader: 8 warps per CTA have made their query rows
  uint64_t sc_ready;                           // this CTA: the scales of the run's tiles are in shared memory
  uint64_t tree_go;                            // this CTA: the expansion is kTreeAhead tiles from the end of the prefix
  int tree_k[4], tree_v[4];                    // exponents of the tree's groups of 32 nodes
  uint2 tree_max[4][4];                        // largest magnitudes of K and V of a group, a quarter of the nodes each
  float q_scale[128];
};
constexpr int kCtrlBytesQ8 = 7168;
static_assert(sizeof(CtrlQ8) <= kCtrlBytesQ8, "control block too large");
template <int PAIR, int D>
constexpr int smem_q8() {
  return GeoQ8<PAIR, D>::kCtrl + kCtrlBytesQ8 + kSpxRunQ8 * (int)sizeof(Q8Scales) + 1024;
}

// ---- MMAs issued by a whole warp -----------------------------------------------------------------------------
// All lanes come to the instruction, and it elects the one that issues it (the same one every time), so that the compiler knows
// the operands to be the warp's and keeps them in uniform registers.  Issued by one thread of a diverged warp an MMA takes that
// thread 133 cycles (188 with A in tensor memory), this way 64 to 77: as long as the tensor cores need for it.
template <int PAIR>
__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR == 2)
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// f16, A in tensor memory.
template <int PAIR>
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc,
                                           uint32_t accumulate) {
  if constexpr (PAIR == 2)
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
template <int PAIR>
__device__ __forceinline__ void commit_warp(uint64_t* bar) {
  if constexpr (PAIR == 2)
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
        ::"r"(smem_u32(bar)), "h"((uint16_t)3)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
        ::"r"(smem_u32(bar))
        : "memory");
}
// A wait of the whole warp: true for all lanes or for none.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, wait_c(bar, parity, abort_flag));
}

// A warp's arrival on a barrier of the leader, behind its plain stores of MMA operands to this CTA's shared memory.  They are read
// by the tensor cores of this SM alone, and the proxy fence has them in place for those; what the arrival tells the leader, which
// may be the other CTA, is only that.  (Releasing at the cluster's scope takes 1100 to 1900 cycles, longer than a tile.)
template <int PAIR>
__device__ __forceinline__ void publish(uint64_t* bar, int lane) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) arrive_cluster(leader_addr<PAIR>(bar));
}

// Place of 16-byte column `col` of row `row` in a block of f16 (or bf16): blocks of 64 elements, 128-byte swizzle.
__device__ __forceinline__ int f16_place(int row, int col) { return (col >> 3) * (128 * 128) + row * 128 + (((col ^ row) & 7) << 4); }
// Place of 16-byte piece `c` of row `row` in a tile of codes, rows of W bytes, swizzled as TMA leaves them.
template <int W>
__device__ __forceinline__ int code_place(int row, int c) {
  return row * W + ((W == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4);
}

// One key's codes (W of them) as f16 into a stage.
template <int W>
__device__ __forceinline__ void expand_key(const unsigned char* unit, unsigned char* stage, int key) {
#pragma unroll 1
  for (int c = 0; c < W / 16; c += 2) {
    uint4 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = *reinterpret_cast<const uint4*>(unit + code_place<W>(key, c + i));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *reinterpret_cast<uint4*>(stage + f16_place(key, 2 * (c + i))) = make_uint4(
          e4m3x2_to_f16x2(x[i].x), e4m3x2_to_f16x2(x[i].x >> 16), e4m3x2_to_f16x2(x[i].y), e4m3x2_to_f16x2(x[i].y >> 16));
      *reinterpret_cast<uint4*>(stage + f16_place(key, 2 * (c + i) + 1)) = make_uint4(
          e4m3x2_to_f16x2(x[i].z), e4m3x2_to_f16x2(x[i].z >> 16), e4m3x2_to_f16x2(x[i].w), e4m3x2_to_f16x2(x[i].w >> 16));
    }
  }
}

// bf16 values to e4m3: the power of two 2^-e that takes the largest finite magnitude to [2^7, 2^8).
__device__ __forceinline__ int e4m3_exponent(uint32_t amax) {
  const int e = (int)(amax >> 23) - 127 - 7;
  return amax == 0u ? 0 : max(e, -126);
}
__device__ __forceinline__ uint32_t amax_bf16x8(uint32_t m, uint4 x) {
  return amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(m, x.x), x.y), x.z), x.w);
}
// High and low parts of four bf16 values times f.  As f16 the values are exact (8 bits, at most 2^8), and so is the difference.
// An infinity becomes NaN, which e4m3 has (the conversion would make it 448).
__device__ __forceinline__ void split4(uint32_t a, uint32_t b, float f, uint32_t& hi, uint32_t& lo) {
  uint32_t x0 = bf16x2_to_f16x2(a, f), x1 = bf16x2_to_f16x2(b, f);
  x0 = add_f16x2(x0, sub_f16x2(x0, x0));
  x1 = add_f16x2(x1, sub_f16x2(x1, x1));
  const uint32_t h0 = f16x2_to_e4m3x2(x0), h1 = f16x2_to_e4m3x2(x1);
  hi = h0 | (h1 << 16);
  lo = f16x2_to_e4m3x2(sub_f16x2(x0, e4m3x2_to_f16x2(h0))) | (f16x2_to_e4m3x2(sub_f16x2(x1, e4m3x2_to_f16x2(h1))) << 16);
}
// 16 bf16 values (two 16-byte pieces) as a piece of high parts and one of low parts.
__device__ __forceinline__ void split16(uint4 x, uint4 y, float f, unsigned char* hi, unsigned char* lo) {
  uint4 h, l;
  split4(x.x, x.y, f, h.x, l.x);
  split4(x.z, x.w, f, h.y, l.y);
  split4(y.x, y.y, f, h.z, l.z);
  split4(y.z, y.w, f, h.w, l.w);
  *reinterpret_cast<uint4*>(hi) = h;
  *reinterpret_cast<uint4*>(lo) = l;
}

// 16 bytes of a tree node's row into shared memory, or zeros.
__device__ __forceinline__ void copy_node(unsigned char* dst, const __nv_bfloat16* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Issuers of the S and of the PV MMAs (issue_s and issue_pv of core.cuh for one run of tiles, by whole warps of the leader CTA).
// has_tree: the last tile of the run is the tree's, two units of K.
template <int PAIR, int D>
__device__ __forceinline__ bool issue_s_q8(CtrlQ8* ctl8, unsigned char* base, int n_tiles, bool has_tree, volatile int* abort_flag) {
  using G = GeoQ8<PAIR, D>;
  Ctrl* ctl = &ctl8->c;
  const uint32_t tmem = __shfl_sync(0xffffffffu, ctl->tmem_base, 0);
  constexpr uint32_t idesc = idesc_f32<true>(128 * PAIR, SPX_TILE_KEYS, false, false);     // (e4m3: type fields 0 as for f16)
  // rows of D bytes, 8-row groups of 8 D; 128-byte swizzle, or 64-byte (mode 4) for D = 64
  constexpr uint32_t hi = D == 128 ? desc_hi(1024) : ((512u >> 4) | (1u << 14) | (4u << 29));
  const uint32_t q_lo = desc_lo(smem_u32(base), 16), k_lo = desc_lo(smem_u32(base + G::k8_off), 16);
  int st = 0;
  uint32_t ph = 0;
  bool ok = wait_warp(&ctl8->q_ready, 0, abort_flag);
  for (int j = 0; j < n_tiles && ok; ++j) {
    const int w = j & 1, units = has_tree && j == n_tiles - 1 ? 2 : 1;
    // the rows of the tile before last are in registers: its S buffer is free
    if (j >= kWG) ok = wait_warp(&ctl->s_free[w], (j / kWG - 1) & 1, abort_flag);
    const uint32_t d = tmem + kColS + w * 128;
    for (int u = 0; u < units && ok; ++u) {
      ok = wait_warp(&ctl8->k_full[st], ph, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint32_t kb = k_lo + st * (G::kKUnit >> 4);
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk)
          mma_f8<PAIR>(d, q_lo + part * (G::kQ >> 4) + kk * 2, kb + kk * 2, hi, idesc, part + kk > 0 || u > 0 ? 1u : 0u);
      commit_warp<PAIR>(&ctl8->k_empty[st]);
      if (++st == G::kKUnits) {
        st = 0;
        ph ^= 1;
      }
    }
    if (ok) commit_warp<PAIR>(&ctl->s_full[w]);
  }
  commit_warp<PAIR>(&ctl->drain);
  return ok;
}
template <int PAIR, int D>
__device__ __forceinline__ bool issue_pv_q8(CtrlQ8* ctl8, unsigned char* base, int n_tiles, volatile int* abort_flag) {
  using G = GeoQ8<PAIR, D>;
  Ctrl* ctl = &ctl8->c;
  const uint32_t tmem = __shfl_sync(0xffffffffu, ctl->tmem_base, 0);
  constexpr uint32_t idesc = idesc_f32<true>(128 * PAIR, D, false, true), hi = desc_hi(1024);
  const uint32_t v_lo = desc_lo(smem_u32(base + G::v_off), PAIR == 2 ? 16 : G::kVBlk);
  int st = 0;
  uint32_t ph = 0;
  bool ok = true;
  for (int j = 0; j < n_tiles && ok; ++j) {
    const int w = j & 1;
    ok = wait_warp(&ctl->v_full[st], ph, abort_flag) && wait_warp(&ctl->p_full[w], (j / kWG) & 1, abort_flag);
    if (!ok) break;
    tc_fence_after();
    const uint32_t vb = v_lo + st * (G::kVStage >> 4), pa = tmem + kColP + w * 64;
#pragma unroll
    for (int kk = 0; kk < SPX_TILE_KEYS / 16; ++kk)
      mma_f16_ts<PAIR>(tmem + kColO, pa + kk * 8, vb + kk * 128, hi, idesc, kk > 0 || j > 0 ? 1u : 0u);
    commit_warp<PAIR>(&ctl->pv_done[w]);
    commit_warp<PAIR>(&ctl->v_empty[st]);
    if (++st == G::nv) {
      st = 0;
      ph ^= 1;
    }
  }
  if (ok) commit_warp<PAIR>(&ctl->o_done);
  // everything issued by both must be complete before tensor memory is released
  commit_warp<PAIR>(&ctl->drain);
  for (int spin = 0; spin < (1 << 22) && !mbar_test_wait(&ctl->drain, 0); ++spin) {}
  __syncwarp();
  return ok;
}

// softmax_tile of core.cuh with scales: `mult` is the row's factor (softmax scale, log2 e, the power of two of the query row).
template <int D, class MaskFn, class SumFn>
__device__ __forceinline__ bool softmax_tile_q8(const RowCtx& rc, const Q8Scales* scales, float mult, uint32_t t, bool need_mask,
                                                MaskFn&& mask, SumFn&& sums, float& m_loc, float& l) {
  Ctrl* ctl = rc.ctl;
  const int w = rc.w, wp = w ^ 1;
  const bool first = t == 0;
  const uint32_t s_addr = rc.lane_tmem + kColS + w * 128, p_addr = rc.lane_tmem + kColP + w * 64;
  if (!wait_c(&ctl->s_full[w], (t / kWG) & 1, rc.abort_flag)) return false;
  tc_fence_after();
  uint32_t s0[32], s1[32], s2[32], s3[32];
  tmem_ld32(s_addr, s0);
  tmem_ld32(s_addr + 32, s1);
  tmem_ld32(s_addr + 64, s2);
  tmem_ld32(s_addr + 96, s3);
  const float4 ks = scales->k, ev = scales->v_log2;
  float m_cur = -INFINITY;
  if (!first) {
    if (!mbar_wait(&ctl->m_pub[wp], ((t - 1) / kWG) & 1, rc.abort_flag)) return false;
    m_cur = ctl->m_row[rc.row_t];
  }
  tmem_wait_ld();
  tc_fence_before();
  warp_arrive_cluster(rc.s_free, rc.lane);           // the S buffer may take the next tile but one
  if (need_mask) {
    unsigned long long lo, hi;
    mask(lo, hi);
    mask_chunk(s0, static_cast<uint32_t>(lo));
    mask_chunk(s1, static_cast<uint32_t>(lo >> 32));
    mask_chunk(s2, static_cast<uint32_t>(hi));
    mask_chunk(s3, static_cast<uint32_t>(hi >> 32));
  }
  auto max_group = [](const uint32_t (&s)[32]) {
    float a = -INFINITY, b = -INFINITY;
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
      a = fmax3(a, __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
      b = fmax3(b, __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
    }
    return fmaxf(a, b);
  };
  float f0 = mult * ks.x, f1 = mult * ks.y, f2 = mult * ks.z, f3 = mult * ks.w;
  if (need_mask) {
    // A masked score is -inf, and times a factor that fell to zero (a small query on a block of zeros) it would be NaN.  (Scores are
    // below 2^25: times the least normal number they are still nothing.  A NaN scale stays.)
    auto positive = [](float f) { return f < 1.17549435e-38f ? 1.17549435e-38f : f; };
    f0 = positive(f0);
    f1 = positive(f1);
    f2 = positive(f2);
    f3 = positive(f3);
  }
  const float m_tile = fmaxf(fmaxf(fmaf(max_group(s0), f0, ev.x), fmaf(max_group(s1), f1, ev.y)),
                             fmaxf(fmaf(max_group(s2), f2, ev.z), fmaf(max_group(s3), f3, ev.w))) - kHeadroom;

  float m_new = m_cur;
  bool rescale = false;
  if (m_tile > m_cur + kRescaleThreshold || m_cur == -INFINITY) {
    m_new = m_tile;
    rescale = !first;
  }
  ctl->m_row[rc.row_t] = m_new;
  warp_arrive(&ctl->m_pub[w], rc.lane);
  if (m_loc != m_new) {
    l *= (m_loc == -INFINITY) ? 0.f : ex2_approx(m_loc - m_new);
    m_loc = m_new;
  }
  if (t >= kWG && !wait_c(&ctl->pv_done[w], (t / kWG - 1) & 1, rc.abort_flag)) return false;
  if (__any_sync(0xffffffffu, rescale)) {
    // O must hold the sum up to the previous tile and nothing may be accumulating into it
    if (!wait_c(&ctl->pv_done[wp], ((t - 1) / kWG) & 1, rc.abort_flag)) return false;
    tc_fence_after();
    const float alpha = rescale ? ex2_approx(m_cur - m_new) : 1.f;
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
      uint32_t v[16];
      tmem_ld16(rc.lane_tmem + kColO + c * 16, v);
      tmem_wait_ld();
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * alpha);
      tmem_st16(rc.lane_tmem + kColO + c * 16, v);
    }
  }
  tc_fence_after();

  auto exp_chunk = [&](uint32_t (&v)[32], int c, float f, float off) {
    if (rc.pad) off = -INFINITY;
    const uint64_t fx2 = pack_f32x2(f, f), off2 = pack_f32x2(off, off);
    uint64_t acc01 = 0ull, acc23 = 0ull;
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
      float e0, e1, e2, e3;
      unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), fx2, off2), e0, e1);
      unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])), fx2, off2), e2, e3);
      e0 = ex2_approx(e0);
      e1 = ex2_approx(e1);
      e2 = ex2_approx(e2);
      e3 = ex2_approx(e3);
      acc01 = add_f32x2(acc01, pack_f32x2(e0, e1));
      acc23 = add_f32x2(acc23, pack_f32x2(e2, e3));
      v[k] = __float_as_uint(e0);
      v[k + 1] = __float_as_uint(e1);
      v[k + 2] = __float_as_uint(e2);
      v[k + 3] = __float_as_uint(e3);
    }
    float gs0, gs1, gs2, gs3;
    unpack_f32x2(acc01, gs0, gs1);
    unpack_f32x2(acc23, gs2, gs3);
    const float inv = reinterpret_cast<const float*>(&scales->v_inv)[c], gs = ((gs0 + gs1) + (gs2 + gs3)) * inv;
    l += gs;
    sums(c, v, gs, inv);
    uint32_t pk[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) pk[k] = pack_f16x2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
    tmem_st16(p_addr + c * 16, pk);
  };
  exp_chunk(s0, 0, f0, ev.x - m_new);
  exp_chunk(s1, 1, f1, ev.y - m_new);
  exp_chunk(s2, 2, f2, ev.z - m_new);
  exp_chunk(s3, 3, f3, ev.w - m_new);
  tmem_wait_st();
  tc_fence_before();
  warp_arrive_cluster(rc.p_full, rc.lane);
  return true;
}

// SCORE: as in verify.cu: 0 no chunk sums, 1 chunks of 32 keys, 2 of 64 or 128, 3 of fewer than 32.
template <int PAIR, int D, int SCORE>
__global__ void __launch_bounds__(kThreadsQ8, 1)
verify_q8_kernel(const __grid_constant__ Q8Args args, const __grid_constant__ Q8Maps maps) {
  using G = GeoQ8<PAIR, D>;
  const AttnArgs& a = args.a;
  const AttnPlan& p = a.plan;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                         ~static_cast<uintptr_t>(1023));
  CtrlQ8* ctl8 = reinterpret_cast<CtrlQ8*>(base + G::kCtrl);
  Ctrl* ctl = &ctl8->c;
  Q8Scales* scales = reinterpret_cast<Q8Scales*>(base + G::kCtrl + kCtrlBytesQ8);
  volatile int* abort_flag = &ctl->abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  const int rank = PAIR == 2 ? (int)cluster_rank() : 0;
  const int worker = blockIdx.x / PAIR, prob = worker / p.cpp;
  const int unit_lo = spx_unit_start(p, worker), n_tiles = spx_unit_start(p, worker + 1) - unit_lo;
  const int tile_lo = unit_lo - prob * p.UPP, g = prob / p.n_rblk, rblk = prob - g * p.n_rblk;
  const bool has_tree = tile_lo + n_tiles == p.UPP;
  const int n_pref = n_tiles - (has_tree ? 1 : 0);
  if (warp == kTreeWarp) {
    if (lane < kMaxUnits) {
      mbar_init(&ctl8->k_full[lane], PAIR);
      mbar_init(&ctl8->k_empty[lane], 1);
      mbar_init(&ctl8->vc_full[lane], 1);
      mbar_init(&ctl8->vc_empty[lane], 4);
    } else if (lane == kMaxUnits) {
      mbar_init(&ctl8->q_land, 1);
      mbar_init(&ctl8->q_read, 8);
      mbar_init(&ctl8->sc_ready, 4);
      mbar_init(&ctl8->tree_go, 1);
      mbar_init(&ctl8->q_ready, 8 * PAIR);
    }
    fence_mbar_init();
  }
  setup<PAIR, false, 4>(ctl, warp, lane);
  pdl_launch_dependents();
  bool ok = true;

  if (warp >= kExpandWarp) {
    // ================================ V and the tree in the tensor cores' types ================
    setmaxnreg_dec<kRegsOtherQ8>();
    const int group = warp - kExpandWarp, key = group * 32 + lane;
    pdl_wait();
    if (has_tree) {
      const __nv_bfloat16 *kt = a.Kt + (long long)g * a.tkv_sh, *vt = a.Vt + (long long)g * a.tkv_sh;
      // scales of the tree, a quarter of every group's nodes a warp, ahead of the keys' and values' copies as far as may be
      constexpr int kLanes = D / 8, kStep = 32 / kLanes;
#pragma unroll 1
      for (int q = 0; q * 32 < p.T; ++q) {
        uint32_t km = 0u, vm = 0u;
#pragma unroll
        for (int i = 0; i < 8; i += kStep) {
          const int node = q * 32 + group * 8 + i + lane / kLanes;
          const long long at = (long long)node * a.tkv_st + (lane % kLanes) * 8;
          const uint4 none = make_uint4(0u, 0u, 0u, 0u);
          km = amax_bf16x8(km, node < p.T ? *reinterpret_cast<const uint4*>(kt + at) : none);
          vm = amax_bf16x8(vm, node < p.T ? *reinterpret_cast<const uint4*>(vt + at) : none);
        }
        km = __reduce_max_sync(0xffffffffu, km);
        vm = __reduce_max_sync(0xffffffffu, vm);
        if (lane == 0) ctl8->tree_max[q][group] = make_uint2(km, vm);
      }
      named_bar_sync(1, 128);
      if (key < 4) {
        uint2 m = make_uint2(0u, 0u);
        if (key * 32 < p.T)
          for (int i = 0; i < 4; ++i) m = make_uint2(max(m.x, ctl8->tree_max[key][i].x), max(m.y, ctl8->tree_max[key][i].y));
        const int ke = e4m3_exponent(m.x), ve = f16_exponent(m.y);
        ctl8->tree_k[key] = ke;
        ctl8->tree_v[key] = ve;
        Q8Scales* sc = scales + n_pref;
        reinterpret_cast<float*>(&sc->k)[key] = exp2_int(ke);
        reinterpret_cast<float*>(&sc->v_log2)[key] = (float)ve;
        reinterpret_cast<float*>(&sc->v_inv)[key] = exp2_int(-ve);
      }
    }
    // scales of the run: a thread has a group of a tile (groups behind the prefix have no key and any scale)
    for (int i = key; i < n_pref * 4; i += 128) {
      const int token = min((tile_lo + (i >> 2)) * SPX_TILE_KEYS + (i & 3) * 32, p.L - 1);
      const long long at = (long long)(token >> args.log_block) * args.s_sb + (long long)g * args.s_sh;
      const uint32_t kc = args.Ks[at], vcode = args.Vs[at];
      Q8Scales* sc = scales + (i >> 2);
      reinterpret_cast<float*>(&sc->k)[i & 3] = e8m0_value(kc);
      reinterpret_cast<float*>(&sc->v_log2)[i & 3] = e8m0_log2(vcode);
      reinterpret_cast<float*>(&sc->v_inv)[i & 3] = e8m0_value(vcode == 255u ? 255u : 254u - vcode);
    }
    warp_arrive(&ctl8->sc_ready, lane);
    // (the queries lie where V's stages will be)
    ok = __all_sync(0xffffffffu, mbar_wait(&ctl8->q_read, 0, abort_flag) && mbar_wait(&ctl8->sc_ready, 0, abort_flag));
    int vc = 0, vst = 0;
    uint32_t vcph = 0, vph = 1;
    if (n_pref < kTreeAhead && key == 0) mbar_arrive(&ctl8->tree_go);
    for (int j = 0; j < n_pref && ok; ++j) {
      // (all lanes give up, or none: those that go on meet below)
      ok = __all_sync(0xffffffffu, mbar_wait(&ctl8->vc_full[vc], vcph, abort_flag) && wait_c(&ctl->v_empty[vst], vph, abort_flag));
      if (!ok) break;
      if (j == n_pref - kTreeAhead && key == 0) mbar_arrive(&ctl8->tree_go);
      expand_key<G::kVRow>(base + G::v8_off + vc * G::kVUnit, base + G::v_off + vst * G::kVStage, key);
      publish<PAIR>(&ctl->v_full[vst], lane);
      if (lane == 0) mbar_arrive(&ctl8->vc_empty[vc]);
      if (++vc == G::kVUnits) {
        vc = 0;
        vcph ^= 1;
      }
      if (++vst == G::nv) {
        vst = 0;
        vph ^= 1;
      }
    }
    if (has_tree && ok) {
      // the tree's V, to where it will lie and converted there: f16 has bf16's room
      const __nv_bfloat16* vt = a.Vt + (long long)g * a.tkv_sh + rank * 64;
      ok = __all_sync(0xffffffffu, wait_c(&ctl->v_empty[vst], vph, abort_flag));
      if (ok) {
        constexpr int kLanes = G::kVRow / 8, kStep = 32 / kLanes;          // lanes a node
        const int c = lane % kLanes;
        unsigned char* stage = base + G::v_off + vst * G::kVStage;
        const float f = exp2_int(-ctl8->tree_v[group]);
#pragma unroll 4
        for (int node = group * 32 + lane / kLanes; node < group * 32 + 32; node += kStep)
          copy_node(stage + f16_place(node, c), vt + (node < p.T ? node * a.tkv_st : 0ll) + 8 * c, node < p.T);
        copies_wait();
#pragma unroll 4
        for (int node = group * 32 + lane / kLanes; node < group * 32 + 32; node += kStep) {
          uint4* at = reinterpret_cast<uint4*>(stage + f16_place(node, c));
          *at = bf16x8_to_f16x8(*at, f);
        }
        publish<PAIR>(&ctl->v_full[vst], lane);
      }
    }
    if (*abort_flag) ok = false;
  } else if (warp == kProducerWarp) {
    // ================================ TMA producer of the codes ==============================
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) {
      const uint64_t stream_once = policy_evict_first();
      const uint32_t kbar = leader_addr<PAIR>(&ctl8->k_full[0]), vbar = smem_u32(&ctl8->vc_full[0]);
      const uint32_t kring = smem_u32(base + G::k8_off), vring = smem_u32(base + G::v8_off);
      int ks = 0, vs = 0;
      uint32_t kph = 1, vph = 1;
      for (int j = 0; j < n_pref && ok; ++j) {
        const int key0 = (tile_lo + j) * SPX_TILE_KEYS;
        ok = wait_c(&ctl8->k_empty[ks], kph, abort_flag);
        if (!ok) break;
        arrive_expect_tx_cluster(kbar + ks * 8, G::kKUnit);
        tma_load_hint<PAIR>(kring + ks * G::kKUnit, &maps.k, kbar + ks * 8, 0, g, key0 + rank * (SPX_TILE_KEYS / PAIR), stream_once);
        if (++ks == G::kKUnits) {
          ks = 0;
          kph ^= 1;
        }
        ok = wait_c(&ctl8->vc_empty[vs], vph, abort_flag);
        if (!ok) break;
        arrive_expect_tx_cluster(vbar + vs * 8, G::kVUnit);
        tma_load_hint<1>(vring + vs * G::kVUnit, &maps.v, vbar + vs * 8, rank * 64, g, key0, stream_once);
        if (++vs == G::kVUnits) {
          vs = 0;
          vph ^= 1;
        }
      }
      if (*abort_flag) ok = false;
    }
  } else if (warp == kMmaWarp) {
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();                                          // (a bounded wait must not count the time of the kernel before)
    if (rank == 0) ok = issue_s_q8<PAIR, D>(ctl8, base, n_tiles, has_tree, abort_flag);
  } else if (warp == kPvWarp) {
    setmaxnreg_dec<kRegsOtherQ8>();
    if (lane == 0) {
      // the first tiles are asked for in L2 ahead of the dependency wait, by a thread that has nothing else to do yet
      for (int j = 0; j < min(n_pref, 2); ++j) {
        tma_prefetch_3d(&maps.k, 0, g, (tile_lo + j) * SPX_TILE_KEYS + rank * (SPX_TILE_KEYS / PAIR));
        tma_prefetch_3d(&maps.v, rank * 64, g, (tile_lo + j) * SPX_TILE_KEYS);
      }
    }
    pdl_wait();
    __syncwarp();
    if (rank == 0) ok = issue_pv_q8<PAIR, D>(ctl8, base, n_tiles, abort_flag);
  } else if (warp == kTreeWarp) {
    // ================================ ancestor masks, TMA producer of Q =======================
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) {
      const uint32_t bar = smem_u32(&ctl8->q_land);
      arrive_expect_tx_cluster(bar, 2 * G::kQ);
#pragma unroll
      for (int ds = 0; ds < D / 64; ++ds)
        tma_load<1>(smem_u32(base + G::v_off + ds * 128 * 128), &maps.q, bar, 64 * ds, g * p.G, (rblk * p.RB + rank * 128) / p.G);
    }
    __syncwarp();
    // Masks by doubling: a node's has those of twice as many ancestors after every round.  (Walks up the tree, 32 nodes at a time, took
    // 130 cycles a level: 16 K for a chain of 60 nodes.)
    constexpr int kQ = kSpxMaxTree / 32;
    int up[kQ];                                            // the ancestor that comes next
    unsigned long long lo[kQ], hi[kQ];
    bool bad = false;
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      const int t = lane + 32 * q;
      up[q] = t < p.T ? a.parent[t] : -1;
      if (up[q] < -1 || up[q] >= t) {
        bad = true;
        up[q] = -1;
      }
      ctl->parent[t] = up[q];
      ctl->anc[t][0] = lo[q] = t < 64 ? 1ull << (t & 63) : 0ull;
      ctl->anc[t][1] = hi[q] = t < 64 ? 0ull : 1ull << (t & 63);
    }
    __syncwarp();
#pragma unroll 1
    while (true) {
      int most = -1;
#pragma unroll
      for (int q = 0; q < kQ; ++q) most = max(most, up[q]);
      if (!__any_sync(0xffffffffu, most >= 0)) break;      // (ancestors have lower numbers: at most 7 rounds)
#pragma unroll
      for (int q = 0; q < kQ; ++q)
        if (up[q] >= 0) {
          const int u = up[q];
          lo[q] |= ctl->anc[u][0];
          hi[q] |= ctl->anc[u][1];
          up[q] = ctl->parent[u];
        }
      __syncwarp();
#pragma unroll
      for (int q = 0; q < kQ; ++q) {
        const int t = lane + 32 * q;
        ctl->anc[t][0] = lo[q];
        ctl->anc[t][1] = hi[q];
        ctl->parent[t] = up[q];
      }
      __syncwarp();
    }
    if (bad && blockIdx.x == 0) spx_raise(a.status, SPECEXT_ERR_BAD_TREE);
    warp_arrive(&ctl->anc_ready, lane);
    if (has_tree) {
      // The tree's K is fetched to where it will lie and converted there, row by row: a bf16 row has the bytes of its two parts.  Some tiles
      // ahead of its turn, by this warp, so that nobody waits for it.  (By the expansion's warps behind the prefix, through
      // registers, K and V took 9 K to 14 K cycles during which the other workers were done: a load takes 1.4 K cycles while the cache
      // streams, and few fit in the registers.)
      const __nv_bfloat16* kt = a.Kt + (long long)g * a.tkv_sh;
      ok = mbar_wait(&ctl8->tree_go, 0, abort_flag) && mbar_wait(&ctl8->sc_ready, 0, abort_flag);
      // (PV of tile n_pref - kTreeAhead - nv is done, so no barrier of the ring can be a phase behind the one that is waited for)
      for (int i = 0; i < 2 && ok; ++i)
        ok = wait_c(&ctl8->k_empty[(n_pref + i) % G::kKUnits], (((n_pref + i) / G::kKUnits) & 1) ^ 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        // high and low parts, two units of the ring behind those of the prefix
        unsigned char *k_hi = base + G::k8_off + n_pref % G::kKUnits * G::kKUnit, *k_lo = base + G::k8_off + (n_pref + 1) % G::kKUnits * G::kKUnit;
        constexpr int kLanes = D / 16, kStep = 32 / kLanes, kKeys = SPX_TILE_KEYS / PAIR;      // lanes a key; this CTA's keys
        const int c = lane % kLanes, first = rank * kKeys;
#pragma unroll 4
        for (int row = lane / kLanes; row < kKeys; row += kStep) {
          const bool in = first + row < p.T;
          const __nv_bfloat16* src = kt + (in ? (first + row) * a.tkv_st : 0ll) + 8 * c;
          copy_node(k_hi + code_place<D>(row, c), src, in);
          copy_node(k_lo + code_place<D>(row, c), src + D / 2, in);
        }
        copies_wait();
        __syncwarp();
        // a lane converts pieces 2 c and 2 c + 1 of a row, which lie in the room of the one part or the other (zeros stay)
        const unsigned char* raw = c < kLanes / 2 ? k_hi : k_lo;
        const int c2 = 2 * c % kLanes;
#pragma unroll 2
        for (int row0 = 0; row0 < kKeys && first + row0 < p.T; row0 += kStep) {
          const int row = row0 + lane / kLanes;
          const uint4 x = *reinterpret_cast<const uint4*>(raw + code_place<D>(row, c2)), y = *reinterpret_cast<const uint4*>(raw + code_place<D>(row, c2 + 1));
          __syncwarp();
          split16(x, y, exp2_int(-ctl8->tree_k[(first + row) >> 5]), k_hi + code_place<D>(row, c), k_lo + code_place<D>(row, c));
        }
        for (int i = 0; i < 2; ++i) publish<PAIR>(&ctl8->k_full[(n_pref + i) % G::kKUnits], lane);
      }
    }
    if (*abort_flag) ok = false;
  } else {
    // ================================ softmax warps ===========================================
    setmaxnreg_inc<kRegsSoftmaxQ8>();
    const int quarter = warp & 3;
    RowCtx rc;
    rc.ctl = ctl;
    rc.w = warp >> 2;
    rc.lane = lane;
    rc.row_t = quarter * 32 + lane;
    rc.lane_tmem = ctl->tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    rc.s_free = leader_addr<PAIR>(&ctl->s_free[rc.w]);
    rc.p_full = leader_addr<PAIR>(&ctl->p_full[rc.w]);
    rc.scale2 = p.scale2;
    rc.abort_flag = abort_flag;
    const int rr = rank * 128 + rc.row_t, r = rblk * p.RB + rr;
    const bool valid = r < p.rows, warp_valid = r - lane < p.rows;
    rc.pad = !valid;
    if (!warp_valid) {
      // zeros for the PV MMAs to read there, once
      uint32_t z[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) z[k] = 0u;
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_st16(rc.lane_tmem + kColP + rc.w * 64 + c * 16, z);
      tmem_wait_st();
      tc_fence_before();
    }
    pdl_wait();
    {
      // Query rows, 16 a warp and two lanes a row: their high and low parts, and the power of two.  The loops stay loops: this
      // runs once, and instructions that are not in the cache yet are what it waits for.  (All unrolled, rows in registers
      // straight from memory, it took 5000 to 7000 cycles, with everybody waiting; four warps in loops 5000.)
      const int row = warp * 16 + (lane >> 1), half = lane & 1;
      const unsigned char* q = base + G::v_off;            // (bf16, where V's stages will be)
      uint32_t m = 0u;
      ok = mbar_wait(&ctl8->q_land, 0, abort_flag);
      if (ok) {
#pragma unroll 2
        for (int c = half * (D / 16); c < (half + 1) * (D / 16); ++c) m = amax_bf16x8(m, *reinterpret_cast<const uint4*>(q + f16_place(row, c)));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        const int e = e4m3_exponent(m);
        const float f = exp2_int(-e);
#pragma unroll 1
        for (int c = half * (D / 32); c < (half + 1) * (D / 32); ++c)
          split16(*reinterpret_cast<const uint4*>(q + f16_place(row, 2 * c)), *reinterpret_cast<const uint4*>(q + f16_place(row, 2 * c + 1)),
                  f, base + code_place<D>(row, c), base + G::kQ + code_place<D>(row, c));
        if (half == 0) ctl8->q_scale[row] = exp2_int(e);
      }
      warp_arrive(&ctl8->q_read, lane);
      publish<PAIR>(&ctl8->q_ready, lane);
    }
    const int t_node = valid ? r / p.G : 0;
    float m_loc = -INFINITY, l = 0.f, mult = 0.f;
    bool known = false;                                  // mult is the row's
    for (int j = rc.w; j < n_tiles && ok; j += kWG) {
      if (!warp_valid) {
        ok = skip_tile(rc, j);
        continue;
      }
      const int tile = tile_lo + j;
      const bool is_tree = tile == p.TPH;
      const int nkeys = is_tree ? p.T : min(SPX_TILE_KEYS, p.L - tile * SPX_TILE_KEYS);
      if (!known || is_tree) {
        // (the scores are there, so these have long been; but the row's factor was written by another warp of this CTA, and the way
        // from there to here by q_ready, the leader's products and s_full goes through another CTA and orders no plain stores)
        ok = mbar_wait(&ctl->s_full[rc.w], (j / kWG) & 1, abort_flag) && mbar_wait(&ctl8->sc_ready, 0, abort_flag) &&
             mbar_wait(&ctl8->q_read, 0, abort_flag);
        if (ok && is_tree) ok = mbar_wait(&ctl->anc_ready, 0, abort_flag);
        if (!ok) break;
        mult = p.scale2 * ctl8->q_scale[rc.row_t];
        known = true;
      }
      float cg[4];                                       // sums of the tile's four groups of 32 keys
      float* mass = nullptr;
      long long rowbase = 0;
      if (SCORE != 0 && !is_tree) {
        rowbase = ((long long)prob * p.TPH + tile) * p.RB + rr;
        mass = a.ws + p.off_mass + rowbase * p.CPT;
      }
      ok = softmax_tile_q8<D>(
          rc, scales + j, mult, j, is_tree || nkeys < SPX_TILE_KEYS,
          [&](unsigned long long& lo, unsigned long long& hi) {
            if (is_tree) {                 // this node and its ancestors (a padding row sees key 0)
              lo = valid ? ctl->anc[t_node][0] : 1ull;
              hi = valid ? ctl->anc[t_node][1] : 0ull;
            } else {
              lo = nkeys >= 64 ? ~0ull : ((1ull << nkeys) - 1ull);
              hi = nkeys <= 64 ? 0ull : ((1ull << (nkeys - 64)) - 1ull);
            }
          },
          [&](int c, const uint32_t (&v)[32], float sum, float inv) {
            if (SCORE == 1 || SCORE == 2) {
              cg[c] = sum;
            } else if (SCORE == 3 && mass) {
              float acc = 0.f;
              float* dst = mass + c * (32 / p.C);
#pragma unroll
              for (int k = 0; k < 32; ++k) {
                acc += __uint_as_float(v[k]);
                if (((k + 1) & (p.C - 1)) == 0) {
                  *dst++ = acc * inv;
                  acc = 0.f;
                }
              }
            }
          },
          m_loc, l);
      if (SCORE != 0 && ok && mass) {
        if (SCORE == 1) {
          *reinterpret_cast<float4*>(mass) = make_float4(cg[0], cg[1], cg[2], cg[3]);
        } else if (SCORE == 2) {
          if (p.C == 64)
            *reinterpret_cast<float2*>(mass) = make_float2(cg[0] + cg[1], cg[2] + cg[3]);
          else
            *mass = (cg[0] + cg[1]) + (cg[2] + cg[3]);
        }
        a.ws[p.off_mref + rowbase] = m_loc;
      }
    }
    // ---- unnormalised O, reference maximum and row sum to the partial slot ----
    float m_fin, l_tot;
    if (ok) ok = segment_end(rc, n_tiles - 1, 0, m_loc, l, m_fin, l_tot);
    if (ok && warp_valid) {
      const int slot = worker + prob;
      float* po = a.ws + p.off_part_o + (long long)slot * (D / 4) * p.RB * 4;
      constexpr int kGroups = D / 16 / kWG;
      const int c_lo = rc.w * kGroups;
#pragma unroll
      for (int c = 0; c < kGroups; ++c) {
        uint32_t v[16];
        tmem_ld16(rc.lane_tmem + kColO + (c_lo + c) * 16, v);
        tmem_wait_ld();
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const float4 x = make_float4(__uint_as_float(v[q4 * 4]), __uint_as_float(v[q4 * 4 + 1]),
                                       __uint_as_float(v[q4 * 4 + 2]), __uint_as_float(v[q4 * 4 + 3]));
          if (valid) *reinterpret_cast<float4*>(po + ((long long)((c_lo + c) * 4 + q4) * p.RB + rr) * 4) = x;
        }
      }
      if (rc.w == 0 && valid) {
        a.ws[p.off_part_m + (long long)slot * p.RB + rr] = m_fin;
        a.ws[p.off_part_l + (long long)slot * p.RB + rr] = l_tot;
      }
    }
  }

  if (!ok) {
    if (lane == 0) spx_raise(a.status, SPECEXT_ERR_TIMEOUT);
    settle();
  }
  finish<PAIR>(ctl, warp);
}

template <int PAIR, int D, int SCORE>
cudaError_t launch(const Q8Args& q, const Q8Maps& maps, cudaStream_t st) {
  static SpxOncePerDevice once;
  constexpr int smem = smem_q8<PAIR, D>();
  static_assert(smem <= 232448, "more shared memory than a CTA can have");
  const cudaError_t ec = spx_opt_in_smem(verify_q8_kernel<PAIR, D, SCORE>, smem, &once);
  if (ec != cudaSuccess) return ec;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(q.a.plan.n_cta * PAIR);
  cfg.blockDim = dim3(kThreadsQ8);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = PAIR;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR == 2 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, verify_q8_kernel<PAIR, D, SCORE>, q, maps);
}

template <int PAIR, int D>
cudaError_t launch_class(const Q8Args& q, const Q8Maps& maps, cudaStream_t st) {
  const AttnPlan& p = q.a.plan;
  if (!p.want_score) return launch<PAIR, D, 0>(q, maps, st);
  return p.C == 32  ? launch<PAIR, D, 1>(q, maps, st)
         : p.C > 32 ? launch<PAIR, D, 2>(q, maps, st)
                    : launch<PAIR, D, 3>(q, maps, st);
}

}  // namespace

// Row blocks of 128, or of 256 on pairs of CTAs (plan.RB); plan.n_cta counts CTAs, or pairs.
cudaError_t spx_launch_verify_q8(const Q8Args& q, cudaStream_t st, int* n_launches) {
  const AttnArgs& a = q.a;
  const AttnPlan& p = a.plan;
  const bool pair = p.RB == 256;
  Q8Maps maps;
  bool ok = spx_encode_map(&maps.q, a.Q, p.D, p.Hq, a.q_sh, p.T, a.q_st, p.G, 128 / p.G);
  if (p.L > 0) {
    ok = ok && spx_encode_map8(&maps.k, q.Kc, p.D, p.Hkv, a.kv_sh, p.L, a.kv_sl, p.D, pair ? SPX_TILE_KEYS / 2 : SPX_TILE_KEYS);
    ok = ok && spx_encode_map8(&maps.v, q.Vc, p.D, p.Hkv, a.kv_sh, p.L, a.kv_sl, pair ? 64 : p.D, SPX_TILE_KEYS);
  } else {
    maps.k = maps.v = maps.q;                            // never used
  }
  if (!ok) return cudaErrorInvalidValue;
  *n_launches += 1;
  if (pair) return launch_class<2, 128>(q, maps, st);
  return p.D == 128 ? launch_class<1, 128>(q, maps, st) : launch_class<1, 64>(q, maps, st);
}
