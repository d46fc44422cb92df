// Hybrid Tree Attention over a prefix cache in 8 bits (codes e4m3, scales e8m0, see q8.cuh), on the pipeline of core.cuh with one
// CTA per worker: partial attention of 128 stacked (query head x tree node) rows of one KV head against a run of 128-key tiles.
//
// The tensor cores multiply f16.  e4m3 values are f16 values, so a tile is expanded by one conversion per two codes and no
// rounding; bf16 would take four integer instructions and a multiplication (a conversion and an integer instruction cost the
// same two cycles a warp, and the expansion is what this kernel does more of than the one for bf16).  The scales stay outside:
//   S = (q 2^-e) . k_code                          e: the row's own power of two, so that bf16 queries are exact in f16
//   z = S * (scale log2(e) 2^e k_scale) + log2(v_scale)
//   P = 2^(z - M) rounded to f16,  O += P v_code,  l += 2^(z - M) / v_scale
// with M the reference maximum of z: the V scale rides on the exponent, at no cost per element, and P stays in f16's range
// whatever the scales are.  M is 2^6 below the maximum it was taken from and may fall 2^8 more behind, so P is at most 2^14;
// f16 keeps 11 bits down to 2^-20 of the row's largest weight and reaches 2^-30.
// The tree's bf16 keys and values become f16 with a power of two for each group of 32 (finite values decide it).
//
// Warps: 0-7 softmax, 8 TMA producer of the codes, 9 issuer of the S MMAs, 10 of the PV MMAs, 11 ancestor masks and TMA
// producer of Q, 12-15 expansion (a thread has a key: codes from the staging ring, f16 into the K or V stage; Q, a thread has a
// row, in place).  Every wait is bounded; all threads reach the final barrier before tensor memory is freed.
#include <cstddef>

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
constexpr int kMaxUnits = 8, kScaleSlots = 8;

struct Q8Maps {
  CUtensorMap q, k, v;
};

// Shared memory: Q | K stages | V stages (f16) | staging ring of code tiles | control.
template <int D>
struct GeoQ8 {
  static constexpr int kBlocks = D / 64;
  static constexpr int kKBlk = SPX_TILE_KEYS * 128, kVBlk = kKBlk;
  static constexpr int kKStage = kKBlk * kBlocks, kVStage = kKStage;
  static constexpr int q_blk = 128 * 128;
  static constexpr int nk = D == 128 ? 2 : 3, nv = nk;
  static constexpr uint32_t k_off = q_blk * kBlocks, v_off = k_off + nk * kKStage;
  static constexpr uint32_t st_off = v_off + nv * kVStage;
  static constexpr int kUnit = SPX_TILE_KEYS * D, kUnits = D == 128 ? 3 : 8;
  static constexpr int kCtrl = st_off + kUnits * kUnit;
};

// Scales of a tile, per group of 32 keys.
struct alignas(16) Q8Scales {
  float k[4], v_log2[4], v_inv[4];
};
struct CtrlQ8 {
  Ctrl c;
  uint64_t st_full[kMaxUnits], st_empty[kMaxUnits];
  uint64_t q_land;
  // by tile, modulo kScaleSlots: tile t + 8 is expanded only after the S MMA of tile t + 6, hence after the warpgroup of tile t
  // has taken the scores of tile t + 4
  Q8Scales sc[kScaleSlots];
  float q_scale[128];
};
constexpr int kCtrlBytesQ8 = 8192;
static_assert(sizeof(CtrlQ8) <= kCtrlBytesQ8, "control block too large");
static_assert(sizeof(Q8Scales) == 48 && offsetof(CtrlQ8, sc) % 16 == 0, "scales are read as float4");
static_assert(GeoQ8<64>::kCtrl % 1024 == 0 && GeoQ8<128>::kCtrl % 1024 == 0, "stages begin on 1024 bytes");
template <int D>
constexpr int smem_q8() {
  return GeoQ8<D>::kCtrl + kCtrlBytesQ8 + 1024;
}

// A worker has one run of tiles of one problem.
struct OneRun {
  int n;
  bool done;
  __device__ __forceinline__ bool next() {
    const bool first = !done;
    done = true;
    return first;
  }
};

// Place of 16-byte column `col` (of D * 2 / 16) of row `row` in a K or V stage, or in Q: blocks of 64 elements, 128-byte swizzle.
__device__ __forceinline__ int f16_place(int row, int col) { return (col >> 3) * (128 * 128) + row * 128 + (((col ^ row) & 7) << 4); }

// One key's codes from a staged tile (rows of D bytes, swizzled as TMA left them) as f16 into a stage.
template <int D>
__device__ __forceinline__ void expand_key(const unsigned char* unit, unsigned char* stage, int key) {
#pragma unroll 4
  for (int c = 0; c < D / 16; ++c) {
    const int at = D == 128 ? c ^ (key & 7) : c ^ ((key >> 1) & 3);
    const uint4 x = *reinterpret_cast<const uint4*>(unit + key * D + (at << 4));
    *reinterpret_cast<uint4*>(stage + f16_place(key, 2 * c)) =
        make_uint4(e4m3x2_to_f16x2(x.x), e4m3x2_to_f16x2(x.x >> 16), e4m3x2_to_f16x2(x.y), e4m3x2_to_f16x2(x.y >> 16));
    *reinterpret_cast<uint4*>(stage + f16_place(key, 2 * c + 1)) =
        make_uint4(e4m3x2_to_f16x2(x.z), e4m3x2_to_f16x2(x.z >> 16), e4m3x2_to_f16x2(x.w), e4m3x2_to_f16x2(x.w >> 16));
  }
}

// The power of two that takes the bf16 keys or values of a warp's 32 tree nodes to f16 (a lane has one; its row of D).
template <int D>
__device__ __forceinline__ int tree_exponent(const __nv_bfloat16* src, bool valid) {
  uint32_t m = 0u;
  const uint4* row = reinterpret_cast<const uint4*>(src);
#pragma unroll 4
  for (int c = 0; c < D / 8; ++c) {
    const uint4 x = valid ? row[c] : make_uint4(0u, 0u, 0u, 0u);
    m = amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(m, x.x), x.y), x.z), x.w);
  }
  return f16_exponent(__reduce_max_sync(0xffffffffu, m));
}
// One tree node's key or value as f16 into a stage.
template <int D>
__device__ __forceinline__ void expand_node(const __nv_bfloat16* src, bool valid, unsigned char* stage, int key, float f) {
  const uint4* row = reinterpret_cast<const uint4*>(src);
#pragma unroll 4
  for (int c = 0; c < D / 8; ++c)
    *reinterpret_cast<uint4*>(stage + f16_place(key, c)) = bf16x8_to_f16x8(valid ? row[c] : make_uint4(0u, 0u, 0u, 0u), f);
}

// softmax_tile of core.cuh with scales: `mult` is the row's factor (softmax scale, log2 e, the power of two of the query row).
template <int D, class MaskFn, class SumFn>
__device__ __forceinline__ bool softmax_tile_q8(const RowCtx& rc, const Q8Scales* sc, float mult, uint32_t t, bool need_mask,
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
  const float4 ks = *reinterpret_cast<const float4*>(sc->k), ev = *reinterpret_cast<const float4*>(sc->v_log2);
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
  const float f0 = mult * ks.x, f1 = mult * ks.y, f2 = mult * ks.z, f3 = mult * ks.w;
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
    const float inv = sc->v_inv[c], gs = ((gs0 + gs1) + (gs2 + gs3)) * inv;
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
template <int D, int SCORE>
__global__ void __launch_bounds__(kThreadsQ8, 1)
verify_q8_kernel(const __grid_constant__ Q8Args args, const __grid_constant__ Q8Maps maps) {
  using G = GeoQ8<D>;
  const AttnArgs& a = args.a;
  const AttnPlan& p = a.plan;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                         ~static_cast<uintptr_t>(1023));
  CtrlQ8* ctl8 = reinterpret_cast<CtrlQ8*>(base + G::kCtrl);
  Ctrl* ctl = &ctl8->c;
  volatile int* abort_flag = &ctl->abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const G geo;

  const int worker = blockIdx.x, prob = worker / p.cpp;
  const int unit_lo = spx_unit_start(p, worker), n_tiles = spx_unit_start(p, worker + 1) - unit_lo;
  const int tile_lo = unit_lo - prob * p.UPP, g = prob / p.n_rblk, rblk = prob - g * p.n_rblk;
  if (warp == kTreeWarp) {
    if (lane < kMaxUnits) {
      mbar_init(&ctl8->st_full[lane], 1);
      mbar_init(&ctl8->st_empty[lane], 4);
    } else if (lane == kMaxUnits) {
      mbar_init(&ctl8->q_land, 1);
    }
    fence_mbar_init();
  }
  setup<1, false, 4>(ctl, warp, lane);
  pdl_launch_dependents();
  bool ok = true;
  OneRun work{n_tiles, false};

  if (warp >= kExpandWarp) {
    // ================================ expansion to f16 ========================================
    setmaxnreg_dec<kRegsOtherQ8>();
    const int group = warp - kExpandWarp, key = group * 32 + lane;
    auto scale_of = [&](const uint8_t* s, int tile) -> uint32_t {
      const int token = tile * SPX_TILE_KEYS + group * 32;
      return tile < p.TPH && token < p.L ? s[(long long)(token >> args.log_block) * args.s_sb + (long long)g * args.s_sh] : 127u;
    };
    pdl_wait();
    uint32_t ks = scale_of(args.Ks, tile_lo), vs = scale_of(args.Vs, tile_lo);
    ok = mbar_wait(&ctl8->q_land, 0, abort_flag);
    if (ok) {
      uint32_t m = 0u;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        const uint4 x = *reinterpret_cast<const uint4*>(base + f16_place(key, c));
        m = amax_bf16x2(amax_bf16x2(amax_bf16x2(amax_bf16x2(m, x.x), x.y), x.z), x.w);
      }
      const int e = f16_exponent(m);
      const float f = exp2_int(-e);
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        uint4* x = reinterpret_cast<uint4*>(base + f16_place(key, c));
        *x = bf16x8_to_f16x8(*x, f);
      }
      ctl8->q_scale[key] = exp2_int(e);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      warp_arrive(&ctl->q_full, lane);
    }
    int st = 0, kst = 0, vst = 0;
    uint32_t stph = 0, kph = 1, vph = 1;
    for (int j = 0; j < n_tiles && ok; ++j) {
      const int tile = tile_lo + j;
      const bool is_tree = tile == p.TPH, node = key < p.T;
      Q8Scales* sc = &ctl8->sc[j & (kScaleSlots - 1)];
      const uint32_t ks_next = scale_of(args.Ks, tile + 1), vs_next = scale_of(args.Vs, tile + 1);
      const long long node_at = (long long)key * a.tkv_st + (long long)g * a.tkv_sh;
      int ke = 0, ve = 0;
      if (is_tree) {
        ke = tree_exponent<D>(a.Kt + node_at, node);
        ve = tree_exponent<D>(a.Vt + node_at, node);
      }
#pragma unroll 1
      for (int half = 0; half < 2 && ok; ++half) {
        // K, then V
        uint64_t* full = half ? &ctl->v_full[vst] : &ctl->k_full[kst];
        unsigned char* stage = base + (half ? G::v_off + vst * G::kVStage : G::k_off + kst * G::kKStage);
        if (!is_tree) ok = mbar_wait(&ctl8->st_full[st], stph, abort_flag);
        if (ok) ok = half ? wait_c(&ctl->v_empty[vst], vph, abort_flag) : wait_c(&ctl->k_empty[kst], kph, abort_flag);
        if (!ok) break;
        // (the scales of K and of V: both are read as soon as the tile's scores are there)
        if (lane == 0 && half == 0) {
          sc->k[group] = is_tree ? exp2_int(ke) : e8m0_value(ks);
          sc->v_log2[group] = is_tree ? (float)ve : e8m0_log2(vs);
          sc->v_inv[group] = is_tree ? exp2_int(-ve) : e8m0_value(vs == 255u ? 255u : 254u - vs);
        }
        if (is_tree) expand_node<D>((half ? a.Vt : a.Kt) + node_at, node, stage, key, exp2_int(half ? -ve : -ke));
        else expand_key<D>(base + G::st_off + st * G::kUnit, stage, key);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        warp_arrive(full, lane);
        if (!is_tree) {
          if (lane == 0) mbar_arrive(&ctl8->st_empty[st]);
          if (++st == G::kUnits) {
            st = 0;
            stph ^= 1;
          }
        }
      }
      if (++kst == G::nk) {
        kst = 0;
        kph ^= 1;
      }
      if (++vst == G::nv) {
        vst = 0;
        vph ^= 1;
      }
      ks = ks_next;
      vs = vs_next;
    }
    if (*abort_flag) ok = false;
  } else if (warp == kProducerWarp) {
    // ================================ TMA producer of the codes ==============================
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) {
      const uint64_t stream_once = policy_evict_first();
      const uint32_t full0 = smem_u32(&ctl8->st_full[0]), ring = smem_u32(base + G::st_off);
      int st = 0;
      uint32_t ph = 1;
      for (int u = 0; u < 2 * n_tiles && ok; ++u) {
        const int tile = tile_lo + (u >> 1);
        if (tile == p.TPH) break;                        // the tree's keys and values are not staged
        ok = wait_c(&ctl8->st_empty[st], ph, abort_flag);
        if (!ok) break;
        arrive_expect_tx_cluster(full0 + st * 8, G::kUnit);
        tma_load_hint<1>(ring + st * G::kUnit, u & 1 ? &maps.v : &maps.k, full0 + st * 8, 0, g, tile * SPX_TILE_KEYS, stream_once);
        if (++st == G::kUnits) {
          st = 0;
          ph ^= 1;
        }
      }
      if (*abort_flag) ok = false;
    }
  } else if (warp == kMmaWarp) {
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) ok = issue_s<1, D, true>(ctl, base, geo, work, abort_flag);
  } else if (warp == kPvWarp) {
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) ok = issue_pv<1, D, true>(ctl, base, geo, work, abort_flag);
  } else if (warp == kTreeWarp) {
    // ================================ ancestor masks, TMA producer of Q =======================
    setmaxnreg_dec<kRegsOtherQ8>();
    pdl_wait();
    if (lane == 0) {
      const uint32_t bar = smem_u32(&ctl8->q_land);
      arrive_expect_tx_cluster(bar, G::q_blk * G::kBlocks);
#pragma unroll
      for (int ds = 0; ds < G::kBlocks; ++ds)
        tma_load<1>(smem_u32(base + ds * G::q_blk), &maps.q, bar, 64 * ds, g * p.G, rblk * p.RB / p.G);
    }
    __syncwarp();
#pragma unroll
    for (int q = 0; q < kSpxMaxTree / 32; ++q) ctl->parent[lane + 32 * q] = lane + 32 * q < p.T ? a.parent[lane + 32 * q] : -1;
    __syncwarp();
    bool bad = false;
#pragma unroll 1
    for (int q = 0; q < kSpxMaxTree / 32; ++q) {
      const int t = lane + 32 * q;
      SpxMask128 m = {0ull, 0ull};
      if (t < p.T) m = spx_walk_up(ctl->parent, p.T, t, bad);
      ctl->anc[t][0] = m.lo;
      ctl->anc[t][1] = m.hi;
    }
    if (bad && blockIdx.x == 0) spx_raise(a.status, SPECEXT_ERR_BAD_TREE);
    warp_arrive(&ctl->anc_ready, lane);
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
    rc.s_free = smem_u32(&ctl->s_free[rc.w]);
    rc.p_full = smem_u32(&ctl->p_full[rc.w]);
    rc.scale2 = p.scale2;
    rc.abort_flag = abort_flag;
    const int rr = rc.row_t, r = rblk * p.RB + rr;
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
      if (is_tree) {
        ok = mbar_wait(&ctl->anc_ready, 0, abort_flag);
        if (!ok) break;
      }
      if (!known) {
        ok = mbar_wait(&ctl->q_full, 0, abort_flag);
        if (!ok) break;
        mult = p.scale2 * ctl8->q_scale[rr];
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
          rc, &ctl8->sc[j & (kScaleSlots - 1)], mult, j, is_tree || nkeys < SPX_TILE_KEYS,
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
  finish<1>(ctl, warp);
}

template <int D, int SCORE>
cudaError_t launch(const Q8Args& q, const Q8Maps& maps, cudaStream_t st) {
  static SpxOncePerDevice once;
  constexpr int smem = smem_q8<D>();
  static_assert(smem <= 232448, "more shared memory than a CTA can have");
  const cudaError_t ec = spx_opt_in_smem(verify_q8_kernel<D, SCORE>, smem, &once);
  if (ec != cudaSuccess) return ec;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(q.a.plan.n_cta);
  cfg.blockDim = dim3(kThreadsQ8);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_q8_kernel<D, SCORE>, q, maps);
}

template <int D>
cudaError_t launch_class(const Q8Args& q, const Q8Maps& maps, cudaStream_t st) {
  const AttnPlan& p = q.a.plan;
  if (!p.want_score) return launch<D, 0>(q, maps, st);
  return p.C == 32 ? launch<D, 1>(q, maps, st) : p.C > 32 ? launch<D, 2>(q, maps, st) : launch<D, 3>(q, maps, st);
}

}  // namespace

cudaError_t spx_launch_verify_q8(const Q8Args& q, cudaStream_t st, int* n_launches) {
  const AttnArgs& a = q.a;
  const AttnPlan& p = a.plan;
  Q8Maps maps;
  bool ok = spx_encode_map(&maps.q, a.Q, p.D, p.Hq, a.q_sh, p.T, a.q_st, p.G, 128 / p.G);
  if (p.L > 0) {
    ok = ok && spx_encode_map8(&maps.k, q.Kc, p.D, p.Hkv, a.kv_sh, p.L, a.kv_sl, p.D, SPX_TILE_KEYS);
    ok = ok && spx_encode_map8(&maps.v, q.Vc, p.D, p.Hkv, a.kv_sh, p.L, a.kv_sl, p.D, SPX_TILE_KEYS);
  } else {
    maps.k = maps.v = maps.q;                            // never used
  }
  if (!ok) return cudaErrorInvalidValue;
  *n_launches += 1;
  return p.D == 128 ? launch_class<128>(q, maps, st) : launch_class<64>(q, maps, st);
}
