// What the kernels of the 8-bit cache share.
//
// A cached value is code * 2^(scale - 127): the code is e4m3 (4 significant bits), the scale e8m0, one byte for each block of
// B tokens and head.  A power of two costs e4m3 no precision, lets a block's scale grow without a second rounding, and makes
// every product with it exact.
#ifndef SPECEXT_Q8_CUH_
#define SPECEXT_Q8_CUH_

#include <cuda_fp16.h>

#include "common.cuh"
#include "sm100.cuh"

struct Q8Args {
  AttnArgs a;                                   // (Kp, Vp unused)
  const uint8_t *Kc, *Vc;                       // codes [>=L][Hkv][D], byte strides a.kv_sl, a.kv_sh
  const uint8_t *Ks, *Vs;                       // scales [>=ceil(L/B)][Hkv]
  long long s_sb, s_sh;
  int log_block;                                // B = 32, 64 or 128 tokens
};

// e8m0: 2^(code - 127); 255 is NaN.  (Code 0, which no written block has, is a subnormal and counts as zero.)
__device__ __forceinline__ float e8m0_value(uint32_t code) {
  return __uint_as_float(code == 255u ? 0x7fc00000u : code << 23);
}
__device__ __forceinline__ float e8m0_log2(uint32_t code) {
  // (2^23 + code, less 2^23 + 127: an integer conversion takes longer)
  return code == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x4b000000u | code) - 8388735.0f;
}

// Two e4m3 codes as two f16 values: every e4m3 value is one.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)codes));
  return r;
}

// bf16 values go to f16 with a power of two 2^-e: the e for which the largest finite magnitude `amax` (bits of a non-negative
// float) comes to lie in [2^14, 2^15); 0 for zeros.
__device__ __forceinline__ int f16_exponent(uint32_t amax) {
  const int e = (int)(amax >> 23) - 127 - 14;
  return amax == 0u ? 0 : max(e, -126);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }    // -126 <= e <= 127

// Magnitude bits of the two bf16 of a word as floats, non-finite ones as zero; the larger of both and `m`.
__device__ __forceinline__ uint32_t amax_bf16x2(uint32_t m, uint32_t w) {
  uint32_t lo = (w << 16) & 0x7fffffffu, hi = w & 0x7fff0000u;
  if (lo >= 0x7f800000u) lo = 0u;
  if (hi >= 0x7f800000u) hi = 0u;
  return max(m, max(lo, hi));
}
__device__ __forceinline__ uint32_t bf16x2_to_f16x2(uint32_t w, float f) {
  return sm100::pack_f16x2(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
}
__device__ __forceinline__ uint4 bf16x8_to_f16x8(uint4 x, float f) {
  return make_uint4(bf16x2_to_f16x2(x.x, f), bf16x2_to_f16x2(x.y, f), bf16x2_to_f16x2(x.z, f), bf16x2_to_f16x2(x.w, f));
}

// Two floats as e4m3, rounded to nearest even; |x| <= 448.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t f16x2_to_e4m3x2(uint32_t x) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

constexpr int kSpxRunQ8 = 144;                      // tiles of a worker's run (their scales are kept in shared memory)
cudaError_t spx_launch_verify_q8(const Q8Args& q, cudaStream_t st, int* n_launches);      // any rows, chunk sums
cudaError_t spx_launch_rows_q8(const Q8Args& q, cudaStream_t st, int* n_launches);        // row blocks of 8 or 16, no chunk sums
int spx_rows_q8_max_clusters(int dev, int size);

#endif  // SPECEXT_Q8_CUH_
