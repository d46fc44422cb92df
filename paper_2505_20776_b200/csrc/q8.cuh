// What the kernels of the 8-bit cache share.
//
// A cached value is code * 2^(scale - 127): the code is e4m3 (4 significant bits), the scale e8m0, one byte for each block of
// B tokens and head.  A power of two costs e4m3 no precision, lets a block's scale grow without a second rounding, and makes
// every product with it exact.
#ifndef SPECEXT_Q8_CUH_
#define SPECEXT_Q8_CUH_

#include "common.cuh"

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
  return code == 255u ? __uint_as_float(0x7fc00000u) : (float)((int)code - 127);
}

// Two e4m3 codes as two f16 values: every e4m3 value is one.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)codes));
  return r;
}

cudaError_t spx_launch_verify_q8(const Q8Args& q, cudaStream_t st, int* n_launches);

#endif  // SPECEXT_Q8_CUH_
