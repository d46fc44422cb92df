// Tokens into the 8-bit cache (see q8.cuh): bf16 keys and values become e4m3 codes with an e8m0 scale per block of B tokens and
// head.  The scale is the smallest power of two s with max |x| <= 448 s over the block's new tokens (448 is e4m3's largest
// value), found from the exponent and mantissa bits of the maximum; dividing by it is exact, so a value is rounded once.  A block
// that the first new token falls into the middle of keeps its scale or gets a larger one; the codes before are then multiplied by
// the ratio of both, a power of two, which rounds only what falls among e4m3's subnormals.
//
// What bounds it: memory for prompts, latency for the few tokens of a decoding step.  A thread block has one block of one head
// of K or V, all of it in registers between the maximum and the rounding, so everything is read and written once.  Replayed, 8 heads
// of 128: 60 tokens 1.8 us, 2000 4.9, 16384 17.4 (5.8 TB/s of reads and writes), 131072 117 (6.9).
#include "q8.cuh"
#include "sm100.cuh"

using namespace sm100;

namespace {

struct QuantArgs {
  const __nv_bfloat16 *K, *V;
  uint8_t *Kc, *Vc, *Ks, *Vs;
  const int32_t* rows;                          // source row of each token, or null: token i is row i
  int32_t* status;
  long long x_sl, x_sh, c_sl, c_sh, s_sb, s_sh;
  int start, n, n_src, n_heads, log_block;
};

constexpr int kPerThread = 4;                   // pieces of 16 values a thread holds
constexpr uint32_t kScaleFloor = 27;            // 2^-100: of a block of zeros

// The scale of a block whose largest magnitude has these bits.
__device__ __forceinline__ uint32_t scale_code(uint32_t amax_bits) {
  const uint32_t e = (amax_bits >> 23) + ((amax_bits & 0x7fffffu) > 0x600000u ? 1u : 0u);      // 448 = 1.75 * 2^8
  return e < kScaleFloor + 8 ? kScaleFloor : e - 8;
}

__device__ __forceinline__ uint32_t bf16x4_to_e4m3x4(uint32_t a, uint32_t b, float f) {
  return f32x2_to_e4m3x2(__uint_as_float(a << 16) * f, __uint_as_float(a & 0xffff0000u) * f) |
         (f32x2_to_e4m3x2(__uint_as_float(b << 16) * f, __uint_as_float(b & 0xffff0000u) * f) << 16);
}
// Four codes times f.
__device__ __forceinline__ uint32_t scaled_e4m3x4(uint32_t codes, float f) {
  const float2 x = f16x2_to_f32x2(e4m3x2_to_f16x2(codes)), y = f16x2_to_f32x2(e4m3x2_to_f16x2(codes >> 16));
  return f32x2_to_e4m3x2(x.x * f, x.y * f) | (f32x2_to_e4m3x2(y.x * f, y.y * f) << 16);
}
// The larger magnitudes, half by half: bf16 without its sign orders as an integer does, infinities and NaN above all.
__device__ __forceinline__ uint32_t magnitudes(uint32_t m, uint4 x) {
  m = __vmaxu2(__vmaxu2(m, x.x & 0x7fff7fffu), x.y & 0x7fff7fffu);
  return __vmaxu2(__vmaxu2(m, x.z & 0x7fff7fffu), x.w & 0x7fff7fffu);
}

// grid: (heads of every block touched, the head varying fastest; K and V); block: B * D / 64 threads.
template <int D>
__global__ void __launch_bounds__(256) quantize_kernel(const __grid_constant__ QuantArgs q) {
  constexpr int kCols = D / 16;
  __shared__ uint32_t warp_max[8];
  pdl_launch_dependents();
  const int nth = (int)blockIdx.x / q.n_heads, h = (int)blockIdx.x - nth * q.n_heads;
  const int block = (q.start >> q.log_block) + nth, B = 1 << q.log_block;
  const __nv_bfloat16* x = blockIdx.y ? q.V : q.K;
  uint8_t* codes = (blockIdx.y ? q.Vc : q.Kc) + (long long)h * q.c_sh;
  uint8_t* scale = (blockIdx.y ? q.Vs : q.Ks) + (long long)block * q.s_sb + (long long)h * q.s_sh;
  const int token0 = block << q.log_block;       // (at most 2^24)
  const int lead = max(q.start - token0, 0), end = min(B, q.start + q.n - token0);      // new tokens: [lead, end) of the block
  pdl_wait();
  const uint32_t old = lead > 0 ? *scale : 0u;
  uint4 v[kPerThread][2];
  bool outside = false;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int i = threadIdx.x + k * blockDim.x, t = i / kCols, c = i % kCols;
    v[k][0] = v[k][1] = make_uint4(0u, 0u, 0u, 0u);
    if (t >= lead && t < end) {
      int row = token0 + t - q.start;
      if (q.rows) row = q.rows[row];
      if (row >= 0 && row < q.n_src) {
        const uint4* src = reinterpret_cast<const uint4*>(x + (long long)row * q.x_sl + (long long)h * q.x_sh + c * 16);
        v[k][0] = src[0];
        v[k][1] = src[1];
      } else {
        outside = true;
      }
    }
  }
  uint32_t m2 = 0u;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) m2 = magnitudes(magnitudes(m2, v[k][0]), v[k][1]);
  uint32_t m = __reduce_max_sync(0xffffffffu, max(m2 << 16, m2 & 0xffff0000u));
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
  for (int i = 0; i < (int)blockDim.x >> 5; ++i) m = max(m, warp_max[i]);
  if (outside) spx_raise(q.status, SPECEXT_ERR_INVALID_ARG);
  // a NaN or infinity (exponent 255) makes the block NaN, and so it stays; its codes are left as they are
  const uint32_t code = m >= 0x7f800000u || old == 255u ? 255u : max(scale_code(m), old);
  if (threadIdx.x == 0) *scale = (uint8_t)code;
  if (code == 255u) return;
  const float f = __uint_as_float((254u - code) << 23);      // 2^(127 - code), code in [27, 247]
  const bool grown = lead > 0 && code != old;
  const int down = (int)code - (int)old;          // (by 2^127 and more nothing is left)
  const float ratio = grown && down < 127 ? __uint_as_float((uint32_t)(127 - down) << 23) : 0.f;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int i = threadIdx.x + k * blockDim.x, t = i / kCols, c = i % kCols;
    uint4* dst = reinterpret_cast<uint4*>(codes + (long long)(token0 + t) * q.c_sl + c * 16);
    if (t >= lead && t < end) {
      *dst = make_uint4(bf16x4_to_e4m3x4(v[k][0].x, v[k][0].y, f), bf16x4_to_e4m3x4(v[k][0].z, v[k][0].w, f),
                        bf16x4_to_e4m3x4(v[k][1].x, v[k][1].y, f), bf16x4_to_e4m3x4(v[k][1].z, v[k][1].w, f));
    } else if (t < lead && grown) {
      const uint4 o = *dst;
      *dst = make_uint4(scaled_e4m3x4(o.x, ratio), scaled_e4m3x4(o.y, ratio), scaled_e4m3x4(o.z, ratio), scaled_e4m3x4(o.w, ratio));
    }
  }
}

}  // namespace

cudaError_t spx_launch_quantize(const void* K, const void* V, int n_kv_heads, int head_dim, long long x_sl, long long x_sh,
                                const int32_t* rows, int n_src, int n, int start, void* Kc, void* Vc, long long c_sl,
                                long long c_sh, void* Ks, void* Vs, long long s_sb, long long s_sh, int log_block,
                                int32_t* status, cudaStream_t st) {
  QuantArgs q;
  q.K = static_cast<const __nv_bfloat16*>(K); q.V = static_cast<const __nv_bfloat16*>(V);
  q.Kc = static_cast<uint8_t*>(Kc); q.Vc = static_cast<uint8_t*>(Vc);
  q.Ks = static_cast<uint8_t*>(Ks); q.Vs = static_cast<uint8_t*>(Vs);
  q.rows = rows; q.status = status;
  q.x_sl = x_sl; q.x_sh = x_sh; q.c_sl = c_sl; q.c_sh = c_sh; q.s_sb = s_sb; q.s_sh = s_sh;
  q.start = start; q.n = n; q.n_src = n_src; q.n_heads = n_kv_heads; q.log_block = log_block;
  const int first = start >> log_block, last = (start + n - 1) >> log_block;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_kv_heads * (unsigned)(last - first + 1), 2);
  cfg.blockDim = dim3((head_dim << log_block) / (16 * kPerThread));
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return head_dim == 128 ? cudaLaunchKernelEx(&cfg, quantize_kernel<128>, q) : cudaLaunchKernelEx(&cfg, quantize_kernel<64>, q);
}
