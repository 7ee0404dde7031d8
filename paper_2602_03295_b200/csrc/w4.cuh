// 4-bit weights (internal): arguments of their product with few rows. The layout is stated in pop_kernels.h.
#pragma once
#include "common.cuh"

#include <cuda_fp16.h>

namespace pop {

struct Gemv4Args {
  const bf16* x; int64_t ldx;                          // [B][ldx]
  const uint8_t* codes;                                // [N / 16][K / 128][16][64]
  const bf16* scales;                                  // [N / 16][K / 128][16][128 / group]
  const uint8_t* zeros;                                // like the scales, or null: 8
  int group;
  void* out; int64_t ldo;                              // mode 0: fp32 store; 2: fp32 +=; 3: gated -> bf16 [B][n_valid]
  int B, N, K, mode, act, n_valid;
  void* workspace; size_t workspace_bytes;             // see pop_k_gemv_w4_workspace_bytes
};
size_t gemv4_workspace_bytes(int B, int N, int K, int group);
int launch_gemv4(const Gemv4Args& a, cudaStream_t s);
// Slabs of rows in which the activations are converted
constexpr int cols_of(int B) { return B <= 8 ? 8 : B <= 16 ? 16 : B <= 32 ? 32 : 64; }
__host__ __device__ constexpr int64_t slab_bytes(int cols, int gpc, int64_t kt) { return kt * cols * (256 + 4 * (1 + gpc)); }
// chunks of 128 inputs that a slab has room for: with more than 8 rows they come in pairs
constexpr int64_t slab_chunks(int cols, int64_t kt) { return cols == 8 ? kt : (kt + 1) / 2 * 2; }
// the products from 9 rows on, unless they are small, with the activations converted
int launch_gemm4(const Gemv4Args& a, const uint8_t* xq, cudaStream_t s);
int device_sms();                                      // SMs of the device that was current at the first call

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float act_of(float g, int act) {
  if (act == 0) return g / (1.0f + expf(-g));
  return 0.5f * g * (1.0f + tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g)));
}

// What a lane of a half-warp makes of its 8 of a chunk's 128 activations: f16 values times a common power of two, those that
// meet codes of bits 4 .. 7 divided by 16; `unit` takes them back, `sum` is that of the lane's group times the power of two
// `of_sum`, which each value is multiplied with before it is added: the plain sum may leave fp32.
template <int GRP>
__device__ __forceinline__ uint4 convert8(const uint4& v, float of_sum, float& sum, float& unit) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
  float x[8];
  sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m = max(m, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
    x[2 * j] = __uint_as_float(w[j] << 16);
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    sum += fmaf(x[2 * j], of_sum, x[2 * j + 1] * of_sum);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
  for (int o = 1; o < GRP / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  // a power of two that brings the largest to 2^15 .. 65280, which f16 still has, as far as fp32 has it (an infinity or NaN stays
  // what it is, beside values that no longer matter). The smallest step of f16, times 16, is then 2^-35 of the largest at most
  const int sh = m == 0 ? 0 : min(15 + 127 - (int)(m >> 7), 126);
  const float f = __uint_as_float((uint32_t)(127 + sh) << 23), f16th = f * 0.0625f;
  unit = __uint_as_float((uint32_t)(127 - sh) << 23);
  return make_uint4(pack_f16(x[0] * f, x[1] * f), pack_f16(x[2] * f16th, x[3] * f16th), pack_f16(x[4] * f, x[5] * f),
                    pack_f16(x[6] * f16th, x[7] * f16th));
}
// Sums of groups in the unit of code products (2^-24), without zeros times the 8 that stands for them
__host__ __device__ constexpr float sum_scale(bool zeros) { return (zeros ? 1.f : 8.f) * 0x1p-24f; }

}  // namespace pop
