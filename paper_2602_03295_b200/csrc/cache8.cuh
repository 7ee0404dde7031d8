// The 8-bit paged cache (internal): layout, scales and conversions shared by the kernels that fill and read it.
//
// Codes are OCP E4M3, head-major inside a page: [pages][n_kv][page_size][hd] bytes, so that the positions of one page
// and kv head are contiguous (a block of 16 positions is 16 hd bytes in one piece). Every block of 16 positions and
// kv head has one E8M0 scale, a power of two stored as its exponent + 127: [pages][n_kv][page_size / 16] bytes.
// A power of two costs no relative precision in a floating-point code, its product with a code is an exact bf16 value,
// raising it for a later, larger row only shifts exponents of the codes that are there, and its logarithm is an
// integer, which the attention kernels add to a score instead of multiplying values.
#pragma once
#include "common.cuh"

#include <cuda_fp16.h>

#include <atomic>

namespace pop {

constexpr int C8_BLOCK = 16;          // positions per scale
constexpr int C8_MIN_EXP = 127 - 64;  // smallest scale, 2^-64: a block of zeros, and anything below 448 * 2^-64

// E8M0 byte of the smallest power of two s >= 2^-64 with amax <= 448 s. 448 = 1.75 * 2^8: with amax = 1.f * 2^E that is
// 2^(E-8), one more when 1.f > 1.75, i.e. when adding 0x1fffff to the fraction bits carries into the exponent.
// amax = inf gives 2^120, whose codes saturate at 448.
__device__ __forceinline__ int c8_scale_exp(float amax) {
  const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
  return e > C8_MIN_EXP ? (e < 247 ? e : 247) : C8_MIN_EXP;
}
// 2^(d) for -126 <= d <= 127; 0 below
__device__ __forceinline__ float c8_pow2(int d) { return d < -126 ? 0.f : __uint_as_float((uint32_t)(d + 127) << 23); }

// four fp32 values -> four codes, round to nearest even, saturating, the first in the low byte
__device__ __forceinline__ uint32_t c8_codes4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// the same of two packed f16 pairs
__device__ __forceinline__ uint32_t c8_codes4_h2(uint32_t ab, uint32_t cd) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(lo) : "r"(ab));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(hi) : "r"(cd));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// two codes (low and high byte of h) -> packed f16, exact
__device__ __forceinline__ uint32_t c8_half2(uint16_t h) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
  return r;
}
__device__ __forceinline__ uint32_t c8_half2_lo(uint32_t w) { return c8_half2((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ uint32_t c8_half2_hi(uint32_t w) { return c8_half2((uint16_t)(w >> 16)); }

// device addresses of one layer of the cache
struct Cache8 {
  uint8_t* k; uint8_t* v;              // [pages][n_kv][page_size][hd]
  uint8_t* ks; uint8_t* vs;            // [pages][n_kv][page_size / 16]
  const int32_t* table;                // [batch][max_pages]
  int page_size, num_pages, max_pages;
};

// what both attention kernels take besides the queries
inline bool c8_cache_ok(const Cache8& c) {
  return c.k && c.v && c.ks && c.vs && c.table && page_size_ok(c.page_size) && c.num_pages >= 1 && c.max_pages >= 1 &&
         reinterpret_cast<uintptr_t>(c.k) % 16 == 0 && reinterpret_cast<uintptr_t>(c.v) % 16 == 0;
}

struct Quant8Args {
  const bf16* k; const bf16* v; int64_t layer_stride;          // [layers][pages][page_size][n_kv][hd]
  const int32_t* table; int page_size, num_pages, max_pages;
  Cache8 dst; int64_t code_layer_stride, scale_layer_stride;
  const int32_t* seq_lens; int max_len;
  int layers, batch, n_kv, head_dim;
};
int launch_quant_cache8(const Quant8Args& a, cudaStream_t s);

struct Append8Args {
  const void* in; bool in_bf16; int64_t ld_in;                 // rows [q heads | k heads | v heads] * hd
  const int32_t* cu; int rows;                                 // packed rows of each sequence, at most `rows`
  const int32_t* start; int pos0;                              // position of a sequence's first row
  int batch;
  bf16* q_out; int64_t ldq;
  Cache8 dst;
  const float* q_gain; const float* k_gain; float eps;
  const float2* table; int table_rows;
  const int32_t* positions; int64_t ld_pos; const uint8_t* pair_axis; int n_axes;
  int n_q, n_kv, head_dim;
};
int launch_append8(const Append8Args& a, cudaStream_t s);

struct Attn8Args {
  const bf16* q; int64_t ldq;
  Cache8 c;
  const int32_t* cu; int rows;                                 // prompt form: query rows of each sequence
  const int32_t* seq_lens; int kv_len;                         // cached positions, the query rows' own included
  bf16* out; int64_t ldo;
  int batch, n_q, n_kv, head_dim, window;
  void* workspace; size_t workspace_bytes;
};
int launch_decode_attention8(const Attn8Args& a, cudaStream_t s);
int launch_attention8(const Attn8Args& a, cudaStream_t s);
int launch_few8(const Attn8Args& a, cudaStream_t s);           // few rows; arguments checked by the two above
// Lets a kernel have `bytes` of dynamic shared memory on the current device; done: a bit per device that has been asked
inline bool c8_allow_smem(std::atomic<uint64_t>& done, const void* kernel, int bytes) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}
int device_sms();                                              // SMs of the device that was current at the first call

}  // namespace pop
