// 4-bit weights (internal): arguments of their product with few rows. The layout is stated in pop_kernels.h.
#pragma once
#include "common.cuh"

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
size_t gemv4_workspace_bytes(int B, int K, int group);
int launch_gemv4(const Gemv4Args& a, cudaStream_t s);
int device_sms();                                      // SMs of the device that was current at the first call

}  // namespace pop
