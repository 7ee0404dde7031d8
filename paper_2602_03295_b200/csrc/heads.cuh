// A head's row held by hd / 8 lanes of a warp: load, RMSNorm, rotation and store, shared by the kernels that append to a
// cache (paper Eq. 2-3). A lane has elements j0 .. j0 + 3 and their rotation partners j0 + hd/2 ...
#pragma once
#include "common.cuh"

namespace pop {

constexpr uint32_t FULL = 0xffffffffu;

__device__ __forceinline__ void unpack_bf16x2(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}

// Elements j0 .. j0 + 3 of a head's row into x[0..3], their rotation partners j0 + hd/2 .. into x[4..7]
template <int HD, bool IN_BF16>
__device__ __forceinline__ void load_row8(const void* in, int64_t off, float (&x)[8]) {
  if constexpr (IN_BF16) {
    const uint2 l = __ldg(reinterpret_cast<const uint2*>(static_cast<const bf16*>(in) + off));
    const uint2 m = __ldg(reinterpret_cast<const uint2*>(static_cast<const bf16*>(in) + off + HD / 2));
    unpack_bf16x2(l.x, x[0], x[1]);
    unpack_bf16x2(l.y, x[2], x[3]);
    unpack_bf16x2(m.x, x[4], x[5]);
    unpack_bf16x2(m.y, x[6], x[7]);
  } else {
    const float4 l = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(in) + off));
    const float4 m = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(in) + off + HD / 2));
    x[0] = l.x; x[1] = l.y; x[2] = l.z; x[3] = l.w;
    x[4] = m.x; x[5] = m.y; x[6] = m.z; x[7] = m.w;
  }
}
// RMSNorm over the row that hd / 8 lanes hold, by all lanes of the warp
template <int HD>
__device__ __forceinline__ void norm_row8(float (&x)[8], float4 g0, float4 g1, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) ss = fmaf(x[u], x[u], ss);
#pragma unroll
  for (int o = HD / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(FULL, ss, o);
  const float rstd = rsqrtf(ss / (float)HD + eps);
  x[0] = x[0] * rstd * g0.x; x[1] = x[1] * rstd * g0.y;
  x[2] = x[2] * rstd * g0.z; x[3] = x[3] * rstd * g0.w;
  x[4] = x[4] * rstd * g1.x; x[5] = x[5] * rstd * g1.y;
  x[6] = x[6] * rstd * g1.z; x[7] = x[7] * rstd * g1.w;
}
__device__ __forceinline__ void turn_row8(float (&x)[8], const float2 (&cs)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float c = x[u] * cs[u].x - x[u + 4] * cs[u].y;
    const float d = x[u + 4] * cs[u].x + x[u] * cs[u].y;
    x[u] = c;
    x[u + 4] = d;
  }
}
template <int HD>
__device__ __forceinline__ void store_q8(bf16* dst, const float (&x)[8]) {
  __nv_bfloat162 w0 = __floats2bfloat162_rn(x[0], x[1]), w1 = __floats2bfloat162_rn(x[2], x[3]);
  __nv_bfloat162 w2 = __floats2bfloat162_rn(x[4], x[5]), w3 = __floats2bfloat162_rn(x[6], x[7]);
  uint2 o;
  o.x = *reinterpret_cast<uint32_t*>(&w0); o.y = *reinterpret_cast<uint32_t*>(&w1);
  *reinterpret_cast<uint2*>(dst) = o;
  o.x = *reinterpret_cast<uint32_t*>(&w2); o.y = *reinterpret_cast<uint32_t*>(&w3);
  *reinterpret_cast<uint2*>(dst + HD / 2) = o;
}

}  // namespace pop
