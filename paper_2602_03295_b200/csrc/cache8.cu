// Filling the 8-bit paged cache: conversion of a bf16 paged cache, and the append of a step's rows with per-head
// RMSNorm and rotation (paper Eq. 2-3, Eq. 14) on the way.
#include "cache8.cuh"

namespace pop {

int device_sms() {
  static const int sms = [] {          // asked once, however many threads call at the same time
    int dev = 0, n = 0;
    const bool known = cudaGetDevice(&dev) == cudaSuccess &&
                       cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0;
    return known ? n : 148;
  }();
  return sms;
}

namespace {

constexpr uint32_t FULL = 0xffffffffu;

__device__ __forceinline__ float warp_amax(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL, v, o));
  return v;
}
__device__ __forceinline__ void unpack_bf16x2(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}

// page of a position's block, or -1 (status word raised) for an entry or position that is no place in the pool
__device__ __forceinline__ int page_of(const int32_t* table, int b, int max_pages, int num_pages, int page_index,
                                       int* status, int lane) {
  if (page_index < max_pages) {
    const int page = table[(int64_t)b * max_pages + page_index];
    if ((unsigned)page < (unsigned)num_pages) return page;
  }
  if (lane == 0) atomicMin(status, (int)POP_E_INVALID);
  return -1;
}

// ------------------------------------------------------------------------------ bf16 cache -> 8-bit cache
// One warp per (layer, K or V, sequence, block of 16 positions, kv head): hd / 8 lanes take one row, 16 bytes each;
// all loads of the block go out before the maximum. 6 bytes move per pair of values, nothing else happens: bound by memory, 8
// layers of 8192 positions (8 heads of 128) 64 us, 6.3 TB/s (0.96 of a copy's rate) at four CTAs per SM, 80 us at two.
struct Quant8Dev {
  Quant8Args a;
  int* status;
};

template <int HD>
__global__ void __launch_bounds__(256, HD == 256 ? 2 : 4) quant_cache8_kernel(const __grid_constant__ Quant8Dev p) {
  constexpr int LPR = HD / 8, RPW = 32 / LPR, NP = C8_BLOCK / RPW;
  const Quant8Args& a = p.a;
  chain_trigger();
  chain_wait();
  const int lane = threadIdx.x & 31, sub = lane / LPR, col = (lane % LPR) * 8;
  const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int h = (int)(item % a.n_kv), blk = (int)(item / a.n_kv), b = blockIdx.y;
  const int layer = blockIdx.z >> 1;
  const bool is_v = blockIdx.z & 1;
  int n = a.seq_lens ? a.seq_lens[b] : a.max_len;
  if (n > a.max_len) {
    n = a.max_len;
    if (lane == 0) atomicMin(p.status, (int)POP_E_INVALID);
  }
  const int pos = blk * C8_BLOCK;
  if (pos >= n) return;
  const int src_page = page_of(a.table, b, a.max_pages, a.num_pages, pos / a.page_size, p.status, lane);
  const int dst_page = page_of(a.dst.table, b, a.dst.max_pages, a.dst.num_pages, pos / a.dst.page_size, p.status, lane);
  if (src_page < 0 || dst_page < 0) return;
  const bf16* src = (is_v ? a.v : a.k) + (int64_t)layer * a.layer_stride +
                    (((int64_t)src_page * a.page_size + pos % a.page_size) * a.n_kv + h) * HD + col;
  const int live = n - pos;            // rows of the block (from its first on) that hold something
  uint4 raw[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int r = i * RPW + sub;
    raw[i] = r < live ? *reinterpret_cast<const uint4*>(src + (int64_t)r * a.n_kv * HD) : make_uint4(0, 0, 0, 0);
  }
  float am = 0.f;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x, y;
      unpack_bf16x2(w[j], x, y);
      am = fmaxf(am, fmaxf(fabsf(x), fabsf(y)));
    }
  }
  const int e = c8_scale_exp(warp_amax(am));
  const float inv = c8_pow2(127 - e);
  const int slot = pos % a.dst.page_size;
  const int64_t tile = (int64_t)dst_page * a.n_kv + h;
  uint8_t* dst = (is_v ? a.dst.v : a.dst.k) + (int64_t)layer * a.code_layer_stride +
                 (tile * a.dst.page_size + slot) * HD + col;
  if (lane == 0)
    ((is_v ? a.dst.vs : a.dst.ks) + (int64_t)layer * a.scale_layer_stride)[tile * (a.dst.page_size / C8_BLOCK) +
                                                                          slot / C8_BLOCK] = (uint8_t)e;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int r = i * RPW + sub;
    if (r >= live) continue;
    float f[8];
    unpack_bf16x2(raw[i].x, f[0], f[1]);
    unpack_bf16x2(raw[i].y, f[2], f[3]);
    unpack_bf16x2(raw[i].z, f[4], f[5]);
    unpack_bf16x2(raw[i].w, f[6], f[7]);
    uint2 o;
    o.x = c8_codes4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    o.y = c8_codes4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
    *reinterpret_cast<uint2*>(dst + (int64_t)r * HD) = o;
  }
}

// ------------------------------------------------------------------------------ norm + rotation + append
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
// four codes times a power of two, rounded again
__device__ __forceinline__ uint32_t rescaled4(uint32_t w, float f) {
  const uint32_t l = c8_half2_lo(w), m = c8_half2_hi(w);
  const float2 v0 = __half22float2(*reinterpret_cast<const __half2*>(&l));
  const float2 v1 = __half22float2(*reinterpret_cast<const __half2*>(&m));
  return c8_codes4(v0.x * f, v0.y * f, v1.x * f, v1.y * f);
}

// Two warps per (sequence, block of 16 cache positions that the new rows touch, head), eight slots each. hd / 8 lanes take
// one row, each four rotation pairs (j, j + hd/2): two 16-byte loads of fp32 (8-byte of bf16). The rows stay in registers
// until the block's maximum is known, which the two warps exchange (one warp for all 16 rows: 128 registers, 72 us for 6656
// rows of 32 + 16 heads; two warps at four CTAs per SM 57 us, 4.0 TB/s; the bytes take 35). Bound by the loads that the
// resident warps keep in flight: bf16 rows, with half the bytes in each, take 63 us where the bytes take 23. A CTA is four
// heads of the same rows, so the rotary rows come from L1 after the first.
struct Append8Dev {
  Append8Args a;
  int head_groups;              // CTAs per block of positions: four heads each
  int* status;
};

template <int HD, bool IN_BF16>
__global__ void __launch_bounds__(256, HD == 256 ? 2 : 4) append8_kernel(const __grid_constant__ Append8Dev p) {
  constexpr int LPR = HD / 8, RPW = 32 / LPR, NP = C8_BLOCK / 2 / RPW, HALF = HD / 2;
  __shared__ float half_max[8];
  const Append8Args& a = p.a;
  chain_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j0 = (lane % LPR) * 4;
  const int sub = (warp & 1) * (C8_BLOCK / 2) + lane / LPR;                       // slot of the lane's first row
  const int heads = a.n_q + 2 * a.n_kv;
  const int blk = blockIdx.x / p.head_groups, b = blockIdx.y;
  int h = (int)(blockIdx.x - blk * p.head_groups) * 4 + (warp >> 1);
  const bool idle = h >= heads;                                                   // works on the last head, stores nothing
  if (idle) h = heads - 1;
  const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
  chain_wait();
  const int row0 = a.cu ? __ldg(a.cu + b) : b * a.rows;
  const int n = a.cu ? __ldg(a.cu + b + 1) - row0 : a.rows;
  const int start = a.start ? __ldg(a.start + b) : a.pos0;
  bool bad = (n > 0) & ((n > a.rows) | (start < 0) | (start > 0x7ffffff0 - a.rows));      // no rows: whatever the start is
  if (bad || n <= 0) {
    if (bad && lane == 0) atomicMin(p.status, (int)POP_E_INVALID);
    return;
  }
  const int first = (start / C8_BLOCK + blk) * C8_BLOCK;                          // position of the block's slot 0
  if (first >= start + n) return;
  const int lo = max(start - first, 0), hi = idle ? 0 : min(start + n - first, C8_BLOCK);    // live slots of the block
  const int64_t r_base = (int64_t)row0 + first - start;                           // packed row of slot 0

  // Everything that is read is asked for before anything is computed: the page, the rows, the positions, the old scale. What
  // the checks find is raised once, at the end: a status write between loads would put them in order.
  int page = -1;
  if (!is_q) {
    const int pi = first / a.dst.page_size;
    if (pi < a.dst.max_pages) page = __ldg(a.dst.table + (int64_t)b * a.dst.max_pages + pi);
  }
  float x[NP][8];               // [.. 0..3] elements j0 + i, [.. 4..7] their partners j0 + i + hd/2
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int s = i * RPW + sub;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[i][u] = 0.f;
    if (s < lo || s >= hi) continue;
    const int64_t off = (r_base + s) * a.ld_in + (int64_t)h * HD + j0;
    load_row8<HD, IN_BF16>(a.in, off, x[i]);
  }
  if (!is_v) {
    int axis[4] = {0, 0, 0, 0};
    if (a.pair_axis != nullptr) {
      const uchar4 v = __ldg(reinterpret_cast<const uchar4*>(a.pair_axis + j0));
      axis[0] = v.x; axis[1] = v.y; axis[2] = v.z; axis[3] = v.w;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (axis[u] >= a.n_axes) {             // never turned into an address
          bad = true;
          axis[u] = 0;
        }
    }
    const bool one_axis = axis[0] == axis[1] && axis[1] == axis[2] && axis[2] == axis[3];
    int tp[NP];                                // table row of the lane's first pair
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = i * RPW + sub;
      tp[i] = first + s;
      if (a.positions != nullptr) tp[i] = s >= lo && s < hi ? __ldg(a.positions + axis[0] * a.ld_pos + r_base + s) : 0;
    }
    const float* gain = is_q ? a.q_gain : a.k_gain;
    float4 g0 = make_float4(1.f, 1.f, 1.f, 1.f), g1 = g0;
    if (gain != nullptr) {
      g0 = make_float4(__ldg(gain + j0), __ldg(gain + j0 + 1), __ldg(gain + j0 + 2), __ldg(gain + j0 + 3));
      g1 = make_float4(__ldg(gain + j0 + HALF), __ldg(gain + j0 + HALF + 1), __ldg(gain + j0 + HALF + 2), __ldg(gain + j0 + HALF + 3));
    }
    auto row_of = [&](int t) {
      if ((unsigned)t >= (unsigned)a.table_rows) {      // never turned into an address
        bad = true;
        t = 0;
      }
      return a.table + (int64_t)t * HALF + j0;
    };
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = i * RPW + sub;
      const bool live = s >= lo && s < hi;
      float2 cs[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) cs[u] = make_float2(1.f, 0.f);
      if (live) {
        if (one_axis) {
          const float4* t = reinterpret_cast<const float4*>(row_of(tp[i]));
          const float4 t0 = __ldg(t), t1 = __ldg(t + 1);
          cs[0] = make_float2(t0.x, t0.y); cs[1] = make_float2(t0.z, t0.w);
          cs[2] = make_float2(t1.x, t1.y); cs[3] = make_float2(t1.z, t1.w);
        } else {
          cs[0] = __ldg(row_of(tp[i]));
#pragma unroll
          for (int u = 1; u < 4; ++u) cs[u] = __ldg(row_of(__ldg(a.positions + axis[u] * a.ld_pos + r_base + s)) + u);
        }
      }
      if (gain != nullptr) norm_row8<HD>(x[i], g0, g1, a.eps);
      turn_row8(x[i], cs);
      if (is_q && live) store_q8<HD>(a.q_out + (r_base + s) * a.ldq + (int64_t)h * HD + j0, x[i]);
    }
  }
  // the other half of the block's rows is in the neighbouring warp
  const bool stores = !is_q && !idle && (unsigned)page < (unsigned)a.dst.num_pages;       // else never turned into an address
  bad |= !is_q && !idle && !stores;
  const int slot = first % a.dst.page_size;
  const int64_t tile = (int64_t)(stores ? page : 0) * a.n_kv + (stores ? h - a.n_q - (is_v ? a.n_kv : 0) : 0);
  uint8_t* dst = (is_v ? a.dst.v : a.dst.k) + (tile * a.dst.page_size + slot) * HD + j0;
  uint8_t* scale = (is_v ? a.dst.vs : a.dst.ks) + tile * (a.dst.page_size / C8_BLOCK) + slot / C8_BLOCK;
  int was = 0;                                           // the scale of earlier positions in the block
  if (stores) {
    if (lo > 0) was = *scale;
    float am = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int u = 0; u < 8; ++u) am = fmaxf(am, fabsf(x[i][u]));      // dead slots are zeros
    am = warp_amax(am);
    if (lane == 0) half_max[warp] = am;
  }
  __syncthreads();                                       // also: both warps have read the old scale
  if (stores) {
    int e = c8_scale_exp(fmaxf(half_max[warp], half_max[warp ^ 1]));
    if (e > was && lo > 0) {    // bring the earlier codes to the larger scale: exponents shift, small codes round again
      const float f = c8_pow2(was - e);
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int s = i * RPW + sub;
        if (s >= lo) continue;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t* w = reinterpret_cast<uint32_t*>(dst + (int64_t)s * HD + half * HALF);
          *w = rescaled4(*w, f);
        }
      }
    }
    e = max(e, was);
    if (lane == 0 && (warp & 1) == 0) *scale = (uint8_t)e;
    const float inv = c8_pow2(127 - e);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int s = i * RPW + sub;
      if (s < lo || s >= hi) continue;
      *reinterpret_cast<uint32_t*>(dst + (int64_t)s * HD) =
          c8_codes4(x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv);
      *reinterpret_cast<uint32_t*>(dst + (int64_t)s * HD + HALF) =
          c8_codes4(x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv);
    }
  }
  if (bad) atomicMin(p.status, (int)POP_E_INVALID);
}

// The form of one row per sequence, a decode step: hd / 8 lanes per (sequence, head), one CTA for 256 / (hd / 8) heads. The
// same arithmetic; the codes that a larger scale brings along are the only thing beyond one row. Bound by its chain of
// loads (start, page, old scale); the kernel above, whose lanes would be empty in 15 of 16 slots, took 9.3 us for 96
// sequences of 32 + 16 heads (two rounds of CTAs), this one 3.3; one sequence 2.8 and 1.8 (in a captured
// graph; an eager call's host time is 15 or more).
template <int HD, bool IN_BF16>
__global__ void __launch_bounds__(256) append8_row_kernel(const __grid_constant__ Append8Dev p) {
  constexpr int LPR = HD / 8, HALF = HD / 2;
  const Append8Args& a = p.a;
  chain_trigger();
  const int lane = threadIdx.x & 31, j0 = (lane % LPR) * 4, b = blockIdx.y;
  const int heads = a.n_q + 2 * a.n_kv;
  int h = (int)(blockIdx.x * (256 / LPR) + threadIdx.x / LPR);
  const bool idle = h >= heads;                                                   // works on the last head, stores nothing
  if (idle) h = heads - 1;
  const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
  chain_wait();
  const int row = a.cu ? __ldg(a.cu + b) : b;
  const int n = a.cu ? __ldg(a.cu + b + 1) - row : 1;
  const int at = a.start ? __ldg(a.start + b) : a.pos0;                           // the row's cache position
  bool bad = (n > 0) & ((n > 1) | (at < 0) | (at > 0x7ffffff0 - 1));              // no row: whatever the start is
  if (bad || n <= 0) {
    if (bad && threadIdx.x == 0) atomicMin(p.status, (int)POP_E_INVALID);
    return;
  }
  const int lo = at % C8_BLOCK, first = at - lo;                                  // earlier positions of its block
  int page = -1;
  if (!is_q) {
    const int pi = first / a.dst.page_size;
    if (pi < a.dst.max_pages) page = __ldg(a.dst.table + (int64_t)b * a.dst.max_pages + pi);
  }
  float x[8];
  load_row8<HD, IN_BF16>(a.in, (int64_t)row * a.ld_in + (int64_t)h * HD + j0, x);
  float2 cs[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) cs[u] = make_float2(1.f, 0.f);
  if (!is_v) {
    uchar4 axis = make_uchar4(0, 0, 0, 0);
    if (a.pair_axis != nullptr) axis = __ldg(reinterpret_cast<const uchar4*>(a.pair_axis + j0));
    const int ax[4] = {axis.x, axis.y, axis.z, axis.w};
    const float2* from[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool known = a.pair_axis == nullptr || ax[u] < a.n_axes;              // else never turned into an address
      int t = a.positions != nullptr && known ? __ldg(a.positions + ax[u] * a.ld_pos + row) : at;
      if (!known || (unsigned)t >= (unsigned)a.table_rows) {
        bad = true;
        t = 0;
      }
      from[u] = a.table + (int64_t)t * HALF + j0 + u;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) cs[u] = __ldg(from[u]);
  }
  const float* gain = is_q ? a.q_gain : is_v ? nullptr : a.k_gain;
  if (a.q_gain != nullptr || a.k_gain != nullptr) {                               // by all lanes: heads of a warp may differ
    float4 g0 = make_float4(1.f, 1.f, 1.f, 1.f), g1 = g0;
    if (gain != nullptr) {
      g0 = make_float4(__ldg(gain + j0), __ldg(gain + j0 + 1), __ldg(gain + j0 + 2), __ldg(gain + j0 + 3));
      g1 = make_float4(__ldg(gain + j0 + HALF), __ldg(gain + j0 + HALF + 1), __ldg(gain + j0 + HALF + 2), __ldg(gain + j0 + HALF + 3));
    }
    float y[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) y[u] = x[u];
    norm_row8<HD>(y, g0, g1, a.eps);
    if (gain != nullptr) {
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = y[u];
    }
  }
  if (!is_v) turn_row8(x, cs);
  if (is_q && !idle) store_q8<HD>(a.q_out + (int64_t)row * a.ldq + (int64_t)h * HD + j0, x);
  const bool stores = !is_q && !idle && (unsigned)page < (unsigned)a.dst.num_pages;       // else never turned into an address
  bad |= !is_q && !idle && !stores;
  const int slot = first % a.dst.page_size;
  const int64_t tile = (int64_t)(stores ? page : 0) * a.n_kv + (stores ? h - a.n_q - (is_v ? a.n_kv : 0) : 0);
  uint8_t* dst = (is_v ? a.dst.v : a.dst.k) + (tile * a.dst.page_size + slot) * HD + j0;
  uint8_t* scale = (is_v ? a.dst.vs : a.dst.ks) + tile * (a.dst.page_size / C8_BLOCK) + slot / C8_BLOCK;
  const int was = stores && lo > 0 ? *scale : 0;                                  // the scale of earlier positions in the block
  float am = 0.f;
#pragma unroll
  for (int u = 0; u < 8; ++u) am = fmaxf(am, fabsf(x[u]));
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(FULL, am, o));
  __syncwarp();                                          // every lane has the old scale
  if (stores) {
    int e = c8_scale_exp(am);
    if (e > was && lo > 0) {    // bring the earlier codes to the larger scale: exponents shift, small codes round again
      const float f = c8_pow2(was - e);
#pragma unroll 5
      for (int i = 0; i < lo; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t* w = reinterpret_cast<uint32_t*>(dst + (int64_t)i * HD + half * HALF);
          *w = rescaled4(*w, f);
        }
    }
    e = max(e, was);
    if (j0 == 0) *scale = (uint8_t)e;
    const float inv = c8_pow2(127 - e);
    uint32_t* to = reinterpret_cast<uint32_t*>(dst + (int64_t)lo * HD);
    to[0] = c8_codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    to[HALF / 4] = c8_codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
  }
  if (bad) atomicMin(p.status, (int)POP_E_INVALID);
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

int launch_quant_cache8(const Quant8Args& a, cudaStream_t s) {
  if (!a.k || !a.v || !a.table || !c8_cache_ok(a.dst)) return POP_E_INVALID;
  if (a.layers < 1 || a.layers > 32767 || a.batch < 1 || a.batch > 65535 || a.n_kv < 1 || a.n_kv > 1024 ||
      a.max_len < 0 || a.max_len > 0x7fff0000 || !page_size_ok(a.page_size) || a.num_pages < 1 || a.max_pages < 1)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (!aligned(a.k, 16) || !aligned(a.v, 16) || a.layer_stride % 8 || a.code_layer_stride % 16) return POP_E_INVALID;
  if ((int64_t)a.max_len > (int64_t)a.max_pages * a.page_size ||
      (int64_t)a.max_len > (int64_t)a.dst.max_pages * a.dst.page_size)
    return POP_E_NOSPACE;
  if (a.max_len == 0) return POP_OK;
  Quant8Dev p;
  p.a = a;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  const int64_t items = (((int64_t)a.max_len + C8_BLOCK - 1) / C8_BLOCK) * a.n_kv;
  if ((items + 7) / 8 > 0x7fffffff) return POP_E_INVALID;
  const dim3 grid((unsigned)((items + 7) / 8), a.batch, a.layers * 2);
  ProfScope prof(PROF_ELEMENTWISE, (double)a.layers * a.batch * a.max_len * a.n_kv * a.head_dim * 6.0, s);
  cudaError_t rc;
  switch (a.head_dim) {
    case 64: rc = launch_chained(quant_cache8_kernel<64>, grid, dim3(256), 0, s, p); break;
    case 128: rc = launch_chained(quant_cache8_kernel<128>, grid, dim3(256), 0, s, p); break;
    default: rc = launch_chained(quant_cache8_kernel<256>, grid, dim3(256), 0, s, p); break;
  }
  if (rc != cudaSuccess) return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

int launch_append8(const Append8Args& a, cudaStream_t s) {
  if (!a.in || !a.table || !c8_cache_ok(a.dst) || (a.n_q > 0 && !a.q_out)) return POP_E_INVALID;
  if (a.batch < 1 || a.batch > 65535 || a.rows < 0 || a.n_q < 0 || a.n_kv < 1 || a.n_q > 4096 || a.n_kv > 1024 ||
      a.pos0 < 0 || a.table_rows < 1)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (a.positions != nullptr && a.n_axes < 1) return POP_E_INVALID;
  if (a.pair_axis != nullptr && (a.positions == nullptr || a.n_axes > 255 || !aligned(a.pair_axis, 4))) return POP_E_INVALID;
  if (!aligned(a.in, 16) || !aligned(a.table, 16) || a.ld_in % 4 || (a.n_q > 0 && (!aligned(a.q_out, 8) || a.ldq % 4)))
    return POP_E_INVALID;
  if ((int64_t)a.batch * a.rows > 0x7fffffff) return POP_E_INVALID;
  if (a.n_q > 0 && (int64_t)a.batch * a.rows > 1 && a.ldq < (int64_t)a.n_q * a.head_dim) return POP_E_INVALID;
  if (a.start == nullptr && (int64_t)a.pos0 + a.rows > (int64_t)a.dst.max_pages * a.dst.page_size) return POP_E_NOSPACE;
  if (a.rows == 0) return POP_OK;
  Append8Dev p{};
  p.a = a;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  const int heads = a.n_q + 2 * a.n_kv;
  p.head_groups = ceil_div(heads, 4);
  // rows that start anywhere in a block touch at most this many blocks
  const int64_t blocks = ((int64_t)a.rows + 2 * C8_BLOCK - 2) / C8_BLOCK;
  const int64_t gx = blocks * p.head_groups;
  if (gx > 0x7fffffff) return POP_E_INVALID;
  const dim3 grid((unsigned)gx, a.batch);
  ProfScope prof(PROF_ELEMENTWISE,
                 (double)a.batch * a.rows * a.head_dim * (heads * (a.in_bf16 ? 2.0 : 4.0) + a.n_q * 2.0 + a.n_kv * 2.0), s);
  void (*kernel)(Append8Dev);
  dim3 g = grid;
  if (a.rows == 1) {
    g.x = ceil_div(heads, 2048 / a.head_dim);
    switch (a.head_dim) {
      case 64: kernel = a.in_bf16 ? append8_row_kernel<64, true> : append8_row_kernel<64, false>; break;
      case 128: kernel = a.in_bf16 ? append8_row_kernel<128, true> : append8_row_kernel<128, false>; break;
      default: kernel = a.in_bf16 ? append8_row_kernel<256, true> : append8_row_kernel<256, false>; break;
    }
  } else {
    switch (a.head_dim) {
      case 64: kernel = a.in_bf16 ? append8_kernel<64, true> : append8_kernel<64, false>; break;
      case 128: kernel = a.in_bf16 ? append8_kernel<128, true> : append8_kernel<128, false>; break;
      default: kernel = a.in_bf16 ? append8_kernel<256, true> : append8_kernel<256, false>; break;
    }
  }
  const cudaError_t rc = launch_chained(kernel, g, dim3(256), 0, s, p);
  if (rc != cudaSuccess) return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

}  // namespace pop
