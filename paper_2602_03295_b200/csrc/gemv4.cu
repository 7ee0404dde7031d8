// Projections of few rows with 4-bit weights (the decode stage of paper Sec. 3.2 at full depth; narrow weights for that
// stage alone are the stage-aware quantisation that Sec. 6 names as a direction):
//   out[b][n] = sum_k x[b][k] (code[n][k] - zero[n][k / group]) scale[n][k / group]
#include "common.cuh"
#include "ptx.cuh"
#include "w4.cuh"

#include <cuda_fp16.h>

#include <atomic>

namespace pop {
namespace {

constexpr int WARPS = 16;       // of a CTA, one CTA per SM
constexpr int SLOT = 2;         // chunks of 128 inputs in a slot of a warp's ring
constexpr int RING = 4;
constexpr int SMEM_LIMIT = 227 * 1024;

template <int GRP>
struct G4 {
  static constexpr int GPC = 128 / GRP;             // groups of a chunk
  static constexpr int SC = 32 * GPC, ZR = 16 * GPC;
  static constexpr int SLOT_BYTES = SLOT * (1024 + SC + ZR);      // codes, then scales, then zeros
  static constexpr int RING_BYTES = WARPS * RING * SLOT_BYTES;
};

struct Gemv4Dev {
  const bf16* x; int64_t ldx;
  const uint8_t* codes; const uint8_t* scales; const uint8_t* zeros;
  void* out; int64_t ldo;
  int B, N, K, mode, act, n_valid;
  int kt;                       // chunks of 128 inputs
  int tiles;                    // tiles of 16 rows
  int clusters, cs;             // cs CTAs of a cluster share tiles and split their chunks
  int sc, passes;               // chunks of a CTA in a pass over x; passes
  int tpr, rounds;              // tiles of a warp between two exchanges of sums; such rounds
  int* status;
};

__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float act_of(float g, int act) {
  if (act == 0) return g / (1.0f + expf(-g));
  return 0.5f * g * (1.0f + tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g)));
}

// A code in the low bits of an f16 is code * 2^-24, in bits 4 .. 7 code * 2^-20: subnormals are linear, so that a mask alone
// makes a tensor-core operand of two codes of a word, and one shift the other half of them. The activations go in as f16 too,
// those of a chunk of 128 inputs times a power of two that brings their largest near 2^15 (bf16 values stay exact down to
// 2^-27 of it, and within 2^-36 of it below), inputs that meet the codes of bits 4 .. 7 divided by 16. So all products are
// exact; a group's sum is built in the MMA's fp32 accumulator from zero and enters the row's fp32 sum as
//   scale (2^-shift sum_k code_k x'_k - zero sum_k x_k),   the second sum made once with the conversion.
// (Subtracting the zero from every pair of codes took 32 more operations per KB of codes; codes as bf16 128 + code, 64.)
//
// The weight rows are the M side of the warp-level MMA, up to 8 NT activation rows its N side: a tile of 16 rows x 128 inputs
// is 1 KB in one piece, 16 bytes of row g and 16 of row g + 8 to lane (g = lane / 4, t = lane % 4), word j inputs 32 j + 8 t ..
// + 7. A warp streams whole tiles through a ring of its own with bulk copies, so nothing is exchanged between warps. The CTAs
// of a cluster have the same tiles and a part of the inputs each: their activations are converted once, into shared memory,
// and the sums of some tiles per warp are exchanged at a time, added in the order of the ranks.
template <int GRP, int NT, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 1) gemv4_kernel(const __grid_constant__ Gemv4Dev p) {
  using C = G4<GRP>;
  constexpr int GPC = C::GPC, COLS = NT * 8;
  extern __shared__ __align__(128) uint8_t smem[];
  const int xs = p.sc * 256 + 64;                   // bytes of an activation row: 64 off a multiple of 128, so that the
                                                    // rows of a quarter-warp's loads lie in other banks
  uint8_t* s_x = smem + C::RING_BYTES;
  uint8_t* s_zero = s_x + COLS * xs;                // 256 zeros: what lanes without an activation row read
  float* s_acc = reinterpret_cast<float*>(s_zero + 256);          // [tpr][WARPS][COLS][16]
  float* s_sum = s_acc + p.tpr * WARPS * COLS * 16;               // [sc][1 + GPC][COLS]: 2^-shift; sums of the groups
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_sum + p.sc * (1 + GPC) * COLS);      // [WARPS][RING]
  const int tid = threadIdx.x, lane = tid & 31, wic = tid >> 5, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x % p.cs, cluster = blockIdx.x / p.cs;
  const int row0 = blockIdx.y * COLS, rows = min(p.B - row0, COLS);
  const int warps = p.clusters * WARPS, me = cluster * WARPS + wic;
  const int mine = p.tiles > me ? (p.tiles - me + warps - 1) / warps : 0;         // tiles me, me + warps, ..
  const bool gated = p.mode == 3;
  chain_trigger();

  // gated: gate tile and up tile follow each other, so that both are in one cluster
  auto tile_of = [&](int i) {
    const int u = me + i * warps;
    return gated ? (u >> 4) * 16 + ((u >> 1) & 7) + 8 * (u & 1) : u;
  };
  auto chunks_of = [&](int pass, int& c0) {
    c0 = min((pass * p.cs + rank) * p.sc, p.kt);
    return min(p.sc, p.kt - c0);
  };
  uint64_t* bar = bars + wic * RING;
  if (lane < RING) mbar_init(&bar[lane], 1);
  fence_barrier_init();
  for (int i = tid; i < 64; i += WARPS * 32) reinterpret_cast<uint32_t*>(s_zero)[i] = 0;
  __syncwarp();

  // ---- the order of slots: round, pass over x, tile, chunks
  const uint32_t ring = smem_u32(smem + wic * (RING * C::SLOT_BYTES)), bar0 = smem_u32(bar);
  int l_round = 0, l_pass = 0, l_i = -1, l_left = 0, l_slot = 0;
  int64_t l_chunk = 0;
  auto issue = [&] {
    while (l_left <= 0) {                           // to the next tile that there is
      if (l_round >= p.rounds) return;
      if (++l_i >= min(mine, (l_round + 1) * p.tpr)) {
        if (++l_pass >= p.passes) {
          l_pass = 0;
          ++l_round;
        }
        l_i = l_round * p.tpr - 1;
        continue;
      }
      int c0;
      l_left = chunks_of(l_pass, c0);
      l_chunk = (int64_t)tile_of(l_i) * p.kt + c0;
    }
    const int cnt = min(SLOT, l_left);
    if (lane == 0) {
      const uint32_t dst = ring + l_slot * C::SLOT_BYTES, b = bar0 + l_slot * 8;
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(cnt * (1024 + C::SC + (ZEROS ? C::ZR : 0))) : "memory");
      bulk_load(dst, p.codes + l_chunk * 1024, cnt * 1024, b);
      bulk_load(dst + SLOT * 1024, p.scales + l_chunk * C::SC, cnt * C::SC, b);
      if (ZEROS) bulk_load(dst + SLOT * (1024 + C::SC), p.zeros + l_chunk * C::ZR, cnt * C::ZR, b);
    }
    l_slot = l_slot == RING - 1 ? 0 : l_slot + 1;
    l_chunk += cnt;
    l_left -= cnt;
  };
  // the first weights go out before the wait on the preceding kernel: no kernel of the library writes them
#pragma unroll 1
  for (int i = 0; i < RING; ++i) issue();
  chain_wait();

  uint32_t xp[NT], xstep[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool has = n * 8 + g < rows;
    xp[n] = smem_u32(has ? s_x + (n * 8 + g) * xs : s_zero) + t * 16;
    xstep[n] = has ? 256 : 0;
  }
  int slot = 0;
  uint32_t phase = 0;
  bool ok = true, pending = false;                  // pending: peers may still be reading this CTA's sums
  auto settle = [&] {
    if (pending) cluster_wait();
    pending = false;
  };
  for (int round = 0; round < p.rounds; ++round) {
    for (int pass = 0; pass < p.passes; ++pass) {
      int c0;
      const int nc = chunks_of(pass, c0);
      if (p.passes > 1 || round == 0) {
        // ---- activations of the CTA's chunks to f16, a half-warp per row and chunk, with the sums of its groups
        if (p.passes > 1) __syncthreads();
        const int h = lane & 15;
#pragma unroll 2
        for (int item = wic * 2 + (lane >> 4); (item & ~1) < rows * nc; item += WARPS * 2) {
          const int r = item / nc, c = item - r * nc, k = (c0 + c) * 128 + h * 8;
          const bool in = r < rows;
          const uint4 v = in && k < p.K ? *reinterpret_cast<const uint4*>(p.x + (row0 + r) * p.ldx + k) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
          uint32_t m = 0;
          float x[8], sum = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
            m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));      // infinities and NaN stay what they are
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            sum += x[2 * i] + x[2 * i + 1];
          }
#pragma unroll
          for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
          for (int o = 1; o < GRP / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          // a power of two that brings the largest to 2^14 .. 2^15, as far as fp32 has it
          const int sh = m == 0 ? 0 : min(14 + 127 - (int)(m >> 7), 126);
          const float f = __uint_as_float((uint32_t)(127 + sh) << 23), f16th = f * 0.0625f;
          if (in) {
            *reinterpret_cast<uint4*>(s_x + r * xs + c * 256 + h * 16) =
                make_uint4(pack_f16(x[0] * f, x[1] * f), pack_f16(x[2] * f16th, x[3] * f16th), pack_f16(x[4] * f, x[5] * f),
                           pack_f16(x[6] * f16th, x[7] * f16th));
            float* to = s_sum + c * (1 + GPC) * COLS + r;
            if (h == 0) to[0] = __uint_as_float((uint32_t)(127 - sh) << 23);
            if (h % (GRP / 8) == 0) to[(1 + h / (GRP / 8)) * COLS] = sum * ((ZEROS ? 1.f : 8.f) * 0x1p-24f);
          }
        }
        __syncthreads();
      }
      const int end = min(mine, (round + 1) * p.tpr);
      for (int i = round * p.tpr; i < end && ok; ++i) {
        float tot[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) tot[n][0] = tot[n][1] = tot[n][2] = tot[n][3] = 0.f;
        uint32_t x_at[NT], sum_at = smem_u32(s_sum) + t * 8;
#pragma unroll
        for (int n = 0; n < NT; ++n) x_at[n] = xp[n];
        for (int s = 0; s < nc; s += SLOT) {
          if (!mbar_wait(&bar[slot], phase)) {
            ok = false;
            break;
          }
          const uint32_t base = ring + slot * C::SLOT_BYTES;
#pragma unroll
          for (int q = 0; q < SLOT; ++q) {
            if (s + q < nc) {
              const uint32_t cb = base + q * 1024 + lane * 16;
              const uint4 lo = lds128(cb), hi = lds128(cb + 512);
              const uint32_t sb = base + SLOT * 1024 + q * C::SC + g * (4 * GPC);
              const uint32_t zb = base + SLOT * (1024 + C::SC) + q * C::ZR + g * (2 * GPC);
              uint32_t sw[GPC], zw[2] = {0, 0};
              if constexpr (GPC == 1) {
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sw[0]) : "r"(sb));
              } else if constexpr (GPC == 2) {
                asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(sw[0]), "=r"(sw[1]) : "r"(sb));
              } else {
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(sw[0]), "=r"(sw[1]), "=r"(sw[2]), "=r"(sw[3]) : "r"(sb));
              }
              if constexpr (ZEROS) {
                if constexpr (GPC == 1) {
                  uint16_t z;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(z) : "r"(zb));
                  zw[0] = z;
                } else if constexpr (GPC == 2) {
                  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(zw[0]) : "r"(zb));
                } else {
                  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(zw[0]), "=r"(zw[1]) : "r"(zb));
                }
              }
              float2 fx[NT];
#pragma unroll
              for (int n = 0; n < NT; ++n) fx[n] = lds_f2(sum_at + n * 32);
              constexpr int JPG = 4 / GPC;          // words of a group
#pragma unroll
              for (int grp = 0; grp < GPC; ++grp) {
                float d[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
#pragma unroll
                for (int jj = 0; jj < JPG; ++jj) {
                  const int j = grp * JPG + jj;
                  const uint32_t wl = j == 0 ? lo.x : j == 1 ? lo.y : j == 2 ? lo.z : lo.w;
                  const uint32_t wh = j == 0 ? hi.x : j == 1 ? hi.y : j == 2 ? hi.z : hi.w;
                  const uint32_t ul = wl >> 8, uh = wh >> 8;
#pragma unroll
                  for (int n = 0; n < NT; ++n) {
                    const uint4 xv = lds128(x_at[n] + j * 64);
                    mma_f16(d[n], wl & 0x000f000fu, wh & 0x000f000fu, wl & 0x00f000f0u, wh & 0x00f000f0u, xv.x, xv.y);
                    mma_f16(d[n], ul & 0x000f000fu, uh & 0x000f000fu, ul & 0x00f000f0u, uh & 0x00f000f0u, xv.z, xv.w);
                  }
                }
                // scales lie as [row half][group], halves of words; zeros as bytes. What lies behind K is never used.
                const uint32_t w0 = sw[grp / 2], w1 = sw[(GPC + grp) / 2];
                float f0 = __uint_as_float(grp & 1 ? w0 & 0xffff0000u : w0 << 16);
                float f1 = __uint_as_float((GPC + grp) & 1 ? w1 & 0xffff0000u : w1 << 16);
                if (GPC > 1 && grp > 0 && (c0 + s + q) * 128 + grp * GRP >= p.K) f0 = f1 = 0.f;
                float z0 = 1.f, z1 = 1.f;
                if constexpr (ZEROS) {              // 2^23 + zero, minus 2^23
                  const uint32_t b0 = zw[0] >> (8 * grp), b1 = GPC == 4 ? zw[1] >> (8 * grp) : zw[0] >> (8 * (GPC + grp));
                  z0 = __uint_as_float((b0 & 15u) | 0x4b000000u) - 8388608.f;
                  z1 = __uint_as_float((b1 & 15u) | 0x4b000000u) - 8388608.f;
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const float2 sx = lds_f2(sum_at + (1 + grp) * (COLS * 4) + n * 32);
                  tot[n][0] = fmaf(fmaf(d[n][0], fx[n].x, -z0 * sx.x), f0, tot[n][0]);
                  tot[n][1] = fmaf(fmaf(d[n][1], fx[n].y, -z0 * sx.y), f0, tot[n][1]);
                  tot[n][2] = fmaf(fmaf(d[n][2], fx[n].x, -z1 * sx.x), f1, tot[n][2]);
                  tot[n][3] = fmaf(fmaf(d[n][3], fx[n].y, -z1 * sx.y), f1, tot[n][3]);
                }
              }
#pragma unroll
              for (int n = 0; n < NT; ++n) x_at[n] += xstep[n];
              sum_at += (1 + GPC) * (COLS * 4);
            }
          }
          __syncwarp();
          issue();                                  // into the slot that is free now
          slot = slot == RING - 1 ? 0 : slot + 1;
          phase ^= slot == 0 ? 1u : 0u;
        }
        settle();
        // sum i of n-tile n: row g + 8 (i / 2) of the tile, activation row 2 t + i % 2
        float* acc = s_acc + ((i - round * p.tpr) * WARPS + wic) * (COLS * 16);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float* dst = acc + (n * 8 + 2 * t + (r & 1)) * 16 + g + 8 * (r >> 1);
            *dst = pass == 0 ? tot[n][r] : *dst + tot[n][r];
          }
      }
    }
    // ---- exchange: every rank finishes its share of the tiles
    settle();
    if (p.cs > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    const int step = gated ? 2 : 1;
    for (int e = tid + WARPS * 32 * rank; e < p.tpr * WARPS / step * (COLS * 16); e += WARPS * 32 * p.cs) {
      const int row = e & 15, b = (e >> 4) % COLS, sl = (e >> 4) / COLS * step;
      const int u = cluster * WARPS + (sl % WARPS) + (round * p.tpr + sl / WARPS) * warps;
      if (u >= p.tiles || b >= rows) continue;
      auto sum_of = [&](int sl_) {
        const uint32_t a = smem_u32(s_acc + sl_ * (COLS * 16) + b * 16 + row);
        float v = 0.f;
        for (int r = 0; r < p.cs; ++r) {
          float w;
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(mapa_u32(a, r)));
          v += w;
        }
        return v * 0x1p24f;
      };
      if (gated) {
        const float gate = sum_of(sl), up = sum_of(sl + 1);
        const int o = (u >> 4) * 128 + ((u >> 1) & 7) * 16 + row;
        if (o < p.n_valid)
          static_cast<bf16*>(p.out)[(int64_t)(row0 + b) * p.ldo + o] = __float2bfloat16_rn(act_of(gate, p.act) * up);
      } else {
        const int o = u * 16 + row;
        if (o < p.N) {
          float* dst = static_cast<float*>(p.out) + (int64_t)(row0 + b) * p.ldo + o;
          const float v = sum_of(sl);
          *dst = p.mode == 0 ? v : *dst + v;
        }
      }
    }
    if (p.cs > 1) cluster_arrive();                 // this CTA has read its peers' sums
    else if (round + 1 < p.rounds) __syncthreads();
    pending = p.cs > 1;
  }
  settle();
  if (!ok) {
    if (lane == 0) atomicMin(p.status, (int)POP_E_DEVICE_TIMEOUT);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // let in-flight bulk copies land
  }
}

// Clusters of cs CTAs that the GPU holds at once (of the device that was current at the first call)
template <int GRP, int NT, bool ZEROS>
int max_clusters(int cs) {
  static std::atomic<int> known[9];
  int most = known[cs].load(std::memory_order_relaxed);
  if (most > 0) return most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cs);
  cfg.blockDim = dim3(WARPS * 32);
  cfg.dynamicSmemBytes = SMEM_LIMIT;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cs;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&most, gemv4_kernel<GRP, NT, ZEROS>, &cfg) != cudaSuccess || most < 1) {
    cudaGetLastError();
    return device_sms() / cs;
  }
  known[cs].store(most, std::memory_order_relaxed);
  return most;
}

template <int GRP, int NT, bool ZEROS>
int launch_t(Gemv4Dev& p, cudaStream_t s) {
  using C = G4<GRP>;
  static std::atomic<uint64_t> configured{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return POP_E_CUDA;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev >= 64 || !(configured.load(std::memory_order_relaxed) & bit)) {
    if (cudaFuncSetAttribute(gemv4_kernel<GRP, NT, ZEROS>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_LIMIT) != cudaSuccess)
      return POP_E_CUDA;
    configured.fetch_or(bit, std::memory_order_relaxed);
  }
  constexpr int COLS = NT * 8;
  // shared memory beside the ring: activations with their sums, and sums of products
  constexpr int ROOM = SMEM_LIMIT - C::RING_BYTES - 256 - COLS * 64 - WARPS * RING * 8 - 128;
  constexpr int TPR_BYTES = WARPS * COLS * 64, SC_BYTES = COLS * (256 + 4 + 4 * C::GPC);
  static_assert(ROOM >= TPR_BYTES + 8 * SC_BYTES, "shared memory budget");
  // Warps take tiles in turn: the cluster size whose busiest warp has the fewest chunks. A tile's beginning and end cost
  // about one chunk, the exchange within a cluster two.
  int64_t best = INT64_MAX;
  for (int cs = 1; cs <= 8 && cs <= p.kt; cs *= 2) {
    const int most = max_clusters<GRP, NT, ZEROS>(cs);
    const int64_t warps = (int64_t)most * WARPS, per = (p.tiles + warps - 1) / warps;
    const int64_t cost = per * ((p.kt + cs - 1) / cs + 1) + (cs > 1 ? 2 : 0) + (p.kt + cs - 1) / cs;
    if (cost < best) {
      best = cost;
      p.cs = cs;
      const int want = ceil_div(p.tiles, WARPS);
      p.clusters = want < most ? want : most;
    }
  }
  // all chunks of a CTA at once if they fit beside the sums of one tile per warp, then as many tiles as fit
  const int n_i = ceil_div(p.tiles, p.clusters * WARPS), all = ceil_div(p.kt, p.cs), most_sc = (ROOM - TPR_BYTES) / SC_BYTES;
  p.passes = ceil_div(all, most_sc);
  p.sc = ceil_div(p.kt, p.passes * p.cs);
  const int most_tpr = (ROOM - p.sc * SC_BYTES) / TPR_BYTES;
  p.rounds = ceil_div(n_i, most_tpr);
  p.tpr = ceil_div(n_i, p.rounds);
  const int slabs = ceil_div(p.B, COLS);
  if (slabs > 65535) return POP_E_INVALID;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  const size_t smem = C::RING_BYTES + (size_t)p.sc * SC_BYTES + COLS * 64 + 256 + (size_t)p.tpr * TPR_BYTES + WARPS * RING * 8;
  ProfScope prof(PROF_GEMV, (double)p.N * p.K * (0.5 + (p.zeros ? 3.0 : 2.0) / GRP) * slabs, s);
  if (launch_chained_cluster_x(gemv4_kernel<GRP, NT, ZEROS>, dim3(p.clusters * p.cs, slabs), dim3(WARPS * 32), smem, s,
                               (unsigned)p.cs, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

template <int GRP>
int launch_grp(Gemv4Dev& p, cudaStream_t s) {
  if (p.zeros) return p.B <= 8 ? launch_t<GRP, 1, true>(p, s) : launch_t<GRP, 2, true>(p, s);
  return p.B <= 8 ? launch_t<GRP, 1, false>(p, s) : launch_t<GRP, 2, false>(p, s);
}

}  // namespace

int launch_gemv4(const Gemv4Args& a, cudaStream_t s) {
  if (!a.x || !a.codes || !a.scales || !a.out || a.B < 1 || a.N < 1 || a.K < 8 || a.K % 8) return POP_E_INVALID;
  if (a.mode != 0 && a.mode != 2 && a.mode != 3) return POP_E_INVALID;
  if (a.group != 32 && a.group != 64 && a.group != 128) return POP_E_INVALID;
  if (a.mode == 3 && (a.N % 256 || a.n_valid < 0 || a.n_valid > a.N / 2 || (a.act != 0 && a.act != 1))) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.x) % 16 || a.ldx % 8 || reinterpret_cast<uintptr_t>(a.codes) % 16 ||
      reinterpret_cast<uintptr_t>(a.scales) % 16 || reinterpret_cast<uintptr_t>(a.zeros) % 16 ||
      reinterpret_cast<uintptr_t>(a.out) % (a.mode == 3 ? 2 : 4))
    return POP_E_INVALID;
  if (a.N > (1 << 30) || a.K > (1 << 30)) return POP_E_INVALID;
  if (a.B > 1 && (a.ldx < a.K || a.ldo < (a.mode == 3 ? a.n_valid : a.N))) return POP_E_INVALID;     // rows over each other
  Gemv4Dev p{};
  p.x = a.x; p.ldx = a.ldx;
  p.codes = a.codes; p.scales = reinterpret_cast<const uint8_t*>(a.scales); p.zeros = a.zeros;
  p.out = a.out; p.ldo = a.ldo;
  p.B = a.B; p.N = a.N; p.K = a.K; p.mode = a.mode; p.act = a.act; p.n_valid = a.n_valid;
  p.kt = ceil_div(a.K, 128);
  p.tiles = ceil_div(a.N, 16);
  switch (a.group) {
    case 32: return launch_grp<32>(p, s);
    case 64: return launch_grp<64>(p, s);
    default: return launch_grp<128>(p, s);
  }
}

}  // namespace pop
