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

constexpr int WARPS = 8;        // of a CTA. Two CTAs per SM, so that one's beginning and end (and the next launch's) lie beside
                                // the other's work
constexpr int SMEM_LIMIT = 112 * 1024;

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
__device__ __forceinline__ uint4 ld_codes(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// D = A B + (first ? 0 : D), m16n8k16
__device__ __forceinline__ void mma_f16(float (&d)[4], bool first, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  if (first)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
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
// + 7. A warp streams whole tiles into registers, so nothing is exchanged between warps. The CTAs of a cluster have the same
// tiles and a part of the inputs each: their activations are converted once, into shared memory, and the sums of some tiles
// per warp are exchanged at a time, added in the order of the ranks.
template <int GRP, int NT, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 2) gemv4_kernel(const __grid_constant__ Gemv4Dev p) {
  constexpr int GPC = 128 / GRP, COLS = NT * 8, SC = 32 * GPC, ZR = 16 * GPC;
  constexpr int U = GPC == 1 && NT == 1 ? 4 : 2;    // chunks of a batch of loads; two batches are in flight
  extern __shared__ __align__(128) uint8_t smem[];
  const int xs = p.sc * 256 + 64;                   // bytes of an activation row: 64 off a multiple of 128, so that the
                                                    // rows of a quarter-warp's loads lie in other banks
  uint8_t* s_zero = smem;                           // 256 zeros: what lanes without an activation row read
  uint8_t* s_x = smem + 256;
  float* s_acc = reinterpret_cast<float*>(s_x + COLS * xs);       // [tpr][WARPS][NT][32 lanes][4]
  float* s_sum = s_acc + p.tpr * WARPS * COLS * 16;               // [sc][1 + GPC][COLS]: 2^-shift; sums of the groups
  const int tid = threadIdx.x, lane = tid & 31, wic = tid >> 5, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x % p.cs, cluster = blockIdx.x / p.cs;
  const int row0 = blockIdx.y * COLS, rows = min(p.B - row0, COLS);
  const int warps = p.clusters * WARPS, me = cluster * WARPS + wic;
  const int mine = p.tiles > me ? (p.tiles - me + warps - 1) / warps : 0;         // tiles me, me + warps, ..
  const bool gated = p.mode == 3;
  chain_trigger();
  auto chunks_of = [&](int pass, int& c0) {
    c0 = min((pass * p.cs + rank) * p.sc, p.kt);
    return min(p.sc, p.kt - c0);
  };

  // ---- loads: the batches of a round and pass in their order
  struct Batch {
    uint4 lo[U], hi[U];
    uint32_t sc[U][GPC];                            // scales of row g, then of row g + 8
    uint32_t zr[U][GPC == 4 ? 2 : 1];               // their zeros, a byte each
  };
  Batch b0, b1;
  int l_i = 0, l_end = 0, l_s = 0, l_nc = 0, l_c0 = 0;
  const uint8_t *l_codes = nullptr, *l_scales = nullptr, *l_zeros = nullptr;
  auto set_tile = [&] {
    // gated: gate tile and up tile follow each other, so that both are in one cluster
    const int u = me + l_i * warps, tile = gated ? (u >> 4) * 16 + ((u >> 1) & 7) + 8 * (u & 1) : u;
    const int64_t chunk = (int64_t)tile * p.kt + l_c0;
    l_codes = p.codes + chunk * 1024 + lane * 16;
    l_scales = p.scales + chunk * SC + g * (4 * GPC);
    if (ZEROS) l_zeros = p.zeros + chunk * ZR + g * (2 * GPC);
    l_s = 0;
  };
  auto load_next = [&](Batch& q) {
    if (l_i >= l_end) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (l_s + u < l_nc) {
        q.lo[u] = ld_codes(l_codes + u * 1024);
        q.hi[u] = ld_codes(l_codes + u * 1024 + 512);
        if constexpr (GPC == 1) {
          q.sc[u][0] = __ldg(reinterpret_cast<const uint32_t*>(l_scales + u * SC));
        } else if constexpr (GPC == 2) {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(l_scales + u * SC));
          q.sc[u][0] = v.x; q.sc[u][1] = v.y;
        } else {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(l_scales + u * SC));
          q.sc[u][0] = v.x; q.sc[u][1] = v.y; q.sc[u][2] = v.z; q.sc[u][3] = v.w;
        }
        if constexpr (ZEROS) {
          if constexpr (GPC == 1) {
            q.zr[u][0] = __ldg(reinterpret_cast<const uint16_t*>(l_zeros + u * ZR));
          } else if constexpr (GPC == 2) {
            q.zr[u][0] = __ldg(reinterpret_cast<const uint32_t*>(l_zeros + u * ZR));
          } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(l_zeros + u * ZR));
            q.zr[u][0] = v.x; q.zr[u][1] = v.y;
          }
        }
      }
    }
    l_s += U;
    l_codes += U * 1024;
    l_scales += U * SC;
    if (ZEROS) l_zeros += U * ZR;
    if (l_s >= l_nc && ++l_i < l_end) set_tile();
  };
  auto begin = [&](int round, int pass) {
    l_nc = chunks_of(pass, l_c0);
    l_i = round * p.tpr;
    l_end = l_nc > 0 ? min(mine, l_i + p.tpr) : 0;
    if (l_i < l_end) set_tile();
    load_next(b0);
    load_next(b1);
  };
  // the first weights go out before the wait on the preceding kernel: no kernel of the library writes them
  begin(0, 0);
  if (tid < 64) reinterpret_cast<uint32_t*>(s_zero)[tid] = 0;
  chain_wait();

  uint32_t xp[NT], xstep[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool has = n * 8 + g < rows;
    xp[n] = smem_u32(has ? s_x + (n * 8 + g) * xs : s_zero) + t * 16;
    xstep[n] = has ? 256 : 0;
  }
  bool pending = false;                             // peers may still be reading this CTA's sums
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
      // ---- products
      const int tiles = nc > 0 ? max(0, min(mine - round * p.tpr, p.tpr)) : 0, ppt = (nc + U - 1) / U;
      float4* acc = reinterpret_cast<float4*>(s_acc) + wic * (NT * 32) + lane;
      float tot[NT][4];
      uint32_t x_at[NT], sum_at = 0;
      int s = 0;
      auto reset = [&] {
        s = 0;
        sum_at = smem_u32(s_sum) + t * 8;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          x_at[n] = xp[n];
          tot[n][0] = tot[n][1] = tot[n][2] = tot[n][3] = 0.f;
        }
      };
      auto store = [&] {
        settle();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float4 v = make_float4(tot[n][0], tot[n][1], tot[n][2], tot[n][3]);
          if (pass > 0) {
            const float4 o = acc[n * 32];
            v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
          }
          acc[n * 32] = v;
        }
        acc += WARPS * (NT * 32);
      };
      reset();
      auto step = [&](Batch& q) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (s + u < nc) {
            const uint4 lo = q.lo[u], hi = q.hi[u];
            float2 fx[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) fx[n] = lds_f2(sum_at + u * ((1 + GPC) * COLS * 4) + n * 32);
            constexpr int JPG = 4 / GPC;            // words of a group
#pragma unroll
            for (int grp = 0; grp < GPC; ++grp) {
              float d[NT][4];
#pragma unroll
              for (int jj = 0; jj < JPG; ++jj) {
                const int j = grp * JPG + jj;
                const uint32_t wl = j == 0 ? lo.x : j == 1 ? lo.y : j == 2 ? lo.z : lo.w;
                const uint32_t wh = j == 0 ? hi.x : j == 1 ? hi.y : j == 2 ? hi.z : hi.w;
                const uint32_t ul = wl >> 8, uh = wh >> 8;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const uint4 xv = lds128(x_at[n] + j * 64);
                  mma_f16(d[n], jj == 0, wl & 0x000f000fu, wh & 0x000f000fu, wl & 0x00f000f0u, wh & 0x00f000f0u, xv.x, xv.y);
                  mma_f16(d[n], false, ul & 0x000f000fu, uh & 0x000f000fu, ul & 0x00f000f0u, uh & 0x00f000f0u, xv.z, xv.w);
                }
              }
              // scales lie as [row half][group], halves of words; zeros as bytes. What lies behind K is never used.
              const uint32_t w0 = q.sc[u][grp / 2], w1 = q.sc[u][(GPC + grp) / 2];
              float f0 = __uint_as_float(grp & 1 ? w0 & 0xffff0000u : w0 << 16);
              float f1 = __uint_as_float((GPC + grp) & 1 ? w1 & 0xffff0000u : w1 << 16);
              if (GPC > 1 && grp > 0 && (c0 + s + u) * 128 + grp * GRP >= p.K) f0 = f1 = 0.f;
              float z0 = 1.f, z1 = 1.f;
              if constexpr (ZEROS) {                // 2^23 + zero, minus 2^23
                const uint32_t y0 = q.zr[u][0] >> (8 * grp), y1 = GPC == 4 ? q.zr[u][GPC == 4 ? 1 : 0] >> (8 * grp) : q.zr[u][0] >> (8 * (GPC + grp));
                z0 = __uint_as_float((y0 & 15u) | 0x4b000000u) - 8388608.f;
                z1 = __uint_as_float((y1 & 15u) | 0x4b000000u) - 8388608.f;
              }
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const float2 sx = lds_f2(sum_at + (u * (1 + GPC) + 1 + grp) * (COLS * 4) + n * 32);
                tot[n][0] = fmaf(fmaf(d[n][0], fx[n].x, -z0 * sx.x), f0, tot[n][0]);
                tot[n][1] = fmaf(fmaf(d[n][1], fx[n].y, -z0 * sx.y), f0, tot[n][1]);
                tot[n][2] = fmaf(fmaf(d[n][2], fx[n].x, -z1 * sx.x), f1, tot[n][2]);
                tot[n][3] = fmaf(fmaf(d[n][3], fx[n].y, -z1 * sx.y), f1, tot[n][3]);
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) x_at[n] += xstep[n];
          }
        }
        load_next(q);
        s += U;
        sum_at += U * ((1 + GPC) * COLS * 4);
        if (s >= nc) {
          store();
          reset();
        }
      };
      const int pieces = tiles * ppt;
      for (int f = 0; f < pieces; f += 2) {
        step(b0);
        if (f + 1 < pieces) step(b1);
      }
      if (nc == 0 && pass == 0) {                   // more CTAs than chunks: sums of nothing
        for (int i = round * p.tpr; i < min(mine, (round + 1) * p.tpr); ++i) store();
      }
      if (pass + 1 < p.passes) begin(round, pass + 1);
      else if (round + 1 < p.rounds) begin(round + 1, 0);
    }
    // ---- exchange: every rank finishes its share of the tiles
    settle();
    if (p.cs > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    const int each = gated ? 2 : 1;
    for (int e = tid + WARPS * 32 * rank; e < p.tpr * WARPS / each * (COLS * 16); e += WARPS * 32 * p.cs) {
      const int row = e & 15, b = (e >> 4) % COLS, sl = (e >> 4) / COLS * each;
      const int u = cluster * WARPS + (sl % WARPS) + (round * p.tpr + sl / WARPS) * warps;
      if (u >= p.tiles || b >= rows) continue;
      auto sum_of = [&](int sl_) {
        // row g + 8 i of the tile and activation row 2 t + j: value 2 i + j of lane 4 g + t
        const uint32_t a = smem_u32(s_acc + ((sl_ * NT + (b >> 3)) * 32 + (row & 7) * 4 + ((b & 7) >> 1)) * 4 + (row >> 3) * 2 + (b & 1));
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
    return 2 * device_sms() / cs;
  }
  known[cs].store(most, std::memory_order_relaxed);
  return most;
}

template <int GRP, int NT, bool ZEROS>
int launch_t(Gemv4Dev& p, cudaStream_t s) {
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
  // shared memory: activations with their sums, and sums of products
  constexpr int ROOM = SMEM_LIMIT - 256 - COLS * 64;
  constexpr int TPR_BYTES = WARPS * COLS * 64, SC_BYTES = COLS * (256 + 4 + 4 * (128 / GRP));
  static_assert(ROOM >= TPR_BYTES + 4 * SC_BYTES, "shared memory budget");
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
  const size_t smem = 256 + (size_t)p.sc * SC_BYTES + COLS * 64 + (size_t)p.tpr * TPR_BYTES;
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
