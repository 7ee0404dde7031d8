// Projections with 4-bit weights for more rows than a warp-level product covers (drafts of several sequences, or long ones):
//   out[b][n] = sum_k x[b][k] (code[n][k] - zero[n][k / group]) scale[n][k / group]
// with the operands and the exactness of gemv4.cu, on the tensor cores' own memory.
//
// A tile is 128 weight rows and, chunk by chunk, 128 inputs. Two masks per code word (see gemv4.cu) make f16 pairs of it, which
// go to TMEM as the A operand in the order in which a lane finds them; the converted activations lie in the matching order of
// inputs and come as B, swizzled, in one piece per chunk. The sums of a group are fp32 in TMEM, from zero; what enters the
// row's sum in registers is
//   scale (2^-shift sum - zero sum_k x_k).
// The CTAs of a cluster have the same tile (gated: its gate and its up tile) and a part of the inputs each, and join their sums
// through distributed shared memory, in the order of the parts.
// Warps of a CTA, which has an SM to itself (two smaller ones per SM, a chunk a step, took 14 % more for 12 x 14336 -> 4096 and 32 %
// more for 64 x 4096 -> 6144; what a step costs beside its work is many waits):
//   8 warps: the codes of a step of two chunks, a tile of 16 rows each, to TMEM;
//   8 warps: the sums of the groups from TMEM, 32 rows and half of the columns each;
//   1 warp: copies of codes, scales, zeros (a tensor map each: a copy per 16 rows made the copying warp the slowest of all, at 72
//       clocks an instruction) and activations with their sums, through a ring of steps
//       (activations converted here instead: 29 % more for 12 x 14336 -> 4096 by the first eight warps, 51 % more by four others);
//   1 or 2 warps: the products.
// A step takes 1250 clocks with 16 columns: the codes are four times their bytes as f16, 64 KB that are written to TMEM and read
// from it; with 64 columns 2000, the sums' arithmetic. us: 12 x 14336 -> 4096 16.8, 64 x 4096 -> 6144 15.0, with groups of 32 31.6.
#include "common.cuh"
#include "ptx.cuh"
#include "w4.cuh"

#include <atomic>

namespace pop {
namespace {

constexpr int SPREAD = 8, FLUSH = 8;      // warps that bring codes to TMEM, and that take the sums
constexpr int COPY_WARP = SPREAD + FLUSH, MMA_WARP = COPY_WARP + 1;
constexpr int SMEM_BYTES = 227 * 1024;

template <int GRP, int NB, bool ZEROS>
struct G4 {
  static constexpr int GPC = 128 / GRP;
  static constexpr int SC = 32 * GPC, ZR = 16 * GPC;                    // bytes of scales and zeros of 16 rows
  static constexpr int COLS = NB / 2;                                   // of a flushing warp, with 32 rows
  // a step is two chunks of 128 inputs
  static constexpr int X_BYTES = (int)slab_bytes(NB, GPC, 2);           // activations, then their units and sums
  static constexpr int SUMS = NB * 512, CODES = (X_BYTES + 127) / 128 * 128, SCALES = CODES + 16384, ZEROS_AT = SCALES + 16 * SC;
  static constexpr int STAGE_BYTES = ZEROS_AT + (ZEROS ? 16 * ZR : 0);
  static constexpr int STAGE = (STAGE_BYTES + 1023) / 1024 * 1024;
  static constexpr int STAGES = (SMEM_BYTES - 2048) / STAGE < 8 ? (SMEM_BYTES - 2048) / STAGE : 8;
  static constexpr int BATCH = 2 * GPC * NB <= 128 ? 2 * GPC : 128 / NB;        // groups whose sums are taken together
  // Where a step fills one buffer of sums, two warps issue products, every second step each, with buffers of its own
  static constexpr int ISSUERS = BATCH == 2 * GPC ? 2 : 1, THREADS = (MMA_WARP + ISSUERS) * 32;
  static constexpr int D_COLS = BATCH * NB, D_BUFS = 256 / D_COLS < 4 ? 256 / D_COLS : 4;
  static constexpr int A_COL = 256;                                     // two steps of codes, 128 columns each
  static_assert(STAGES >= 3 && STAGES * STAGE >= NB * 512, "ring too shallow");
};

struct __align__(1024) G4Smem {
  uint64_t full[8], empty[8];
  uint64_t a_ready[2], a_free[2];       // codes of chunk f in TMEM, buffer f & 1
  uint64_t d_full[4], d_empty[4];
  uint32_t tmem_base;
  volatile uint32_t abort;
};
static_assert(sizeof(G4Smem) == 1024, "ring begins behind it");

struct G4Dev {
  const uint8_t* xq;
  void* out; int64_t ldo;
  int B, N, K, mode, act, n_valid;
  int steps;                    // of two chunks of 128 inputs
  int cs;                       // parts of the steps
  int wide;                     // four outputs at a time may be stored
  int* status;
};

template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t from, float (&d)[N]) {
  if constexpr (N == 16) tmem_ld_32x32b_x16(from, reinterpret_cast<uint32_t(&)[16]>(d));
  else tmem_ld_32x32b_x8(from, reinterpret_cast<uint32_t(&)[8]>(d));
}

template <int GRP, int NB, bool ZEROS>
__global__ void __launch_bounds__(G4<GRP, NB, ZEROS>::THREADS, 1)
gemm4_kernel(const __grid_constant__ CUtensorMap tm_codes, const __grid_constant__ CUtensorMap tm_scales,
             const __grid_constant__ CUtensorMap tm_zeros, const __grid_constant__ G4Dev p) {
  using C = G4<GRP, NB, ZEROS>;
  constexpr int GPC = C::GPC, STAGES = C::STAGES, THREADS = C::THREADS;
  extern __shared__ uint8_t smem_raw[];
  G4Smem& s = *reinterpret_cast<G4Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = reinterpret_cast<uint8_t*>(&s) + 1024;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool gated = p.mode == 3;
  const int each = gated ? 2 : 1, rank = cluster_ctarank(), part = rank / each;
  const int unit = blockIdx.x / (p.cs * each), tile = unit * each + rank % each;
  const int first = (int)((int64_t)p.steps * part / p.cs), n_steps = (int)((int64_t)p.steps * (part + 1) / p.cs) - first;
  const int row0 = blockIdx.y * NB;
  chain_trigger();
  if (warp == COPY_WARP) {
    if (lane == 0) {
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(&s.full[i], 1);
        mbar_init(&s.empty[i], FLUSH);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s.a_ready[i], SPREAD);
        mbar_init(&s.a_free[i], 1);
      }
      for (int i = 0; i < C::D_BUFS; ++i) {
        mbar_init(&s.d_full[i], 1);
        mbar_init(&s.d_empty[i], FLUSH);
      }
      s.abort = 0;
      fence_barrier_init();
      prefetch_tmap(&tm_codes);
      prefetch_tmap(&tm_scales);
      if (ZEROS) prefetch_tmap(&tm_zeros);
    }
    __syncwarp();
  }
  // ---- copies. Tiles behind the last count, and are zeros
  auto copy_weights = [&](int f) {
    uint8_t* dst = ring + f % STAGES * C::STAGE;
    uint64_t* bar = &s.full[f % STAGES];
    if (lane == 0) {
      mbar_expect_tx(bar, C::STAGE_BYTES - C::CODES + C::X_BYTES);
      tma_load_3d(dst + C::CODES, &tm_codes, bar, 0, (first + f) * 2, tile * 8);
      tma_load_3d(dst + C::SCALES, &tm_scales, bar, 0, (first + f) * 2, tile * 8);
      if (ZEROS) tma_load_3d(dst + C::ZEROS_AT, &tm_zeros, bar, 0, (first + f) * 2, tile * 8);
    }
  };
  auto copy_x = [&](int f) {
    if (lane == 0)
      bulk_load(smem_u32(ring + f % STAGES * C::STAGE), p.xq + blockIdx.y * (int64_t)p.steps * C::X_BYTES + (int64_t)(first + f) * C::X_BYTES,
                C::X_BYTES, smem_u32(&s.full[f % STAGES]));
  };
  const int ahead = min(n_steps, STAGES);
  // the first weights go out before the wait on the preceding kernel: no kernel of the library writes them
  if (warp == COPY_WARP)
    for (int f = 0; f < ahead; ++f) copy_weights(f);
  chain_wait();
  if (warp == MMA_WARP) {
    // columns that a CTA of another call has not given back yet are waited for: that CTA waits for nobody
    tmem_alloc(&s.tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s.tmem_base;
  bool ok = true;
  // A test that does not suspend sees a complete barrier earlier (4 % of 12 x 14336 -> 4096, 6 % of 32 x 4096 -> 6144); with 64
  // columns the longer code costs more than it gives (8 % with groups of 32)
  auto wait = [](uint64_t* bar, uint32_t parity) { return (NB < 64 && mbar_test(bar, parity)) || mbar_wait(bar, parity); };

  float2 acc[C::COLS / 2];

  if (warp == COPY_WARP) {
    for (int f = 0; f < ahead; ++f) copy_x(f);
    for (int f = ahead; f < n_steps && ok && !s.abort; ++f) {
      ok = mbar_wait_relaxed(&s.empty[f % STAGES], (f / STAGES - 1) & 1);
      if (!ok) break;
      copy_weights(f);
      copy_x(f);
    }
  } else if (warp >= MMA_WARP) {
    // f16 operands, fp32 sums, 128 x NB
    constexpr uint32_t idesc = umma_idesc_f16(128, NB);
    const uint32_t leader = elect_one();
    const uint64_t x_desc = umma_smem_desc(smem_u32(ring), 16, 1024);
    int buf = warp - MMA_WARP, turn = 0;
    for (int f = warp - MMA_WARP; f < n_steps && ok && !s.abort; f += C::ISSUERS) {
      const int stage = f % STAGES;
      const uint64_t xd = x_desc + uint64_t(stage * (C::STAGE >> 4));
      ok = wait(&s.full[stage], (f / STAGES) & 1) && wait(&s.a_ready[f & 1], (f >> 1) & 1);
#pragma unroll 1
      for (int g0 = 0; g0 < 2 * GPC && ok; g0 += C::BATCH) {
        if (turn > 0) ok = wait(&s.d_empty[buf], (turn - 1) & 1);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < C::BATCH * (GRP / 16); ++kk) {
          const int k = g0 * (GRP / 16) + kk;
          umma_bf16_ts_w(leader, tmem + buf * C::D_COLS + kk / (GRP / 16) * NB, tmem + C::A_COL + (f & 1) * 128 + k * 8,
                         xd + uint64_t(((k >> 2) * (NB * 128) + (k & 3) * 32) >> 4), idesc, kk % (GRP / 16) > 0 ? 1u : 0u);
        }
        umma_commit_w(leader, &s.d_full[buf]);
        buf += C::ISSUERS;
        if (buf >= C::D_BUFS) {
          buf -= C::D_BUFS;
          ++turn;
        }
      }
      umma_commit_w(leader, &s.a_free[f & 1]);
    }
  } else if (warp < SPREAD) {
    // the codes of a tile of 16 rows, which are in this warp's quarter of TMEM
    const int quarter = warp & 3, half = warp >> 2;
    for (int f = 0; f < n_steps; ++f) {
      const int stage = f % STAGES;
      ok = wait(&s.full[stage], (f / STAGES) & 1);
      const uint8_t* src = ring + stage * C::STAGE + C::CODES + (2 * quarter + half) * 2048 + lane * 16;
      uint4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4*>(src + i * 512);
      if (f >= 2 && ok) ok = wait(&s.a_free[f & 1], ((f >> 1) - 1) & 1);
      ok = warp_agrees(ok);                             // a role whose work has stopped ends at its own limit
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t wl[4] = {w[2 * c].x, w[2 * c].y, w[2 * c].z, w[2 * c].w};
        const uint32_t wh[4] = {w[2 * c + 1].x, w[2 * c + 1].y, w[2 * c + 1].z, w[2 * c + 1].w};
        uint32_t a[32];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t mask = i & 1 ? 0x00f000f0u : 0x000f000fu;
            a[(4 * j + i) * 2] = (wl[j] >> (i & 2) * 4) & mask;
            a[(4 * j + i) * 2 + 1] = (wh[j] >> (i & 2) * 4) & mask;
          }
        tmem_st_16x128b_x16(tmem + (uint32_t(quarter * 32 + half * 16) << 16) + C::A_COL + (f & 1) * 128 + c * 64, a);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.a_ready[f & 1]);
    }
  } else {
    const int row = (warp & 3) * 32 + lane, col = (warp - SPREAD >> 2) * C::COLS;
    const uint32_t from = tmem + (uint32_t((warp & 3) * 32) << 16) + col;
    // of the row's scales of a step's first chunk
    const int at = (row >> 4) * 2 * 16 * GPC + (2 * (row & 7) + ((row >> 3) & 1)) * GPC;
#pragma unroll
    for (int i = 0; i < C::COLS / 2; ++i) acc[i] = make_float2(0.f, 0.f);
    int buf = 0, turn = 0;
    for (int f = 0; f < n_steps && ok; ++f) {
      const int stage = f % STAGES;
      const uint8_t* base = ring + stage * C::STAGE;
      const float* sums = reinterpret_cast<const float*>(base + C::SUMS) + col;
      const bool here = wait(&s.full[stage], (f / STAGES) & 1);
#pragma unroll 1
      for (int g0 = 0; g0 < 2 * GPC && ok; g0 += C::BATCH) {
        float2 sc2[C::BATCH], z2[C::BATCH];
#pragma unroll
        for (int b = 0; b < C::BATCH; ++b) {
          const int q = g0 + b, grp = q % GPC, place = at + q / GPC * (16 * GPC) + grp;
          float scale = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(base + C::SCALES + place * 2) << 16);
          // what lies behind K is never used
          if (q > 0 && (first + f) * 256 + q * GRP >= p.K) scale = 0.f;
          const float z = ZEROS ? (float)(base[C::ZEROS_AT + place] & 15) : 1.f;
          sc2[b] = make_float2(scale, scale);
          z2[b] = make_float2(z, z);
        }
        ok = warp_agrees(here && wait(&s.d_full[buf], turn & 1));
        if (!ok) break;
        tc_fence_after();
        // as many sums at once as registers have room for
        constexpr int PIECE = C::COLS < 16 ? C::COLS : 16, AT_ONCE = C::COLS == 32 ? 1 : 32 / PIECE < C::BATCH ? 32 / PIECE : C::BATCH;
#pragma unroll
        for (int b0 = 0; b0 < C::BATCH; b0 += AT_ONCE)
#pragma unroll
          for (int c = 0; c < C::COLS; c += PIECE) {
            float d[AT_ONCE][PIECE];
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) tmem_ld_cols<PIECE>(from + buf * C::D_COLS + (b0 + b) * NB + c, d[b]);
            tmem_wait_ld();
            if (b0 + AT_ONCE == C::BATCH && c + PIECE == C::COLS) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&s.d_empty[buf]);
            }
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) {
              const float* units = sums + (g0 + b0 + b) / GPC * ((1 + GPC) * NB) + c;
              const float* of = units + (1 + (g0 + b0 + b) % GPC) * NB;
#pragma unroll
              for (int i = 0; i < PIECE / 4; ++i) {
                const float4 u = *reinterpret_cast<const float4*>(units + i * 4);
                const float4 x = *reinterpret_cast<const float4*>(of + i * 4);
                float2& t0 = acc[c / 2 + i * 2];
                float2& t1 = acc[c / 2 + i * 2 + 1];
                // the sums of activations are negative, and without zeros times the 8 that stands for them
                float2 x0 = make_float2(x.x, x.y), x1 = make_float2(x.z, x.w);
                if constexpr (ZEROS) {
                  x0 = __fmul2_rn(z2[b0 + b], x0);
                  x1 = __fmul2_rn(z2[b0 + b], x1);
                }
                t0 = __ffma2_rn(__ffma2_rn(make_float2(d[b][i * 4], d[b][i * 4 + 1]), make_float2(u.x, u.y), x0), sc2[b0 + b], t0);
                t1 = __ffma2_rn(__ffma2_rn(make_float2(d[b][i * 4 + 2], d[b][i * 4 + 3]), make_float2(u.z, u.w), x1), sc2[b0 + b], t1);
              }
            }
          }
        if (++buf == C::D_BUFS) {
          buf = 0;
          ++turn;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.empty[stage]);
    }
  }
  if (!ok) {
    s.abort = 1;
    atomicMin(p.status, (int)POP_E_DEVICE_TIMEOUT);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // let in-flight bulk copies land
  }
  tc_fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  // ---- the parts' sums, [column][row], over the ring: every copy has landed
  float* parts = reinterpret_cast<float*>(ring);
  if (warp >= SPREAD && warp < COPY_WARP) {
    const int row = (warp & 3) * 32 + lane, col = (warp - SPREAD >> 2) * C::COLS;
#pragma unroll
    for (int i = 0; i < C::COLS / 2; ++i) {
      parts[(col + 2 * i) * 128 + row] = acc[i].x;
      parts[(col + 2 * i + 1) * 128 + row] = acc[i].y;
    }
  }
  cluster_arrive();
  cluster_wait();
  const int cols = min(NB, p.B - row0);
  const uint32_t mine = smem_u32(parts);
  for (int e = rank * THREADS + tid; e < cols * 32; e += p.cs * each * THREADS) {
    const int col = e >> 5, r4 = (e & 31) * 4;
    auto joined = [&](int which) {
      float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i0 = 0; i0 < 8; i0 += 4) {
        float4 v[4];
        if (i0 >= p.cs) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (i0 + i < p.cs)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w)
                         : "r"(mapa_u32(mine + (col * 128 + r4) * 4, (i0 + i) * each + which)));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          t.x += v[i].x;
          t.y += v[i].y;
          t.z += v[i].z;
          t.w += v[i].w;
        }
      }
      return make_float4(t.x * 0x1p24f, t.y * 0x1p24f, t.z * 0x1p24f, t.w * 0x1p24f);
    };
    const float4 v = joined(0);
    const float r[4] = {v.x, v.y, v.z, v.w};
    if (gated) {
      const float4 up = joined(1);
      const float u[4] = {up.x, up.y, up.z, up.w};
      const int o = unit * 128 + r4;
      bf16* dst = static_cast<bf16*>(p.out) + (int64_t)(row0 + col) * p.ldo + o;
      bf16 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = __float2bfloat16_rn(act_of(r[i], p.act) * u[i]);
      if (p.wide && o + 3 < p.n_valid) {
        *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (o + i < p.n_valid) dst[i] = y[i];
      }
    } else {
      const int n = tile * 128 + r4;
      float* dst = static_cast<float*>(p.out) + (int64_t)(row0 + col) * p.ldo + n;
      if (p.wide && n + 3 < p.N) {
        float4 o = v;
        if (p.mode == 2) {
          const float4 was = *reinterpret_cast<const float4*>(dst);
          o = make_float4(v.x + was.x, v.y + was.y, v.z + was.z, v.w + was.w);
        }
        *reinterpret_cast<float4*>(dst) = o;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < p.N) dst[i] = p.mode == 0 ? r[i] : dst[i] + r[i];
      }
    }
  }
  cluster_arrive();                                   // its peers have read this CTA's sums
  cluster_wait();
}

// Clusters of n CTAs that the GPU holds at once (of the device that was current at the first call)
template <int GRP, int NB, bool ZEROS>
int max_clusters(int n) {
  static std::atomic<int> known[9];
  int most = known[n].load(std::memory_order_relaxed);
  if (most > 0) return most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n);
  cfg.blockDim = dim3(G4<GRP, NB, ZEROS>::THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = n;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&most, gemm4_kernel<GRP, NB, ZEROS>, &cfg) != cudaSuccess || most < 1) {
    cudaGetLastError();
    return device_sms() / n;
  }
  known[n].store(most, std::memory_order_relaxed);
  return most;
}

template <int GRP, int NB, bool ZEROS>
int launch_t(const Gemv4Args& a, G4Dev& p, cudaStream_t s) {
  using C = G4<GRP, NB, ZEROS>;
  static std::atomic<uint64_t> configured{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return POP_E_CUDA;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev >= 64 || !(configured.load(std::memory_order_relaxed) & bit)) {
    if (cudaFuncSetAttribute(gemm4_kernel<GRP, NB, ZEROS>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES) != cudaSuccess)
      return POP_E_CUDA;
    configured.fetch_or(bit, std::memory_order_relaxed);
  }
  const int each = p.mode == 3 ? 2 : 1, units = ceil_div(p.N, 128 * each), slabs = ceil_div(p.B, NB);
  if (slabs > 65535 || (int64_t)units * each * 8 > 0x7fffffff) return POP_E_INVALID;
  // parts of the inputs: waves of clusters, each of its chunks and of what a CTA costs beside them, in chunks. us in 1 / 2 / 4 / 5
  // parts: 12 x 14336 -> 4096 40.2 / 23.5 / 16.9 / 27.7 (two waves), 16 x 4096 -> 6144 14.1 / 10.3 / 14.9 (two waves) / 15.7
  int64_t best = INT64_MAX;
  for (int cs = 1; cs * each <= 8 && cs <= p.steps; ++cs) {
    const int most = max_clusters<GRP, NB, ZEROS>(cs * each);
    const int64_t cost = ceil_div((int64_t)units * slabs, (int64_t)most) * (ceil_div(p.steps, cs) * 2 + 6 + cs);
    if (cost < best) {
      best = cost;
      p.cs = cs;
    }
  }
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  CUtensorMap codes, scales, zeros;
  const uint64_t tiles16 = ceil_div(p.N, 16), kt = ceil_div(p.K, 128);
  if (make_tmap_u32_tiles(&codes, a.codes, 256, kt, tiles16, 2, 8) != POP_OK ||
      make_tmap_u32_tiles(&scales, a.scales, C::SC / 4, kt, tiles16, 2, 8) != POP_OK)
    return POP_E_CUDA;
  if (ZEROS) {
    if (make_tmap_u32_tiles(&zeros, a.zeros, C::ZR / 4, kt, tiles16, 2, 8) != POP_OK) return POP_E_CUDA;
  } else {
    zeros = scales;
  }
  ProfScope prof(PROF_GEMV, (double)p.N * p.K * (0.5 + (ZEROS ? 3.0 : 2.0) / GRP) * slabs, s);
  if (launch_chained_cluster_x(gemm4_kernel<GRP, NB, ZEROS>, dim3((unsigned)(units * p.cs * each), slabs), dim3(C::THREADS), SMEM_BYTES,
                               s, (unsigned)(p.cs * each), codes, scales, zeros, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

template <int GRP, bool ZEROS>
int launch_nb(const Gemv4Args& a, G4Dev& p, cudaStream_t s) {
  switch (cols_of(p.B)) {
    case 16: return launch_t<GRP, 16, ZEROS>(a, p, s);
    case 32: return launch_t<GRP, 32, ZEROS>(a, p, s);
    default: return launch_t<GRP, 64, ZEROS>(a, p, s);
  }
}

}  // namespace

int launch_gemm4(const Gemv4Args& a, const uint8_t* xq, cudaStream_t s) {
  G4Dev p{};
  p.xq = xq;
  p.out = a.out; p.ldo = a.ldo;
  p.B = a.B; p.N = a.N; p.K = a.K; p.mode = a.mode; p.act = a.act; p.n_valid = a.n_valid;
  p.steps = ceil_div(a.K, 256);
  p.wide = reinterpret_cast<uintptr_t>(a.out) % (a.mode == 3 ? 8 : 16) == 0 && a.ldo % 4 == 0;
  switch (a.group) {
    case 32: return a.zeros ? launch_nb<32, true>(a, p, s) : launch_nb<32, false>(a, p, s);
    case 64: return a.zeros ? launch_nb<64, true>(a, p, s) : launch_nb<64, false>(a, p, s);
    default: return a.zeros ? launch_nb<128, true>(a, p, s) : launch_nb<128, false>(a, p, s);
  }
}

}  // namespace pop
