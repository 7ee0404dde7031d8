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
constexpr int RING = 2;         // slots of a warp's ring
constexpr int SMEM_LIMIT = 112 * 1024;

// Chunks of 128 inputs in a slot. Several n-tiles leave less shared memory, and more work behind each chunk
__host__ __device__ constexpr int slot_chunks(int nt) { return nt == 1 ? 4 : 2; }

struct Gemv4Dev {
  const bf16* x; int64_t ldx;
  const uint8_t* xq;            // activations converted by gemv4_convert_kernel, or null: each CTA converts what it needs
  const uint8_t* codes; const uint8_t* scales; const uint8_t* zeros;
  void* out; int64_t ldo;
  int B, N, K, mode, act, n_valid;
  int kt;                       // chunks of 128 inputs
  int tiles;                    // tiles of 16 rows
  int clusters, cs;             // cs CTAs of a cluster share tiles and split their chunks
  int sc, passes;               // chunks of a CTA in a pass over x; passes
  int tpr, rounds;              // tiles of a cluster between two exchanges of sums; such rounds
  int grain;                    // a warp's stretch begins at a multiple of it
  int deal, deal_rest;          // tiles (gated: pairs) of each cluster; how many clusters have one more
  uint32_t sc_inv, per_inv;     // ceil(2^32 / sc), ceil(2^32 / (16 rows)): products with them replace divisions
  int rows;                     // activation rows that shared memory has room for
  int* status;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// D = A B + (first ? 0 : D), m16n8k16
__device__ __forceinline__ void mma_f16(float (&d)[4], bool first, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
  if (first)
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm(
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

// What a lane of a half-warp makes of its 8 of a chunk's 128 activations: f16 values times a common power of two, those that
// meet codes of bits 4 .. 7 divided by 16; `unit` takes them back, `sum` is that of the lane's group.
template <int GRP>
__device__ __forceinline__ uint4 convert8(const uint4& v, float& sum, float& unit) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t m = 0;
  float x[8];
  sum = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m = max(m, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
    x[2 * j] = __uint_as_float(w[j] << 16);
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    sum += x[2 * j] + x[2 * j + 1];
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
  for (int o = 1; o < GRP / 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  // a power of two that brings the largest to 2^14 .. 2^15, as far as fp32 has it (an infinity or NaN stays what it is, beside
  // values that no longer matter)
  const int sh = m == 0 ? 0 : min(14 + 127 - (int)(m >> 7), 126);
  const float f = __uint_as_float((uint32_t)(127 + sh) << 23), f16th = f * 0.0625f;
  unit = __uint_as_float((uint32_t)(127 - sh) << 23);
  return make_uint4(pack_f16(x[0] * f, x[1] * f), pack_f16(x[2] * f16th, x[3] * f16th), pack_f16(x[4] * f, x[5] * f),
                    pack_f16(x[6] * f16th, x[7] * f16th));
}
// Sums of groups in the unit of code products (2^-24), without zeros times the 8 that stands for them
__host__ __device__ constexpr float sum_scale(bool zeros) { return (zeros ? 1.f : 8.f) * 0x1p-24f; }

// Converted activations for many CTAs: per slab of COLS rows [COLS][kt][128] f16, then [kt][1 + GPC][COLS] units and sums. A
// half-warp per row and chunk; bound by launch and one round through memory.
__host__ __device__ constexpr int64_t slab_bytes(int cols, int gpc, int64_t kt) { return kt * cols * (256 + 4 * (1 + gpc)); }
template <int GRP>
__global__ void __launch_bounds__(256) gemv4_convert_kernel(const bf16* __restrict__ x, int64_t ldx, uint8_t* __restrict__ out,
                                                            int B, int K, int kt, int cols, int zeros) {
  constexpr int GPC = 128 / GRP;
  chain_trigger();
  chain_wait();
  const int h = threadIdx.x & 15, c = blockIdx.x * 16 + (threadIdx.x >> 4), r = blockIdx.y, k = c * 128 + h * 8;
  float sum, unit;
  const uint4 q = convert8<GRP>(c < kt && k < K ? *reinterpret_cast<const uint4*>(x + r * ldx + k) : make_uint4(0, 0, 0, 0), sum, unit);
  if (c >= kt) return;
  uint8_t* slab = out + r / cols * slab_bytes(cols, GPC, kt);
  *reinterpret_cast<uint4*>(slab + ((int64_t)(r % cols) * kt + c) * 256 + h * 16) = q;
  float* to = reinterpret_cast<float*>(slab + (int64_t)cols * kt * 256) + (int64_t)c * (1 + GPC) * cols + r % cols;
  if (h == 0) to[0] = unit;
  if (h % (GRP / 8) == 0) to[(1 + h / (GRP / 8)) * cols] = sum * sum_scale(zeros != 0);
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
// + 7. The chunks of a CTA's tiles are one line, of which each warp streams an equal stretch through a ring of its own; bulk
// copies keep more bytes in flight than loads to registers (1 x 4096 -> 128256: 46 us, 5.8 TB/s, against 55). Where there are
// fewer tiles than CTAs, or many rows to convert, the CTAs of a cluster have the same tiles and a part of the inputs each. The
// loop over the chunks stays rolled: each launch meets its instructions cold (unrolled four times: 0.5 to 1 us more a call).
// What a call costs beside its bytes, 1 x 4096 -> 4096 (4.9 us; the bytes take 1.3): launch, 0.5 us to the first copy, 0.9
// until the activations are converted, 0.8 for exchange and stores.
template <int GRP, int NT, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 2) gemv4_kernel(const __grid_constant__ Gemv4Dev p) {
  constexpr int GPC = 128 / GRP, COLS = NT * 8, SC = 32 * GPC, ZR = 16 * GPC, SLOT = slot_chunks(NT);
  constexpr int SLOT_BYTES = SLOT * (1024 + SC + (ZEROS ? ZR : 0));     // codes, then scales, then zeros
  extern __shared__ __align__(128) uint8_t smem[];
  const int xs = p.sc * 256 + 64;                   // bytes of an activation row: 64 off a multiple of 128, so that the
                                                    // rows of a quarter-warp's loads lie in other banks
  const int tid = threadIdx.x, lane = tid & 31, wic = tid >> 5, g = lane >> 2, t = lane & 3;
  const int row0 = blockIdx.y * COLS, rows = min(p.B - row0, COLS);
  const uint8_t* s_ring = smem + wic * (RING * SLOT_BYTES);
  uint8_t* s_zero = smem + WARPS * RING * SLOT_BYTES;             // 256 zeros: what lanes without an activation row read
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(s_zero + 256);    // [WARPS][RING], and one of the activations
  float* s_sum = reinterpret_cast<float*>(s_bar + WARPS * RING + 2);  // [sc][1 + GPC][COLS]: 2^-shift; sums of the groups
  uint8_t* s_x = reinterpret_cast<uint8_t*>(s_sum + p.sc * (1 + GPC) * COLS);
  float* s_acc = reinterpret_cast<float*>(s_x + p.rows * xs);     // [tpr + WARPS][rows][16]
  const int rank = cluster_ctarank();
  int cluster;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(cluster));
  const bool gated = p.mode == 3;
  // Tiles are dealt to the clusters in turn (gated: a gate tile with its up tile, tiles 2 n and 2 n + 1 of the count)
  const int each = gated ? 2 : 1, dealt = (p.deal + (cluster < p.deal_rest ? 1 : 0)) * each;
  auto tile_of = [&](int n) {
    if (!gated) return n * p.clusters + cluster;
    const int pair = (n >> 1) * p.clusters + cluster;
    return (pair >> 3) * 16 + (pair & 7) + 8 * (n & 1);
  };
  // The chunks of a round's tiles, p.sc each, are one line, and each warp has an equal stretch of it; the sums of tile n in
  // warp w's stretch go to place n + w, which no other part has
  auto stretch = [&](int round, int w) {
    const int tiles = max(0, min(p.tpr, dealt - round * p.tpr)), line = tiles * p.sc;
    return min(((line * w >> 3) + p.grain - 1) & -p.grain, line);
  };
  chain_trigger();
  auto chunks_of = [&](int pass, int& c0) {
    c0 = min((pass * p.cs + rank) * p.sc, p.kt);
    return min(p.sc, p.kt - c0);
  };
  const uint32_t ring = smem_u32(s_ring), bar = smem_u32(s_bar + wic * RING);
  if (lane < RING) mbar_init(s_bar + wic * RING + lane, 1);
  if (tid == RING) mbar_init(s_bar + WARPS * RING, 1);
  fence_barrier_init();
  __syncwarp();

  // ---- copies, in the order in which they are used: round, pass over x, tile, chunks
  int l_round = 0, l_pass = 0, l_left = 0, l_slot = 0, l_at = stretch(0, wic), l_end = stretch(0, wic + 1);
  const uint8_t *l_codes = nullptr, *l_scales = nullptr, *l_zeros = nullptr;
  auto issue = [&] {
    while (l_left <= 0) {                           // to the next part of a tile that there is
      if (l_round >= p.rounds) return;
      if (l_at >= l_end) {
        if (++l_pass >= p.passes) {
          l_pass = 0;
          if (++l_round >= p.rounds) return;
        }
        l_at = stretch(l_round, wic);
        l_end = stretch(l_round, wic + 1);
        continue;
      }
      int c0;
      const int nc = chunks_of(l_pass, c0), n = p.sc == 1 ? l_at : (int)__umulhi(l_at, p.sc_inv), s = l_at - n * p.sc, e = min(l_end - n * p.sc, p.sc);
      l_left = min(e, nc) - s;
      l_at += e - s;
      const int64_t chunk = (int64_t)tile_of(l_round * p.tpr + n) * p.kt + c0 + s;
      l_codes = p.codes + chunk * 1024;
      l_scales = p.scales + chunk * SC;
      if (ZEROS) l_zeros = p.zeros + chunk * ZR;
    }
    const int cnt = min(SLOT, l_left);
    if (lane == 0) {
      const uint32_t dst = ring + l_slot * SLOT_BYTES, b = bar + l_slot * 8;
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(cnt * (1024 + SC + (ZEROS ? ZR : 0))) : "memory");
      bulk_load(dst, l_codes, cnt * 1024, b);
      bulk_load(dst + SLOT * 1024, l_scales, cnt * SC, b);
      if (ZEROS) bulk_load(dst + SLOT * (1024 + SC), l_zeros, cnt * ZR, b);
    }
    l_slot = l_slot == RING - 1 ? 0 : l_slot + 1;
    l_left -= cnt;
    l_codes += SLOT * 1024;
    l_scales += SLOT * SC;
    if (ZEROS) l_zeros += SLOT * ZR;
  };
  // the first weights go out before the wait on the preceding kernel: no kernel of the library writes them
#pragma unroll 1
  for (int i = 0; i < RING; ++i) issue();
  if (tid < 64) reinterpret_cast<uint32_t*>(s_zero)[tid] = 0;
  __syncthreads();
  chain_wait();

  const uint8_t* xp[NT];
  int xstep[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool has = n * 8 + g < rows;
    xp[n] = (has ? s_x + (n * 8 + g) * xs : s_zero) + t * 16;
    xstep[n] = has ? 256 : 0;
  }
  int slot = 0;
  uint32_t phase = 0, x_phase = 0;
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
        if (p.xq != nullptr) {
          // converted already: a copy per row, one of the sums
          if (wic == 0) {
            const uint8_t* slab = p.xq + blockIdx.y * slab_bytes(COLS, GPC, p.kt);
            const uint32_t b = smem_u32(s_bar + WARPS * RING), sums = max(nc, 0) * (1 + GPC) * COLS * 4;
            if (lane == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(rows * nc * 256 + sums) : "memory");
            __syncwarp();
            for (int r = lane; r < rows && nc > 0; r += 32)
              bulk_load(smem_u32(s_x + r * xs), slab + ((int64_t)r * p.kt + c0) * 256, nc * 256, b);
            if (lane == 0 && nc > 0)
              bulk_load(smem_u32(s_sum), slab + (int64_t)COLS * p.kt * 256 + (int64_t)c0 * (1 + GPC) * COLS * 4, sums, b);
          }
          if (!mbar_wait(s_bar + WARPS * RING, x_phase)) ok = false;
          x_phase ^= 1;
        } else {
        const int h = lane & 15;
        int r = 0, c = wic * 2 + (lane >> 4);       // of the item; r * nc + c runs in steps of two per warp
        auto wrap = [&] {
          while (c >= nc && r < rows) {
            c -= nc;
            ++r;
          }
        };
        wrap();
        for (int left = rows * nc - wic * 2; left > 0; left -= 4 * (WARPS * 2)) {
          uint4 v[4];                               // four items' loads are in flight
          int ri[4], ci[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ri[i] = r;
            ci[i] = c;
            const int k = (c0 + c) * 128 + h * 8;
            v[i] = r < rows && k < p.K ? *reinterpret_cast<const uint4*>(p.x + (row0 + r) * p.ldx + k) : make_uint4(0, 0, 0, 0);
            c += WARPS * 2;
            wrap();
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (left <= i * (WARPS * 2)) break;     // the same for the warp
            float sum, unit;
            const uint4 q = convert8<GRP>(v[i], sum, unit);
            if (ri[i] < rows) {
              *reinterpret_cast<uint4*>(s_x + ri[i] * xs + ci[i] * 256 + h * 16) = q;
              float* to = s_sum + ci[i] * (1 + GPC) * COLS + ri[i];
              if (h == 0) to[0] = unit;
              if (h % (GRP / 8) == 0) to[(1 + h / (GRP / 8)) * COLS] = sum * sum_scale(ZEROS);
            }
          }
        }
        __syncthreads();
        }
      }
      // ---- products
      const int end = stretch(round, wic + 1);
      for (int at = stretch(round, wic); at < end && ok;) {
        const int n_tile = p.sc == 1 ? at : (int)__umulhi(at, p.sc_inv), s0 = at - n_tile * p.sc, s1 = min(end - n_tile * p.sc, p.sc), se = min(s1, nc);
        at += s1 - s0;
        float tot[NT][4];
        const uint8_t* x_at[NT];
        const float* sum_at = s_sum + t * 2 + s0 * ((1 + GPC) * COLS);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          x_at[n] = xp[n] + s0 * xstep[n];
          tot[n][0] = tot[n][1] = tot[n][2] = tot[n][3] = 0.f;
        }
        for (int s = s0; s < se; s += SLOT) {
          if (!mbar_try_wait(s_bar + wic * RING + slot, phase) && !mbar_wait(s_bar + wic * RING + slot, phase)) {
            ok = false;
            break;
          }
          const uint8_t* base = s_ring + slot * SLOT_BYTES;
          const uint8_t* cb = base + lane * 16;
          const uint8_t* sb = base + SLOT * 1024 + g * (4 * GPC);
          const uint8_t* zb = base + SLOT * (1024 + SC) + g * (2 * GPC);
          auto chunk = [&](const int c) {
            const uint4 lo = *reinterpret_cast<const uint4*>(cb), hi = *reinterpret_cast<const uint4*>(cb + 512);
            uint32_t sw[GPC], zw[2] = {0, 0};
            if constexpr (GPC == 1) {
              sw[0] = *reinterpret_cast<const uint32_t*>(sb);
            } else if constexpr (GPC == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(sb);
              sw[0] = v.x; sw[1] = v.y;
            } else {
              const uint4 v = *reinterpret_cast<const uint4*>(sb);
              sw[0] = v.x; sw[1] = v.y; sw[2] = v.z; sw[3] = v.w;
            }
            if constexpr (ZEROS) {
              if constexpr (GPC == 1) {
                zw[0] = *reinterpret_cast<const uint16_t*>(zb);
              } else if constexpr (GPC == 2) {
                zw[0] = *reinterpret_cast<const uint32_t*>(zb);
              } else {
                const uint2 v = *reinterpret_cast<const uint2*>(zb);
                zw[0] = v.x; zw[1] = v.y;
              }
            }
            float2 fx[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) fx[n] = *reinterpret_cast<const float2*>(sum_at + n * 8);
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
                  const uint4 xv = *reinterpret_cast<const uint4*>(x_at[n] + j * 64);
                  mma_f16(d[n], jj == 0, wl & 0x000f000fu, wh & 0x000f000fu, wl & 0x00f000f0u, wh & 0x00f000f0u, xv.x, xv.y);
                  mma_f16(d[n], false, ul & 0x000f000fu, uh & 0x000f000fu, ul & 0x00f000f0u, uh & 0x00f000f0u, xv.z, xv.w);
                }
              }
              // scales lie as [row half][group], halves of words; zeros as bytes. What lies behind K is never used.
              const uint32_t w0 = sw[grp / 2], w1 = sw[(GPC + grp) / 2];
              float f0 = __uint_as_float(grp & 1 ? w0 & 0xffff0000u : w0 << 16);
              float f1 = __uint_as_float((GPC + grp) & 1 ? w1 & 0xffff0000u : w1 << 16);
              if (GPC > 1 && grp > 0 && (c0 + c) * 128 + grp * GRP >= p.K) f0 = f1 = 0.f;
              float z0 = 1.f, z1 = 1.f;
              if constexpr (ZEROS) {                // 2^23 + zero, minus 2^23
                const uint32_t y0 = zw[0] >> (8 * grp), y1 = GPC == 4 ? zw[1] >> (8 * grp) : zw[0] >> (8 * (GPC + grp));
                z0 = __uint_as_float((y0 & 15u) | 0x4b000000u) - 8388608.f;
                z1 = __uint_as_float((y1 & 15u) | 0x4b000000u) - 8388608.f;
              }
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const float2 sx = *reinterpret_cast<const float2*>(sum_at + (1 + grp) * COLS + n * 8);
                tot[n][0] = fmaf(fmaf(d[n][0], fx[n].x, -z0 * sx.x), f0, tot[n][0]);
                tot[n][1] = fmaf(fmaf(d[n][1], fx[n].y, -z0 * sx.y), f0, tot[n][1]);
                tot[n][2] = fmaf(fmaf(d[n][2], fx[n].x, -z1 * sx.x), f1, tot[n][2]);
                tot[n][3] = fmaf(fmaf(d[n][3], fx[n].y, -z1 * sx.y), f1, tot[n][3]);
              }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) x_at[n] += xstep[n];
          };
          const int cnt = min(SLOT, se - s);
#pragma unroll 1
          for (int q = 0; q < cnt; ++q) {
            chunk(s + q);
            cb += 1024;
            sb += SC;
            zb += ZR;
            sum_at += (1 + GPC) * COLS;
          }
          __syncwarp();
          issue();                                  // into the slot that is free now
          slot = slot == RING - 1 ? 0 : slot + 1;
          phase ^= slot == 0 ? 1u : 0u;
        }
        settle();
        // sum i of n-tile n: row g + 8 (i / 2) of the tile, activation row 2 t + i % 2
        float* acc = s_acc + (n_tile + wic) * (p.rows * 16) + 2 * t * 16 + g;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float* dst = acc + (n * 8 + (r & 1)) * 16 + 8 * (r >> 1);
            if (n * 8 + 2 * t + (r & 1) < rows) *dst = pass == 0 ? tot[n][r] : *dst + tot[n][r];
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
    const int tiles = max(0, min(p.tpr, dealt - round * p.tpr)), per = p.rows * 16, all = tiles / each * per;
    for (int e = rank * (WARPS * 32) + tid; e < all; e += p.cs * (WARPS * 32)) {
      const int n = __umulhi(e, p.per_inv) * each, at = e - n / each * per, tile = tile_of(round * p.tpr + n);
      if (at >= rows * 16) continue;
      auto sum_of = [&](int m) {
        // the parts of tile m in the order of the warps and ranks; they lie in the same places in all ranks
        float v = 0.f, w[WARPS];
        const float* part = s_acc + m * (p.rows * 16) + at;
        auto has = [&](int i) { return max(stretch(round, i), m * p.sc) < min(stretch(round, i + 1), (m + 1) * p.sc); };
        if (p.cs == 1) {
#pragma unroll
          for (int i = 0; i < WARPS; ++i) w[i] = has(i) ? part[i * (p.rows * 16)] : 0.f;
#pragma unroll
          for (int i = 0; i < WARPS; ++i) v += w[i];
        } else {
#pragma unroll 1
          for (int i = 0; i < WARPS; ++i) {
            if (!has(i)) continue;
            const uint32_t a = smem_u32(part + i * (p.rows * 16));
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              w[r] = 0.f;
              if (r < p.cs) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w[r]) : "r"(mapa_u32(a, r)));
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) v += w[r];
          }
        }
        return v * 0x1p24f;
      };
      const int b = row0 + (at >> 4), row = at & 15;
      const float v = sum_of(n);
      if (gated) {
        const float up = sum_of(n + 1);
        const int o = (tile >> 4) * 128 + (tile & 7) * 16 + row;
        if (o < p.n_valid) static_cast<bf16*>(p.out)[(int64_t)b * p.ldo + o] = __float2bfloat16_rn(act_of(v, p.act) * up);
      } else if (tile * 16 + row < p.N) {
        float* dst = static_cast<float*>(p.out) + (int64_t)b * p.ldo + tile * 16 + row;
        *dst = p.mode == 0 ? v : *dst + v;
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
  constexpr int GPC = 128 / GRP, RING_BYTES = WARPS * RING * slot_chunks(NT) * (1024 + 32 * GPC + (ZEROS ? 16 * GPC : 0));
  constexpr int FIXED = RING_BYTES + 256 + (WARPS * RING + 2) * 8 + COLS * 64;
  static_assert(SMEM_LIMIT - FIXED >= (WARPS + 2) * COLS * 64 + 4 * COLS * (256 + 4 + 4 * GPC), "shared memory budget");
  p.rows = p.B < COLS ? p.B : COLS;
  const int room = SMEM_LIMIT - FIXED, acc_bytes = p.rows * 64, sc_bytes = p.rows * 256 + COLS * (4 + 4 * GPC);
  // Work of an SM with two CTAs, in clocks as measured: 30 to convert a row's chunk, 47 (two n-tiles: 75) for a tile's chunk, the
  // exchange within a cluster. us in clusters of 1 / 2 / 8: 1 x 4096 -> 28672 gated 14.8 / 16.0 / 21.2, 1 x 14336 -> 4096 11.4 /
  // 11.4 / 15.0, 12 x 14336 -> 4096 62 / 38 / 24, 16 x 4096 -> 6144 22 / 26 / 14.
  // A pass over part of the inputs, or a round over part of the tiles, costs 6000 more.
  const int each = p.mode == 3 ? 2 : 1, want = p.tiles / each;
  int64_t best = INT64_MAX;
  for (int cs = 1; cs <= 8 && cs <= p.kt; cs *= 2) {
    const int most = max_clusters<GRP, NT, ZEROS>(cs), clusters = want < most ? want : most;
    // all chunks of a CTA at once if they fit beside the sums of two tiles, then as many tiles as fit
    const int dealt = ceil_div(want, clusters) * each, nc = ceil_div(p.kt, cs);
    const int passes = ceil_div(nc, (room - (WARPS + 2) * acc_bytes) / sc_bytes), sc = ceil_div(p.kt, passes * cs);
    const int rounds = ceil_div(dealt, ((room - sc * sc_bytes) / acc_bytes - WARPS) / 2 * 2);
    const int64_t cost = (int64_t)2 * nc * (p.rows * (p.xq ? 2 : 30) + (int64_t)p.tiles * (NT == 1 ? 47 : NT == 2 ? 60 : 90) / clusters) +
                         (cs > 1 ? 4000 + 1000 * cs : 0) + (passes * rounds - 1) * 6000;
    if (cost < best) {
      best = cost;
      p.cs = cs;
      p.clusters = clusters;
      p.passes = passes;
      p.sc = sc;
      p.rounds = rounds;
      p.tpr = ceil_div(dealt / each, rounds) * each;
    }
  }
  p.grain = p.sc % slot_chunks(NT) == 0 ? slot_chunks(NT) : 1;
  p.deal = p.tiles / each / p.clusters;
  p.deal_rest = p.tiles / each % p.clusters;
  p.sc_inv = (uint32_t)(((1ull << 32) + p.sc - 1) / p.sc);
  p.per_inv = (uint32_t)(((1ull << 32) + p.rows * 16 - 1) / (p.rows * 16));
  const int slabs = ceil_div(p.B, COLS);
  if (slabs > 65535) return POP_E_INVALID;
  const size_t smem = FIXED + (size_t)p.sc * sc_bytes + (size_t)(p.tpr + WARPS) * acc_bytes;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  ProfScope prof(PROF_GEMV, (double)p.N * p.K * (0.5 + (p.zeros ? 3.0 : 2.0) / GRP) * slabs, s);
  if (launch_chained_cluster_x(gemv4_kernel<GRP, NT, ZEROS>, dim3(p.clusters * p.cs, slabs), dim3(WARPS * 32), smem, s,
                               (unsigned)p.cs, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

// Rows from which a launch of its own converts the activations
constexpr int CONVERT_ROWS = 3;
constexpr int cols_of(int B) { return B <= 8 ? 8 : B <= 16 ? 16 : 32; }

template <int GRP>
int launch_grp(Gemv4Dev& p, void* workspace, size_t bytes, cudaStream_t s) {
  if (p.B >= CONVERT_ROWS) {
    const int cols = cols_of(p.B), slabs = ceil_div(p.B, cols);
    if (!workspace || (int64_t)bytes < slabs * slab_bytes(cols, 128 / GRP, p.kt)) return POP_E_NOSPACE;
    if (p.B > 65535) return POP_E_INVALID;
    p.xq = static_cast<uint8_t*>(workspace);
    ProfScope prof(PROF_ELEMENTWISE, (double)p.B * p.K * 4, s);
    if (launch_chained(gemv4_convert_kernel<GRP>, dim3(ceil_div(p.kt, 16), p.B), dim3(256), 0, s, p.x, p.ldx,
                       static_cast<uint8_t*>(workspace), p.B, p.K, p.kt, cols, p.zeros ? 1 : 0) != cudaSuccess)
      return POP_E_CUDA;
    count_launch();
  }
  if (p.zeros) return p.B <= 8 ? launch_t<GRP, 1, true>(p, s) : p.B <= 16 ? launch_t<GRP, 2, true>(p, s) : launch_t<GRP, 4, true>(p, s);
  return p.B <= 8 ? launch_t<GRP, 1, false>(p, s) : p.B <= 16 ? launch_t<GRP, 2, false>(p, s) : launch_t<GRP, 4, false>(p, s);
}

}  // namespace

size_t gemv4_workspace_bytes(int B, int K, int group) {
  if (B < CONVERT_ROWS || K < 1 || (group != 32 && group != 64 && group != 128)) return 0;
  return (size_t)(ceil_div(B, cols_of(B)) * slab_bytes(cols_of(B), 128 / group, ceil_div(K, 128)));
}

int launch_gemv4(const Gemv4Args& a, cudaStream_t s) {
  if (!a.x || !a.codes || !a.scales || !a.out || a.B < 1 || a.N < 1 || a.K < 8 || a.K % 8) return POP_E_INVALID;
  if (a.mode != 0 && a.mode != 2 && a.mode != 3) return POP_E_INVALID;
  if (a.group != 32 && a.group != 64 && a.group != 128) return POP_E_INVALID;
  if (a.mode == 3 && (a.N % 256 || a.n_valid < 0 || a.n_valid > a.N / 2 || (a.act != 0 && a.act != 1))) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.x) % 16 || a.ldx % 8 || reinterpret_cast<uintptr_t>(a.codes) % 16 ||
      reinterpret_cast<uintptr_t>(a.scales) % 16 || reinterpret_cast<uintptr_t>(a.workspace) % 16 || reinterpret_cast<uintptr_t>(a.zeros) % 16 ||
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
    case 32: return launch_grp<32>(p, a.workspace, a.workspace_bytes, s);
    case 64: return launch_grp<64>(p, a.workspace, a.workspace_bytes, s);
    default: return launch_grp<128>(p, a.workspace, a.workspace_bytes, s);
  }
}

}  // namespace pop
