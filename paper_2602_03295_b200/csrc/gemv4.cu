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

constexpr int SLOT = 4;         // chunks of 128 inputs in a slot
constexpr int COLS = 8;         // activation rows of a product

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
  int rows;                     // activation rows that shared memory has room for
  uint32_t sc_inv, per_inv;     // ceil(2^32 / sc), ceil(2^32 / (16 rows)): products with them replace divisions
  int* status;
};

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
// Converted activations for many CTAs: per slab of `cols` rows f16 values, then [kt][1 + GPC][cols] units and sums. The values
// lie as [cols][kt][128]; for slabs of more than 8 rows, chunks come in pairs (K as if filled up with zeros), the values as
// gemm4.cu's products read them in front of the units and the (negative) sums. A half-warp per row and chunk; bound by launch
// and one round through memory.
template <int GRP>
__global__ void __launch_bounds__(256) gemv4_convert_kernel(const bf16* __restrict__ x, int64_t ldx, uint8_t* __restrict__ out,
                                                            int B, int K, int kt, int cols, int zeros) {
  constexpr int GPC = 128 / GRP;
  chain_trigger();
  chain_wait();
  const int h = threadIdx.x & 15, c = blockIdx.x * 16 + (threadIdx.x >> 4), r = blockIdx.y, k = c * 128 + h * 8;
  float sum, unit;
  const uint4 q = convert8<GRP>(c < kt && k < K ? *reinterpret_cast<const uint4*>(x + r * ldx + k) : make_uint4(0, 0, 0, 0),
                                cols == 8 ? sum_scale(zeros != 0) : -sum_scale(zeros != 0), sum, unit);
  if (c >= kt) return;
  uint8_t* slab = out + r / cols * slab_bytes(cols, GPC, kt);
  if (cols == 8) {
    *reinterpret_cast<uint4*>(slab + ((int64_t)(r % cols) * kt + c) * 256 + h * 16) = q;
  } else {
    // a pair of inputs 32 j + 8 t + 2 i goes to 32 j + 8 i + 2 t of the chunk; 64 inputs are a row of 128 swizzled bytes
    const int j = h >> 2, t = h & 3, row = r % cols;
    uint8_t* to = slab + (c >> 1) * slab_bytes(cols, GPC, 2) + (c & 1) * (cols * 256) + (j >> 1) * (cols * 128) + row * 128 + 4 * t;
    const uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(to + ((4 * (j & 1) + i) ^ (row & 7)) * 16) = v[i];
  }
  float* to = reinterpret_cast<float*>(cols == 8 ? slab + (int64_t)cols * kt * 256 + (int64_t)c * (1 + GPC) * cols * 4
                                                 : slab + (c >> 1) * slab_bytes(cols, GPC, 2) + cols * 512 + (c & 1) * ((1 + GPC) * cols * 4)) +
              r % cols;
  if (h == 0) to[0] = unit;
  if (h % (GRP / 8) == 0) to[(1 + h / (GRP / 8)) * cols] = sum;
}

// A code in the low bits of an f16 is code * 2^-24, in bits 4 .. 7 code * 2^-20: subnormals are linear, so that a mask alone
// makes a tensor-core operand of two codes of a word, and one shift the other half of them. The activations go in as f16 too,
// those of a chunk of 128 inputs times a power of two that brings their largest to 2^15 or more (bf16 values stay exact down to
// 2^-28 of it, and within 2^-36 of it below), inputs that meet the codes of bits 4 .. 7 divided by 16. So all products are
// exact; a group's sum is built in the MMA's fp32 accumulator from zero and enters the row's fp32 sum as
//   scale (2^-shift sum_k code_k x'_k - zero sum_k x_k),   the second sum made once with the conversion.
// (Subtracting the zero from every pair of codes took 32 more operations per KB of codes; codes as bf16 128 + code, 64.)
//
// The weight rows are the M side of the warp-level MMA, 8 activation rows of a grid row its N side (many: gemm4.cu): a tile of 16 rows x 128 inputs
// is 1 KB in one piece, 16 bytes of row g and 16 of row g + 8 to lane (g = lane / 4, t = lane % 4), word j inputs 32 j + 8 t ..
// + 7. The chunks of a CTA's tiles are one line, of which each warp streams an equal stretch through a ring of its own; bulk
// copies keep more bytes in flight than loads to registers (1 x 4096 -> 128256: 47 us, 5.7 TB/s; loads took a fifth more). Where there are
// fewer tiles than CTAs, or many rows to convert, the CTAs of a cluster have the same tiles and a part of the inputs each. The
// loop over the chunks stays rolled: each launch meets its instructions cold (unrolled four times: 0.5 to 1 us more a call).
// What a call costs beside its bytes, 1 x 4096 -> 4096 (4.9 us; the bytes take 1.3): launch, 0.5 us to the first copy, 0.9
// until the activations are converted, 0.8 for exchange and stores.
template <int GRP, bool ZEROS>
__global__ void __launch_bounds__(WARPS * 32, 2) gemv4_kernel(const __grid_constant__ Gemv4Dev p) {
  constexpr int GPC = 128 / GRP, SC = 32 * GPC, ZR = 16 * GPC;
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

  const uint8_t* xp = (g < rows ? s_x + g * xs : s_zero) + t * 16;
  const int xstep = g < rows ? 256 : 0;
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
            const uint32_t b = smem_u32(s_bar + WARPS * RING), sums = max(nc, 0) * (1 + GPC) * COLS * 4;
            if (lane == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(rows * nc * 256 + sums) : "memory");
            __syncwarp();
            for (int r = lane; r < rows && nc > 0; r += 32)
              bulk_load(smem_u32(s_x + r * xs), p.xq + ((int64_t)r * p.kt + c0) * 256, nc * 256, b);
            if (lane == 0 && nc > 0)
              bulk_load(smem_u32(s_sum), p.xq + (int64_t)COLS * p.kt * 256 + (int64_t)c0 * (1 + GPC) * COLS * 4, sums, b);
          }
          if (!warp_agrees(mbar_wait(s_bar + WARPS * RING, x_phase))) ok = false;
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
            const uint4 q = convert8<GRP>(v[i], sum_scale(ZEROS), sum, unit);
            if (ri[i] < rows) {
              *reinterpret_cast<uint4*>(s_x + ri[i] * xs + ci[i] * 256 + h * 16) = q;
              float* to = s_sum + ci[i] * (1 + GPC) * COLS + ri[i];
              if (h == 0) to[0] = unit;
              if (h % (GRP / 8) == 0) to[(1 + h / (GRP / 8)) * COLS] = sum;
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
        float tot[4] = {0.f, 0.f, 0.f, 0.f};
        const uint8_t* x_at = xp + s0 * xstep;
        const float* sum_at = s_sum + t * 2 + s0 * ((1 + GPC) * COLS);
        for (int s = s0; s < se; s += SLOT) {
          if (!warp_agrees(mbar_try_wait(s_bar + wic * RING + slot, phase) || mbar_wait(s_bar + wic * RING + slot, phase))) {
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
            const float2 fx = *reinterpret_cast<const float2*>(sum_at);
            constexpr int JPG = 4 / GPC;            // words of a group
#pragma unroll
            for (int grp = 0; grp < GPC; ++grp) {
              float d[4];
#pragma unroll
              for (int jj = 0; jj < JPG; ++jj) {
                const int j = grp * JPG + jj;
                const uint32_t wl = j == 0 ? lo.x : j == 1 ? lo.y : j == 2 ? lo.z : lo.w;
                const uint32_t wh = j == 0 ? hi.x : j == 1 ? hi.y : j == 2 ? hi.z : hi.w;
                const uint32_t ul = wl >> 8, uh = wh >> 8;
                const uint4 xv = *reinterpret_cast<const uint4*>(x_at + j * 64);
                mma_f16(d, jj == 0, wl & 0x000f000fu, wh & 0x000f000fu, wl & 0x00f000f0u, wh & 0x00f000f0u, xv.x, xv.y);
                mma_f16(d, false, ul & 0x000f000fu, uh & 0x000f000fu, ul & 0x00f000f0u, uh & 0x00f000f0u, xv.z, xv.w);
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
              const float2 sx = *reinterpret_cast<const float2*>(sum_at + (1 + grp) * COLS);
              tot[0] = fmaf(fmaf(d[0], fx.x, -z0 * sx.x), f0, tot[0]);
              tot[1] = fmaf(fmaf(d[1], fx.y, -z0 * sx.y), f0, tot[1]);
              tot[2] = fmaf(fmaf(d[2], fx.x, -z1 * sx.x), f1, tot[2]);
              tot[3] = fmaf(fmaf(d[3], fx.y, -z1 * sx.y), f1, tot[3]);
            }
            x_at += xstep;
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
        // sum r: row g + 8 (r / 2) of the tile, activation row 2 t + r % 2
        float* acc = s_acc + (n_tile + wic) * (p.rows * 16) + 2 * t * 16 + g;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float* dst = acc + (r & 1) * 16 + 8 * (r >> 1);
          if (2 * t + (r & 1) < rows) *dst = pass == 0 ? tot[r] : *dst + tot[r];
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
template <int GRP, bool ZEROS>
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
  if (cudaOccupancyMaxActiveClusters(&most, gemv4_kernel<GRP, ZEROS>, &cfg) != cudaSuccess || most < 1) {
    cudaGetLastError();
    return 2 * device_sms() / cs;
  }
  known[cs].store(most, std::memory_order_relaxed);
  return most;
}

template <int GRP, bool ZEROS>
int launch_t(Gemv4Dev& p, cudaStream_t s) {
  static std::atomic<uint64_t> configured{0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return POP_E_CUDA;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev >= 64 || !(configured.load(std::memory_order_relaxed) & bit)) {
    if (cudaFuncSetAttribute(gemv4_kernel<GRP, ZEROS>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_LIMIT) != cudaSuccess)
      return POP_E_CUDA;
    configured.fetch_or(bit, std::memory_order_relaxed);
  }
  // shared memory: activations with their sums, and sums of products
  constexpr int GPC = 128 / GRP, RING_BYTES = WARPS * RING * SLOT * (1024 + 32 * GPC + (ZEROS ? 16 * GPC : 0));
  constexpr int FIXED = RING_BYTES + 256 + (WARPS * RING + 2) * 8 + COLS * 64;
  static_assert(SMEM_LIMIT - FIXED >= (WARPS + 2) * COLS * 64 + 4 * COLS * (256 + 4 + 4 * GPC), "shared memory budget");
  p.rows = p.B < COLS ? p.B : COLS;
  const int slabs = ceil_div(p.B, COLS), room = SMEM_LIMIT - FIXED, acc_bytes = p.rows * 64, sc_bytes = p.rows * 256 + COLS * (4 + 4 * GPC);
  // Work of an SM with two CTAs, in clocks as measured: 30 to convert a row's chunk, 47 for a tile's chunk, the exchange within
  // a cluster. us in clusters of 1 / 2 / 8: 1 x 4096 -> 28672 gated 15.1 / 17.1 / 20.0, 1 x 14336 -> 4096 11.2 / 12.3 / 14.0.
  // A pass over part of the inputs, or a round over part of the tiles, costs 6000 more.
  const int each = p.mode == 3 ? 2 : 1, want = p.tiles / each;
  int64_t best = INT64_MAX;
  for (int cs = 1; cs <= 8 && cs <= p.kt; cs *= 2) {
    const int most = ceil_div(max_clusters<GRP, ZEROS>(cs), slabs), clusters = want < most ? want : most;
    // all chunks of a CTA at once if they fit beside the sums of two tiles, then as many tiles as fit
    const int dealt = ceil_div(want, clusters) * each, nc = ceil_div(p.kt, cs);
    const int passes = ceil_div(nc, (room - (WARPS + 2) * acc_bytes) / sc_bytes), sc = ceil_div(p.kt, passes * cs);
    const int rounds = ceil_div(dealt, ((room - sc * sc_bytes) / acc_bytes - WARPS) / 2 * 2);
    const int64_t cost = (int64_t)2 * nc * (p.rows * (p.xq ? 2 : 30) + (int64_t)p.tiles * 47 / clusters) +
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
  p.grain = p.sc % SLOT == 0 ? SLOT : 1;
  p.deal = p.tiles / each / p.clusters;
  p.deal_rest = p.tiles / each % p.clusters;
  p.sc_inv = (uint32_t)(((1ull << 32) + p.sc - 1) / p.sc);
  p.per_inv = (uint32_t)(((1ull << 32) + p.rows * 16 - 1) / (p.rows * 16));
  const size_t smem = FIXED + (size_t)p.sc * sc_bytes + (size_t)(p.tpr + WARPS) * acc_bytes;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  ProfScope prof(PROF_GEMV, (double)p.N * p.K * (0.5 + (p.zeros ? 3.0 : 2.0) / GRP) * slabs, s);
  if (launch_chained_cluster_x(gemv4_kernel<GRP, ZEROS>, dim3(p.clusters * p.cs, slabs), dim3(WARPS * 32), smem, s,
                               (unsigned)p.cs, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

// Whether each CTA converts the activations that it needs, 8 rows at a time, and no launch of its own does it before. us so / by a
// launch: 3 x 2048 -> 4096 4.5 / 5.1, 8 x 1024 -> 4096 4.6 / 4.6, 8 x 2048 -> 4096 6.3 / 5.5, and beyond 8 rows, where weights are
// read again for each 8 and the other products begin, 16 x 1024 -> 4096 5.0 / 6.0, 64 x 512 -> 512 3.9 / 6.5, 32 x 1024 -> 4096 5.9 /
// 6.4, 32 x 2048 -> 4096 9.2 / 7.7, 16 x 2048 -> 4096 7.1 / 6.9. A call of two launches takes 4 us more of the host.
bool converts_itself(int B, int N, int K) {
  if (B < 3) return true;
  if (B <= COLS) return (int64_t)B * ceil_div(K, 128) <= 64;
  return (int64_t)ceil_div(B, COLS) * N * K < (1 << 24);
}

template <int GRP>
int launch_grp(const Gemv4Args& a, Gemv4Dev& p, cudaStream_t s) {
  void* workspace = a.workspace;
  const size_t bytes = a.workspace_bytes;
  const bool own = converts_itself(p.B, p.N, p.K);
  if (p.B > 65535) return POP_E_INVALID;
  if (!own) {
    const int cols = cols_of(p.B), slabs = ceil_div(p.B, cols), kt = (int)slab_chunks(cols, p.kt);
    if (!workspace || (int64_t)bytes < slabs * slab_bytes(cols, 128 / GRP, kt)) return POP_E_NOSPACE;
    p.xq = static_cast<uint8_t*>(workspace);
    ProfScope prof(PROF_ELEMENTWISE, (double)p.B * p.K * 4, s);
    if (launch_chained(gemv4_convert_kernel<GRP>, dim3(ceil_div(kt, 16), p.B), dim3(256), 0, s, p.x, p.ldx,
                       static_cast<uint8_t*>(workspace), p.B, p.K, kt, cols, p.zeros ? 1 : 0) != cudaSuccess)
      return POP_E_CUDA;
    count_launch();
  }
  if (p.B > COLS && !own) return launch_gemm4(a, p.xq, s);        // at 8 rows the other one is slower: 4096 -> 28672 gated 34 us to 20
  return p.zeros ? launch_t<GRP, true>(p, s) : launch_t<GRP, false>(p, s);
}

}  // namespace

size_t gemv4_workspace_bytes(int B, int N, int K, int group) {
  if (B < 1 || N < 1 || K < 1 || converts_itself(B, N, K) || (group != 32 && group != 64 && group != 128)) return 0;
  return (size_t)(ceil_div(B, cols_of(B)) * slab_bytes(cols_of(B), 128 / group, slab_chunks(cols_of(B), ceil_div(K, 128))));
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
    case 32: return launch_grp<32>(a, p, s);
    case 64: return launch_grp<64>(a, p, s);
    default: return launch_grp<128>(a, p, s);
  }
}

}  // namespace pop
