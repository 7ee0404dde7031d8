// Projections of few rows with 4-bit weights (the decode stage of paper Sec. 3.2 at full depth; narrow weights for that
// stage alone are the stage-aware quantisation that Sec. 6 names as a direction):
//   out[b][n] = sum_k x[b][k] (code[n][k] - zero[n][k / group]) scale[n][k / group]
#include "common.cuh"
#include "heads.cuh"
#include "w4.cuh"

#include <atomic>

namespace pop {
namespace {

__device__ __forceinline__ uint4 ld_codes(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// D = A B + (first ? 0 : D), m16n8k16
__device__ __forceinline__ void mma_w4(float (&d)[4], bool first, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                       uint32_t b0, uint32_t b1) {
  if (first)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Codes i and i + 4 of a word's nibbles (inputs 2 i and 2 i + 1) minus the zero, as packed bf16: a code in the low bits of
// the fraction of 128 is 128 + code; minus (128 + zero) is exact. off: -(128 + zero) in both halves.
__device__ __forceinline__ uint32_t pair_of(uint32_t w, int i, uint32_t off) {
  uint32_t v = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u, r;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(off));
  return r;
}
__device__ __forceinline__ float act_of(float g, int act) {
  if (act == 0) return g / (1.0f + expf(-g));
  return 0.5f * g * (1.0f + tanhf(0.7978845608028654f * (g + 0.044715f * g * g * g)));
}

struct Gemv4Dev {
  const bf16* x; int64_t ldx;
  const uint8_t* codes; const bf16* scales; const uint8_t* zeros;
  void* out; int64_t ldo;
  int B, N, K, mode, act, n_valid;
  int kt;                       // chunks of 128 inputs
  int blocks;                   // row blocks: MT tiles of 16 rows, gated: a gate tile and its up tile
  int ks_log;                   // 2^ks_log warps of a CTA share a row block and take its chunks in turn
};

// The weight rows are the M side of the warp-level MMA, the activation rows its N side. A tile of 16 rows x 128 inputs is
// 1 KB in one piece, 16 bytes of row g and 16 of row g + 8 to lane (g = lane / 4, t = lane % 4): word j of them are inputs
// 32 j + 8 t .. + 7, which are also 16 bytes of activation row g, so that one 16-byte load of activations feeds two MMAs and
// all inputs of an MMA are of one group. Operands are exact (codes minus zero are small integers), a group's sum is built
// from zero in the MMA's fp32 accumulator and enters the row's fp32 sum with its scale.
// U chunks are a batch of loads; two batches are in flight, across the ends of row blocks too.
template <int GRP, int MT, int NT, bool GATED>
__global__ void __launch_bounds__(256, 2) gemv4_kernel(const Gemv4Dev p) {
  constexpr int GPC = 128 / GRP;                    // groups of a chunk
  constexpr int U = (GPC == 4 || NT > 1 ? 2 : 4) / MT;
  constexpr int NR = MT * NT * 4;                   // sums of a lane
  __shared__ float part[8][NR][32];
  const int lane = threadIdx.x & 31, wic = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int ks = 1 << p.ks_log, slice = wic & (ks - 1), gpc = 8 >> p.ks_log;
  const int row0 = blockIdx.y * (NT * 8);
  const int n_rounds = (p.blocks + gpc - 1) / gpc;
  const int my_rounds = n_rounds > (int)blockIdx.x ? (n_rounds - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;
  const int nb_round = ((p.kt + ks - 1) / ks + U - 1) / U;
  const int n_batches = my_rounds * nb_round;
  chain_trigger();

  struct Batch {
    uint4 lo[U][MT], hi[U][MT];
    uint32_t sc[U][MT][GPC];                        // scales of row g, then of row g + 8
    uint32_t zr[U][MT][2];                          // their zeros, a byte each
  };
  Batch buf[2];
  auto block_of = [&](int round) { return ((int)blockIdx.x + round * (int)gridDim.x) * gpc + (wic >> p.ks_log); };
  // Tile numbers of a row block; past the end they repeat the last block (loaded, never stored)
  auto tile_of = [&](int block, int m) {
    block = min(block, p.blocks - 1);
    if (GATED) return (block >> 3) * 16 + (block & 7) + 8 * m;
    return min(block * MT + m, (p.N + 15) / 16 - 1);
  };
  int l_round = 0, l_batch = 0;
  int64_t at[MT];                                   // chunk numbers of the tiles' first chunks
  auto set_rows = [&](int round) {
#pragma unroll
    for (int m = 0; m < MT; ++m) at[m] = (int64_t)tile_of(block_of(round), m) * p.kt;
  };
  if (my_rounds > 0) set_rows(0);
  auto load_next = [&](Batch& q) {
    if (l_round >= my_rounds) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = slice + ((l_batch * U + u) << p.ks_log);
      if (c < p.kt) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int64_t chunk = at[m] + c;
          const uint8_t* src = p.codes + chunk * 1024 + lane * 16;
          q.lo[u][m] = ld_codes(src);
          q.hi[u][m] = ld_codes(src + 512);
          const int64_t sg = (chunk * 8 + g) * (2 * GPC);
          if constexpr (GPC == 1) {
            q.sc[u][m][0] = __ldg(reinterpret_cast<const uint32_t*>(p.scales + sg));
          } else if constexpr (GPC == 2) {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p.scales + sg));
            q.sc[u][m][0] = v.x; q.sc[u][m][1] = v.y;
          } else {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p.scales + sg));
            q.sc[u][m][0] = v.x; q.sc[u][m][1] = v.y; q.sc[u][m][2] = v.z; q.sc[u][m][3] = v.w;
          }
          if (p.zeros != nullptr) {
            if constexpr (GPC == 1) {
              q.zr[u][m][0] = __ldg(reinterpret_cast<const uint16_t*>(p.zeros + sg));
            } else if constexpr (GPC == 2) {
              q.zr[u][m][0] = __ldg(reinterpret_cast<const uint32_t*>(p.zeros + sg));
            } else {
              const uint2 v = __ldg(reinterpret_cast<const uint2*>(p.zeros + sg));
              q.zr[u][m][0] = v.x; q.zr[u][m][1] = v.y;
            }
          } else {
            q.zr[u][m][0] = q.zr[u][m][1] = 0x08080808u;
          }
        }
      }
    }
    if (++l_batch == nb_round) {
      l_batch = 0;
      if (++l_round < my_rounds) set_rows(l_round);
    }
  };
  // the first weights go out before the wait on the preceding kernel: no kernel of the library writes them
  load_next(buf[0]);
  load_next(buf[1]);
  chain_wait();

  const bf16* xr[NT];
  bool has[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    has[n] = row0 + n * 8 + g < p.B;
    xr[n] = p.x + (int64_t)(has[n] ? row0 + n * 8 + g : 0) * p.ldx + t * 8;
  }
  float tot[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) tot[m][n][i] = 0.f;

  int batch = 0, round = 0;
  auto step = [&](Batch& q) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = slice + ((batch * U + u) << p.ks_log);
      if (c < p.kt) {
        float d[MT][NT][4];
        uint32_t off[MT][2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          constexpr int JPG = 4 / GPC;              // words of a group
          const int k = c * 128 + j * 32 + t * 8, grp = j / JPG;
          uint4 xv[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n)
            xv[n] = has[n] && k < p.K ? __ldg(reinterpret_cast<const uint4*>(xr[n] + c * 128 + j * 32)) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (j % JPG == 0) {
              // byte h * GPC + grp: the zero of row g + 8 h
              const uint32_t z0 = q.zr[u][m][0] >> (8 * grp), z1 = GPC == 4 ? q.zr[u][m][1] >> (8 * grp) : q.zr[u][m][0] >> (8 * (GPC + grp));
              off[m][0] = 0xc300c300u | ((z0 & 0x7fu) * 0x10001u);
              off[m][1] = 0xc300c300u | ((z1 & 0x7fu) * 0x10001u);
            }
            const uint4 lo = q.lo[u][m], hi = q.hi[u][m];
            const uint32_t wl = j == 0 ? lo.x : j == 1 ? lo.y : j == 2 ? lo.z : lo.w;
            const uint32_t wh = j == 0 ? hi.x : j == 1 ? hi.y : j == 2 ? hi.z : hi.w;
            uint32_t a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              a[i] = pair_of(wl, i, off[m][0]);
              b[i] = pair_of(wh, i, off[m][1]);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_w4(d[m][n], j % JPG == 0, a[0], b[0], a[1], b[1], xv[n].x, xv[n].y);
              mma_w4(d[m][n], false, a[2], b[2], a[3], b[3], xv[n].z, xv[n].w);
            }
            if (j % JPG == JPG - 1) {
              // scales lie as [row half][group]: halves of words. What lies behind K is never used.
              const int i0 = grp, i1 = GPC + grp;
              const uint32_t s0 = q.sc[u][m][i0 / 2], s1 = q.sc[u][m][i1 / 2];
              const bool in = c * 128 + grp * GRP < p.K;
              const float f0 = in ? __uint_as_float(i0 & 1 ? s0 & 0xffff0000u : s0 << 16) : 0.f;
              const float f1 = in ? __uint_as_float(i1 & 1 ? s1 & 0xffff0000u : s1 << 16) : 0.f;
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                tot[m][n][0] = fmaf(d[m][n][0], f0, tot[m][n][0]);
                tot[m][n][1] = fmaf(d[m][n][1], f0, tot[m][n][1]);
                tot[m][n][2] = fmaf(d[m][n][2], f1, tot[m][n][2]);
                tot[m][n][3] = fmaf(d[m][n][3], f1, tot[m][n][3]);
              }
            }
          }
        }
      }
    }
    load_next(q);
    if (++batch < nb_round) return;
    // ---- end of a row block: the slices' sums meet in shared memory in slice order, each warp finishing a part of them
    batch = 0;
    const int block = block_of(round++);
    if (ks > 1) {
      __syncthreads();                               // the previous block's sums have been read
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) part[wic][(m * NT + n) * 4 + i][lane] = tot[m][n][i];
      __syncthreads();
    }
    const int first = wic & ~(ks - 1);
    auto sum_of = [&](int r) {
      float v = 0.f;
      for (int sl = 0; sl < ks; ++sl) v += part[first + sl][r][lane];
      return v;
    };
    // sum i of n-tile n: row g + 8 (i / 2) of the tile, activation row 2 t + i % 2
#pragma unroll
    for (int r = 0; r < NT * 4; ++r) {
      if (ks == 1 || (r & (ks - 1)) == slice) {
        const int n = r >> 2, i = r & 3, b = row0 + n * 8 + 2 * t + (i & 1);
        if (GATED) {
          const float gate = ks > 1 ? sum_of(r) : tot[0][n][i], up = ks > 1 ? sum_of((MT - 1) * NT * 4 + r) : tot[MT - 1][n][i];
          const int o = (block >> 3) * 128 + (block & 7) * 16 + g + 8 * (i >> 1);
          if (block < p.blocks && b < p.B && o < p.n_valid)
            static_cast<bf16*>(p.out)[(int64_t)b * p.ldo + o] = __float2bfloat16_rn(act_of(gate, p.act) * up);
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const float v = ks > 1 ? sum_of(m * NT * 4 + r) : tot[m][n][i];
            const int o = (block * MT + m) * 16 + g + 8 * (i >> 1);
            if (block < p.blocks && b < p.B && o < p.N) {
              float* dst = static_cast<float*>(p.out) + (int64_t)b * p.ldo + o;
              *dst = p.mode == 0 ? v : *dst + v;
            }
          }
        }
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) tot[m][n][i] = 0.f;
  };
  for (int fb = 0; fb < n_batches; fb += 2) {
    step(buf[0]);
    if (fb + 1 < n_batches) step(buf[1]);
  }
}

template <int GRP, int MT, int NT, bool GATED>
int launch_t(Gemv4Dev& p, cudaStream_t s) {
  const int tiles = (p.N + 15) / 16;
  p.blocks = GATED ? tiles / 2 : (tiles + MT - 1) / MT;
  // warps: as many slices per row block as give every SM its 16 warps, each slice at least one chunk
  const int sms = device_sms();
  int ks = 0;
  while (ks < 3 && ((int64_t)p.blocks << ks) < (int64_t)sms * 16 && (2 << ks) <= p.kt) ++ks;
  p.ks_log = ks;
  const int rounds = ceil_div(p.blocks, 8 >> ks);
  const int grid = rounds < 2 * sms ? rounds : 2 * sms;
  const int slabs = ceil_div(p.B, NT * 8);
  if (slabs > 65535) return POP_E_INVALID;
  ProfScope prof(PROF_GEMV, (double)p.N * p.K * (0.5 + (p.zeros ? 3.0 : 2.0) / GRP) * slabs, s);
  if (launch_chained(gemv4_kernel<GRP, MT, NT, GATED>, dim3(grid, slabs), dim3(256), 0, s, p) != cudaSuccess) return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

template <int GRP>
int launch_grp(Gemv4Dev& p, cudaStream_t s) {
  const bool gated = p.mode == 3;
  if (p.B <= 8) {
    if (gated) return launch_t<GRP, 2, 1, true>(p, s);
    return launch_t<GRP, 1, 1, false>(p, s);
  }
  if (p.B <= 16) return gated ? launch_t<GRP, 2, 2, true>(p, s) : launch_t<GRP, 2, 2, false>(p, s);
  return gated ? launch_t<GRP, 2, 4, true>(p, s) : launch_t<GRP, 2, 4, false>(p, s);
}

}  // namespace

int launch_gemv4(const Gemv4Args& a, cudaStream_t s) {
  if (!a.x || !a.codes || !a.scales || !a.out || a.B < 1 || a.N < 1 || a.K < 8 || a.K % 8) return POP_E_INVALID;
  if (a.mode != 0 && a.mode != 2 && a.mode != 3) return POP_E_INVALID;
  if (a.group != 32 && a.group != 64 && a.group != 128) return POP_E_INVALID;
  if (a.mode == 3 && (a.N % 256 || a.n_valid < 0 || a.n_valid > a.N / 2 || (a.act != 0 && a.act != 1))) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.x) % 16 || a.ldx % 8 || reinterpret_cast<uintptr_t>(a.codes) % 16 ||
      reinterpret_cast<uintptr_t>(a.scales) % 16 || reinterpret_cast<uintptr_t>(a.zeros) % 8 ||
      reinterpret_cast<uintptr_t>(a.out) % (a.mode == 3 ? 2 : 4))
    return POP_E_INVALID;
  if (a.N > (1 << 30) || a.K > (1 << 30)) return POP_E_INVALID;
  if (a.B > 1 && (a.ldx < a.K || a.ldo < (a.mode == 3 ? a.n_valid : a.N))) return POP_E_INVALID;     // rows over each other
  Gemv4Dev p{};
  p.x = a.x; p.ldx = a.ldx;
  p.codes = a.codes; p.scales = a.scales; p.zeros = a.zeros;
  p.out = a.out; p.ldo = a.ldo;
  p.B = a.B; p.N = a.N; p.K = a.K; p.mode = a.mode; p.act = a.act; p.n_valid = a.n_valid;
  p.kt = ceil_div(a.K, 128);
  switch (a.group) {
    case 32: return launch_grp<32>(p, s);
    case 64: return launch_grp<64>(p, s);
    default: return launch_grp<128>(p, s);
  }
}

}  // namespace pop
