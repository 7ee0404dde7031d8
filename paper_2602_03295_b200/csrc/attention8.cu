// Causal attention of many query rows over the 8-bit paged cache (paper Eq. 1, Attn(x_l, K, V)), with an optional
// sliding window: the prompt, a chunk of one, or a few drafted tokens behind a long cache.
//
// The last rows of a sequence are the queries: row i of n at position len - n + i sees positions j <= its own (and
// j > it - window). With codes k_j, v_j, block exponents ek, ev and c = log2(e) / sqrt(hd):
//   w_j = exp2(c q.k_j 2^(ek) + ev - m),  out = sum_j w_j v_j / sum_j w_j 2^(-ev)
// (m the running maximum of the exponent without -m): the block scales never touch the tensor cores' operands, which are
// the K codes as they are, the query as two codes an element, the V codes as f16 (exact) and the weights as f16 (half a
// step: 2^-11 relative). Scores, statistics, sums and the accumulator are fp32.
//
// A CTA owns NQT tiles of 128 rows of one kv head; a row is a (position, query head) pair of that kv head, so that the
// keys are read once for all heads that share them, however few the positions are. K codes are E4M3 operands as they
// lie in the cache (tcgen05 kind::f8f6f4): after a power-of-two scale per row an element of q is the sum of two codes (exactly
// for bf16 elements down to 2^-9 of the row's largest, within 2^-17 of that below), two instruction sets at twice the f16
// rate accumulate both. V has to become f16 (exact) because the weights are f16. Warp roles:
//   NQT softmax warpgroups, one row per thread: place both codes of Q in shared memory, then read S = Q K^T from TMEM 64
//       keys at a time, write the weights over it, rescale the TMEM accumulator when the maximum grew by more than 2^8;
//   a converter warpgroup: 64 keys of V at a time from the staged codes to f16 in the 128-byte-swizzled operand layout;
//       positions past the end, or in front of every row's window, become zeros;
//   a TMA warp: codes of K (128 keys) and V (64 keys) from the paged pools, a row being one position of one head;
//   an MMA warp per tile: scores, then O += P V per 64 keys with P from TMEM. Two score buffers per tile, so that the next
//       scores are there before the softmax is done with the last: 64 keys each for two tiles, 128 for one (a set of 128
//       keys shares the reads of Q, 64 against 48 clocks an instruction, but with two tiles TMEM has room for one such set
//       per tile: 573 us for an 8192-token prompt, 556 with two of 64). One warp for both tiles spent 2190 clocks per 64
//       keys, 1560 of them issuing (54 per instruction), and made the softmax wait for scores;
//   a scale warp: the scales of 32 blocks at a time, converted, in a small ring.
// Where few CTAs would leave SMs idle or wait for the longest sequence, the keys are split over several CTAs, which leave
// unnormalised rows in the workspace for a second, chained launch to merge (512 rows each of three sequences of up to
// 16384, which are 192 CTAs of unequal length: 290 us in one piece, 242 us in two).
//
// Measured in captured graphs, causal, 32 heads over 8, hd 128: 8192 rows of 8192 550 us, 1000 TFLOP/s (0.60 of a bf16 GEMM's;
// 603 us after a second of calls, when the power cap has brought the clock from 1965 to 1777 MHz; hd 64 509 us); hd 256,
// 16 over 8, window 1024: 8192 rows 190 us; 512 rows each of three sequences of up to 16384 242 us (hd 64 224). Bound by
// the softmax warps' dependent steps: 1980 clocks per 64 keys, of which the exponential unit works 1024 (two warps of a
// scheduler) and the tensor pipe 1280; halving the exponentials (a copy, to see) took 14 % off, leaving out the row maximum
// 3 %, the V conversion nothing. A CTA's start takes 13000 clocks and its end 4500, of 145000 (hd 256 with the window: of 50000). Tried and slower:
// one CTA per SM that walks equal shares of all tiles (898 us; the segments' starts and the live state cost more than the
// balance gave), the next tile's scores or scales asked for before this one's weights are stored (551 to 569 against 556),
// query rows by bulk copies (570).
#include "../../include/pop_kernels.h"
#include "cache8.cuh"
#include "ptx.cuh"

namespace pop {
namespace {

constexpr int kSmemLimit = 227 * 1024;
// Up to this many (row, head) pairs of a kv head go to decode8.cu, which reads the keys once per eight of them; here they are
// rows of a tile of 128. Both measured, hd 128, 32 heads over 8: 12 sequences of up to 8000 positions 16 pairs 34 against 94
// us, 32 44 / 94, 64 68 / 95, 96 97 / 95; one of 8192 16 16.4 / 25, 32 16.5 / 25, 48 26 / 25, 64 30 / 25; 40 of up to 500 16
// 21 / 31, 32 36 / 31, 64 65 / 31.
constexpr int FEW_COLUMNS = 32;
constexpr float W_SHIFT = 7.f;        // weights are stored times 2^7; the lazy maximum lets them reach 2^15

template <int HD, int NQT>
struct A8 {
  static constexpr int BKV = 64, PKV = 128;
  static constexpr int INNER = HD < 128 ? HD : 128;            // bytes of a code row in one swizzled slice
  static constexpr int SLICES = HD / INNER;
  static constexpr int Q_PART = 128 * HD;                      // one code per element; two parts per tile
  static constexpr int K_STAGE = PKV * HD;
  static constexpr int VR_STAGE = BKV * HD;                    // V codes
  static constexpr int VF_STAGE = BKV * HD * 2;                // V as f16
  static constexpr int VF_SUB = BKV * 128;                     // one 64-wide slice of it
  static constexpr int NK = HD == 256 ? 2 : 3;
  static constexpr int NVR = HD == 256 ? 2 : 4;
  static constexpr int NVF = HD == 256 ? 2 : 4;
  static constexpr int SK = NQT == 1 ? 128 : 64;               // keys of a set of scores: two buffers of them per tile
  static constexpr int HPS = SK / BKV, SPP = PKV / SK;         // 64-key tiles per set, sets per pair of tiles
  static constexpr int SM_WARPS = NQT * 4;
  static constexpr int THREADS = (SM_WARPS + 8) * 32;
  static constexpr int LOADS = BKV * HD / (16 * 128);          // 16-byte pieces of a V stage per converter thread
  static constexpr int O_COL = 256;                            // S at (t + buffer) * 128, O_t at O_COL + t * HD
  static constexpr uint32_t TMEM_COLS = 512;
  static_assert(O_COL + NQT * HD <= 512, "TMEM budget");
};

template <int HD, int NQT>
struct __align__(1024) A8Smem {
  using C = A8<HD, NQT>;
  uint8_t q[NQT][2][C::Q_PART];
  uint8_t k[C::NK][C::K_STAGE];
  uint8_t vr[C::NVR][C::VR_STAGE];
  uint8_t vf[C::NVF][C::VF_STAGE];
  float4 sc[2][32];             // per block of 16 keys: 2^ek, ev, 2^-ev; two groups of 32 blocks
  float crow[NQT * 128];        // factor of each row's scores
  uint64_t k_full[C::NK], k_empty[C::NK];
  uint64_t vr_full[C::NVR], vr_empty[C::NVR];
  uint64_t vf_full[C::NVF], vf_empty[C::NVF];
  uint64_t sc_full[2], sc_empty[2];
  uint64_t s_full[NQT][2];      // a set of scores complete; index: tile, buffer
  uint64_t p_ready[NQT][2][C::HPS];  // P of 64 keys written over their scores (one arrival per softmax warp)
  uint64_t pv_done[NQT][2][C::HPS];  // O += P V of 64 keys complete
  uint32_t tmem_base;
  uint32_t raised;
  volatile uint32_t abort;
};

struct A8Dev {
  const bf16* q; int64_t ldq;
  Cache8 c;
  int box;                      // rows of one copy: min(page size, 64)
  int pool_rows;                // rows of the pool: pages * n_kv * page size
  const int32_t* cu; int rows;
  const int32_t* seq_lens; int kv_len;
  bf16* out; int64_t ldo;
  bool out32;                   // output rows on 32-byte boundaries
  int n_q, n_kv, G, hg;         // query heads per kv head; head groups of at most 128 per kv head
  int window;
  int per;                      // positions per tile (one head group)
  uint32_t inv;                 // 2^16 / G, rounded up
  int q_tiles;                  // CTAs along the rows of the longest sequence
  int splits, chunk;            // pieces of a tile's keys, each of at most chunk 64-key tiles
  float* partial;               // [CTA][NQT * 128][hd + 4]: m, l, two unused, accumulator
  float scale_log2;
};

// The rows and keys of one CTA (without the split)
struct Job {
  int b, kvh, h0, heads, per;   // heads of this group; positions per tile
  uint32_t inv;                 // 2^16 / heads, rounded up: r / heads = r * inv >> 16 for r < 256
  int row0, n, q0;              // first packed row of the sequence, its rows, first row of the CTA (< 0: none)
  int len, pos0;                // cached positions; position of row q0
  int lo, j_lo, n_tiles;        // first key that its rows see; 64-key tiles that they see
};
template <int NQT>
__device__ __forceinline__ Job job_of(const A8Dev& p, int bx, int by, int b, int* status) {
  Job x;
  x.b = b;
  // the lengths' loads first: all of them are in flight together
  const int c0 = p.cu ? p.cu[b] : b * p.rows, c1 = p.cu ? p.cu[b + 1] : c0 + p.rows;
  x.len = p.seq_lens ? p.seq_lens[b] : p.kv_len;
  if (p.hg == 1) {
    x.kvh = bx;
    x.h0 = bx * p.G;
    x.heads = p.G;
    x.per = p.per;
    x.inv = p.inv;
  } else {
    x.kvh = bx / p.hg;
    const int grp = bx - x.kvh * p.hg;
    x.h0 = x.kvh * p.G + grp * 128;
    x.heads = min(128, p.G - grp * 128);
    x.per = 128 / x.heads;
    x.inv = (65536 + x.heads - 1) / x.heads;
  }
  x.row0 = c0;
  x.n = c1 - c0;
  if (x.len > p.kv_len || x.n > p.rows) {       // more than the caller said: nothing past it is touched
    atomicMin(status, (int)POP_E_INVALID);
    x.n = min(x.n, p.rows);
    x.len = min(x.len, p.kv_len);
  }
  x.len = max(x.len, 0);
  // latest rows first
  const int step = NQT * x.per, tile = (x.n > 0 ? (x.n - 1) / step : -1) - by;
  x.q0 = tile * step;
  x.pos0 = x.len - x.n + x.q0;
  const int last = min(x.pos0 + step - 1, x.len - 1);
  x.lo = p.window > 0 ? max(0, max(0, x.pos0) - p.window + 1) : 0;
  x.j_lo = x.lo / 64;
  x.n_tiles = last < 0 || tile < 0 ? 0 : last / 64 - x.j_lo + 1;
  return x;
}
// Pieces that the CTA's keys are cut into: at least one, and no more than there are CTAs and rows of the workspace for
__device__ __forceinline__ int pieces_of(const A8Dev& p, const Job& x) {
  return min(max(1, (x.n_tiles + p.chunk - 1) / p.chunk), p.splits);
}
__device__ __forceinline__ int row_pos(const Job& x, int r) { return (int)(r * x.inv >> 16); }     // r / heads

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_b2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Instruction descriptor for kind::f16 with f16 A and B (format 0 in both fields); see umma_idesc_bf16
__host__ __device__ constexpr uint32_t umma_idesc_f16(int m, int n, int b_mn_major) {
  return (1u << 4) | (uint32_t(b_mn_major) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}

// the lowest status wins, so a wait that ran out stays to be seen beside wrong arguments
__device__ __forceinline__ bool gave_up(int status) { return status <= (int)POP_E_DEVICE_TIMEOUT; }

#define A8_ABORT(S, status)                           \
  do {                                                \
    (S).abort = 1;                                    \
    atomicMin((status), (int)POP_E_DEVICE_TIMEOUT);   \
  } while (0)

// Shared-memory matrix descriptor of a K-major tile of codes: rows of 128 bytes with 128-byte swizzle, or (hd 64) rows of
// 64 bytes with 64-byte swizzle (layout 4); groups of 8 rows follow each other
template <int INNER>
__device__ __forceinline__ uint64_t code_desc(uint32_t saddr) {
  uint64_t d = umma_smem_desc(saddr, 16, INNER * 8);
  if (INNER == 64) d = (d & ~(uint64_t(7) << 61)) | (uint64_t(4) << 61);
  return d;
}
// where 16-byte piece c of a code row lies in its slice
template <int INNER>
__device__ __forceinline__ int code_at(int row, int c) {
  return INNER == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <int HD, int NQT>
__global__ void __launch_bounds__(A8<HD, NQT>::THREADS, 1)
attn8_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
             const __grid_constant__ A8Dev p, int* __restrict__ status) {
  using C = A8<HD, NQT>;
  constexpr int BKV = C::BKV, PKV = C::PKV, INNER = C::INNER, SLICES = C::SLICES;
  constexpr int SK = C::SK, HPS = C::HPS, SPP = C::SPP;
  extern __shared__ uint8_t smem_raw[];
  A8Smem<HD, NQT>& s =
      *reinterpret_cast<A8Smem<HD, NQT>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  chain_trigger();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);      // known to be the same in the warp: uniform registers
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == (C::SM_WARPS + 4) * 32) {           // the TMA warp's first lane: it uses them before the others do
    for (int i = 0; i < C::NK; ++i) { mbar_init(&s.k_full[i], 1); mbar_init(&s.k_empty[i], NQT); }
    for (int i = 0; i < C::NVR; ++i) { mbar_init(&s.vr_full[i], 1); mbar_init(&s.vr_empty[i], 4); }
    for (int i = 0; i < C::NVF; ++i) { mbar_init(&s.vf_full[i], 4); mbar_init(&s.vf_empty[i], NQT); }
    for (int i = 0; i < 2; ++i) { mbar_init(&s.sc_full[i], 1); mbar_init(&s.sc_empty[i], C::SM_WARPS); }
    for (int t = 0; t < NQT; ++t)
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s.s_full[t][i], 1);
        for (int h = 0; h < C::HPS; ++h) { mbar_init(&s.p_ready[t][i][h], 4); mbar_init(&s.pv_done[t][i][h], 1); }
      }
    s.abort = 0;
    fence_barrier_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  chain_wait();
  // the status word is on its way while the lengths are (read by the TMA warp alone). Only a kernel that gave up on a wait
  // stops this one: a wrong place of another call, or of another sequence of this one, does not touch these rows
  int raised = 0;
  if (warp == C::SM_WARPS + 4) raised = *reinterpret_cast<const volatile int*>(status);
  int split = 0, b = blockIdx.z;
  if (p.splits > 1) {
    b = blockIdx.z / p.splits;
    split = blockIdx.z - b * p.splits;
  }
  const Job x = job_of<NQT>(p, blockIdx.x, blockIdx.y, b, status);
  if (x.q0 < 0) return;                                  // past the rows of this sequence
  int t_lo = 0, n_tiles = x.n_tiles;                     // 64 keys each
  float* part = nullptr;
  if (p.splits > 1) {
    const int pieces = pieces_of(p, x);
    if (split >= pieces) return;                         // fewer keys than the longest sequence's
    const int each = x.n_tiles / pieces, more = x.n_tiles - each * pieces;      // the first `more` have one tile more
    t_lo = split * each + min(split, more);
    n_tiles = each + (split < more ? 1 : 0);
    if (pieces > 1)                                      // a tile of one piece is written at once
      part = p.partial + (((int64_t)(blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * (NQT * 128)) * (HD + 4);
  }
  const int n_pairs = (n_tiles + 1) >> 1;
  const int key0 = (x.j_lo + t_lo) * BKV;                // first key of tile 0

  if (n_tiles <= 0) {                                    // rows that see nothing: zeros
    for (int r = threadIdx.x; r < NQT * 128; r += blockDim.x) {
      const int in_tile = r & 127, ip = row_pos(x, in_tile), i = x.q0 + (r >> 7) * x.per + ip;
      if (in_tile >= x.per * x.heads || i >= x.n) continue;
      uint4* dst = reinterpret_cast<uint4*>(p.out + ((int64_t)x.row0 + i) * p.ldo +
                                            (int64_t)(x.h0 + in_tile - ip * x.heads) * HD);
      for (int c = 0; c < HD / 8; ++c) dst[c] = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;
  const int ps = p.c.page_size;
  // pool row (page * n_kv + head) * page_size + slot of a position, or -1 for a table entry that is no page of the pool
  auto pool_row = [&](int pos) {
    const int pi = pos / ps, page = bt[pi];
    if ((unsigned)page >= (unsigned)p.c.num_pages) {
      atomicMin(status, (int)POP_E_INVALID);
      return -1;
    }
    return (page * p.n_kv + x.kvh) * ps + (pos - pi * ps);
  };


  // TMA: lane l holds the pool row of copy l of a pair (128 keys), fetched a pair ahead. A copy that starts past the end, or
  // ends in front of the window (its page may belong to another sequence by now), is left out; one of a bad page goes past the
  // pool's end and is filled with zeros.
  const int boxes = PKV / p.box, half_boxes = boxes >> 1;
  auto row_of = [&](int J) {
    const int pos = key0 + J * PKV + lane * p.box;
    if (lane >= boxes || J >= n_pairs || pos >= x.len || pos + p.box <= x.lo) return -2;
    const int r = pool_row(pos);
    return r < 0 ? p.pool_rows : r;
  };
  auto copy = [&](const CUtensorMap* tm, uint64_t* bar, uint8_t* dst, int row, int first, int count) {
    const int live = __popc(__ballot_sync(0xffffffffu, row != -2) & (((1u << count) - 1u) << first));
    if (lane == 0) mbar_expect_tx(bar, live * p.box * HD);
    for (int i = 0; i < count; ++i) {
      const int r = __shfl_sync(0xffffffffu, row, first + i);
      if (r != -2 && lane == 0)
        for (int c = 0; c < SLICES; ++c)
          tma_load_2d(dst + c * (count * p.box * INNER) + i * p.box * INNER, tm, bar, c * INNER, r);
    }
  };
  auto load_pair = [&](int J, int row) {
    const int ks = J % C::NK;
    if (!mbar_wait_relaxed(&s.k_empty[ks], ((J / C::NK) & 1) ^ 1)) return false;
    __syncwarp();
    copy(&tmK, &s.k_full[ks], s.k[ks], row, 0, boxes);
    for (int h = 0; h < 2; ++h) {
      const int jj = 2 * J + h, vs = jj % C::NVR;
      if (jj >= n_tiles) break;
      if (!mbar_wait_relaxed(&s.vr_empty[vs], ((jj / C::NVR) & 1) ^ 1)) return false;
      __syncwarp();
      copy(&tmV, &s.vr_full[vs], s.vr[vs], row, h * half_boxes, half_boxes);
    }
    return true;
  };

  // Start: the TMA warp asks for the first pair, the MMA warp for TMEM, the others place the query rows in shared memory:
  // each row scaled so that its largest element is in [2^7, 2^8), as the nearest codes and the nearest codes of what is
  // left. hd / 8 lanes take a row, 16 bytes each, several rows at once.
  int tma_row = -2;
  if (warp == C::SM_WARPS + 4) {
    raised = __shfl_sync(0xffffffffu, raised, 0);
    raised = gave_up(raised) ? 1 : 0;
    if (lane == 0) s.raised = (uint32_t)raised;
    if (raised == 0) {
      tma_row = row_of(0);
      load_pair(0, tma_row);                               // the ring is empty: nothing is waited for
      tma_row = row_of(1);
    }
  } else if (warp == C::SM_WARPS + 5) {
    tmem_alloc(&s.tmem_base, C::TMEM_COLS);
    tmem_relinquish();
  } else if (warp < C::SM_WARPS + 4) {
    constexpr int LPR = HD / 32, RPI = 32 / LPR, WARPS = C::SM_WARPS + 4;     // lanes per row, rows at a time
    constexpr int GROUPS = NQT * 128 / RPI;
    static_assert(NQT * 128 * HD * 2 <= sizeof(s.vf), "the rows pass through the memory of V's stages");
    // asynchronous copies and small loops instead of registers and unrolled code: this runs once per CTA, from a cold
    // instruction cache. A lane takes 32 elements of a row (with 8 each, shuffles and addresses were most of the work).
    const int c = lane % LPR;
    uint8_t* raw = s.vf[0] + lane * 16;
#pragma unroll 1
    for (int g = warp; g < GROUPS; g += WARPS) {
      const int r = g * RPI + lane / LPR, tr = r & 127, ip = row_pos(x, tr), iq = x.q0 + (r >> 7) * x.per + ip;
      const bool live = tr < x.per * x.heads && iq < x.n;
      const bf16* src = p.q;
      if (live) src += ((int64_t)x.row0 + iq) * p.ldq + (int64_t)(x.h0 + tr - ip * x.heads) * HD + c * 16;
#pragma unroll
      for (int k = 0; k < 4; ++k)                          // two neighbouring pieces of 16 bytes, and two LPR pairs behind them
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(raw + g * 2048 + k * 512)),
                     "l"(src + (k >> 1) * (LPR * 16) + (k & 1) * 8), "r"(live ? 16 : 0) : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
    for (int g = warp; g < GROUPS; g += WARPS) {
      const int r = g * RPI + lane / LPR;
      uint4 v[4];                                          // this thread's own copies
      float am = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = *reinterpret_cast<const uint4*>(raw + g * 2048 + k * 512);
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
        for (int u = 0; u < 4; ++u)
          am = max3(am, fabsf(__uint_as_float(w[u] << 16)), fabsf(__uint_as_float(w[u] & 0xffff0000u)));
      }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
      const int eb = max((int)(__float_as_uint(am) >> 23), 20);
      const float mul = eb == 255 ? NAN : c8_pow2(134 - eb);      // an infinite element makes the row NaN, as its softmax is
      if (c == 0) s.crow[r] = c8_pow2(eb - 134) * p.scale_log2;
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint4& y = v[k + (u >> 1)];
          const uint32_t w0 = (u & 1) ? y.z : y.x, w1 = (u & 1) ? y.w : y.y;
          // scaled, a bf16 element is an f16 one exactly (to 2^-25), and so is what its nearest code leaves
          const uint32_t a = pack_h2(__uint_as_float(w0 << 16) * mul, __uint_as_float(w0 & 0xffff0000u) * mul);
          const uint32_t b = pack_h2(__uint_as_float(w1 << 16) * mul, __uint_as_float(w1 & 0xffff0000u) * mul);
          hi[u] = c8_codes4_h2(a, b);
          lo[u] = c8_codes4_h2(sub_h2(a, c8_half2_lo(hi[u])), sub_h2(b, c8_half2_hi(hi[u])));
        }
        const int c16 = (k >> 1) * LPR + c;
        const int at = (c16 / (INNER / 16)) * (128 * INNER) + code_at<INNER>(r & 127, c16 % (INNER / 16));
        *reinterpret_cast<uint4*>(s.q[r >> 7][0] + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(s.q[r >> 7][1] + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s.tmem_base;
  if (*reinterpret_cast<volatile uint32_t*>(&s.raised)) {      // an earlier kernel gave up: do nothing
    if (warp == C::SM_WARPS + 5) tmem_dealloc(tmem_base, C::TMEM_COLS);
    return;
  }
  if (warp >= C::SM_WARPS + 4) {
    if constexpr (NQT == 2) regs_dec<88>();
    const int role = warp - C::SM_WARPS - 4;
    if (role == 0) {
      // ---------------------------------------------------------------- TMA
      bool ok = true;
      for (int J = 1; J < n_pairs && ok && !s.abort; ++J) {
        const int next = row_of(J + 1);
        ok = load_pair(J, tma_row);
        tma_row = next;
      }
      if (!ok) A8_ABORT(s, status);
    } else if (role == 1 || (NQT == 2 && role == 3)) {
      // ---------------------------------------------------------------- MMA of tile t (whole warp, elected lane)
      const uint32_t leader = elect_one();
      // everything that the instructions are made of is the same in the warp, in a way that the compiler sees: descriptors are
      // computed in uniform registers (an 8192-token prompt: 603 -> 577 us)
      const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0);
      const int n_tiles_u = __shfl_sync(0xffffffffu, n_tiles, 0);
      auto wait_all = [&](uint64_t* bar, uint32_t parity) {
        return (bool)__all_sync(0xffffffffu, mbar_wait_relaxed(bar, parity));
      };
      constexpr uint32_t idesc_s = umma_idesc_e4m3(128, SK);
      constexpr uint32_t idesc_o = umma_idesc_f16(128, HD, 1);
      const uint64_t q_desc = code_desc<INNER>(smem_u32(s.q[0][0]));
      const uint64_t k_desc = code_desc<INNER>(smem_u32(s.k[0]));
      const uint64_t v_desc = umma_smem_desc(smem_u32(s.vf[0]), C::VF_SUB, 1024);    // MN-major
      const int t = role >> 1;
      auto issue_s = [&](int i) {                          // set i, both codes of q
        const uint64_t kd = k_desc + uint64_t((i / SPP % C::NK * C::K_STAGE + i % SPP * SK * INNER) >> 4);
        const uint32_t d = tmem_u + t * 128 + (i & 1) * SK;
#pragma unroll
        for (int part_i = 0; part_i < 2; ++part_i) {
          const uint64_t qd = q_desc + uint64_t((t * 2 + part_i) * (C::Q_PART >> 4));
#pragma unroll
          for (int kk = 0; kk < HD / 32; ++kk) {
            const int sl = kk / (INNER / 32), in = kk % (INNER / 32);
            umma_e4m3_ss_w(leader, d, qd + uint64_t((sl * 128 * INNER + in * 32) >> 4),
                           kd + uint64_t((sl * PKV * INNER + in * 32) >> 4), idesc_s, (part_i | kk) ? 1u : 0u);
          }
        }
        umma_commit_w(leader, &s.s_full[t][i & 1]);
      };
      auto issue_pv = [&](int jj) {                        // 64 keys: A = P in TMEM (8 packed columns per 16 keys), B = V
        const int i = jj / HPS, h = jj % HPS;
        const uint32_t pa = tmem_u + t * 128 + (i & 1) * SK + h * BKV;
        const uint64_t vd = v_desc + uint64_t((jj % C::NVF) * (C::VF_STAGE >> 4));
        const uint32_t d = tmem_u + C::O_COL + t * HD;
#pragma unroll
        for (int kk = 0; kk < BKV / 16; ++kk)
          umma_bf16_ts_w(leader, d, pa + kk * 8, vd + uint64_t((kk * 2048) >> 4), idesc_o, (jj > 0 || kk > 0) ? 1u : 0u);
        umma_commit_w(leader, &s.pv_done[t][i & 1][h]);
      };
      const int n_sets = (n_tiles_u + HPS - 1) / HPS;
      // before set i: its keys are there; behind it: they are free once the pair's last set is done
      auto keys_of = [&](int i) {
        if (i % SPP != 0) return true;
        const bool there = wait_all(&s.k_full[i / SPP % C::NK], (i / SPP / C::NK) & 1);
        tc_fence_after();
        return there;
      };
      auto keys_done = [&](int i) {
        if (i % SPP == SPP - 1 || i == n_sets - 1) umma_commit_w(leader, &s.k_empty[i / SPP % C::NK]);
      };
      bool ok = true;
      for (int i = 0; i < 2 && i < n_sets && ok; ++i) {    // all buffers' first scores
        ok = keys_of(i);
        if (ok) {
          issue_s(i);
          keys_done(i);
        }
      }
      for (int jj = 0; jj < n_tiles_u && ok && !__any_sync(0xffffffffu, s.abort); ++jj) {
        const int i = jj / HPS, h = jj % HPS, in = i + 2;  // in: the set whose scores go where this one's are
        const bool more = in < n_sets && h == HPS - 1;
        ok = wait_all(&s.vf_full[jj % C::NVF], (jj / C::NVF) & 1);
        ok = ok && wait_all(&s.p_ready[t][i & 1][h], (i >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        issue_pv(jj);
        umma_commit_w(leader, &s.vf_empty[jj % C::NVF]);
        if (more) {                                        // the buffer is consumed: the pipe runs its instructions in order
          ok = keys_of(in);
          if (!ok) break;
          issue_s(in);
          keys_done(in);
        }
      }
      if (!ok) A8_ABORT(s, status);
    } else if (role == 2) {
      // ---------------------------------------------------------------- scales: 32 blocks (8 tiles) at a time, one per lane
      auto fetch = [&](int grp, int& ke, int& ve) {
        ke = ve = 127;
        const int pos = key0 + (grp * 32 + lane) * C8_BLOCK;
        if (pos < x.len && pos + C8_BLOCK > x.lo && grp * 8 + (lane >> 2) < n_tiles) {
          const int r = pool_row(pos);
          if (r >= 0) {
            ke = p.c.ks[r / C8_BLOCK];
            ve = p.c.vs[r / C8_BLOCK];
          }
        }
      };
      const int groups = (n_tiles + 7) >> 3;
      int ke, ve;
      fetch(0, ke, ve);
      bool ok = true;
      for (int grp = 0; grp < groups && !s.abort; ++grp) {
        ok = mbar_wait_relaxed(&s.sc_empty[grp & 1], ((grp >> 1) & 1) ^ 1);
        if (!ok) break;
        s.sc[grp & 1][lane] = make_float4(c8_pow2(ke - 127), (float)(ve - 127), c8_pow2(127 - ve), 0.f);
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.sc_full[grp & 1]);
        if (grp + 1 < groups) fetch(grp + 1, ke, ve);
      }
      if (!ok) A8_ABORT(s, status);
    }
  } else if (warp >= C::SM_WARPS) {
    // ------------------------------------------------------------------ converters: V codes -> f16, 64 keys at a time
    if constexpr (NQT == 2) regs_dec<72>();
    const int tid = threadIdx.x - C::SM_WARPS * 32;
    constexpr int CPR = HD / 16;                         // 16-code pieces per row
    bool ok = true;
    for (int jj = 0; jj < n_tiles && !s.abort; ++jj) {
      const int vs = jj % C::NVR, vd = jj % C::NVF, kv0 = key0 + jj * BKV;
      ok = mbar_wait_relaxed(&s.vr_full[vs], (jj / C::NVR) & 1) &&
           mbar_wait_relaxed(&s.vf_empty[vd], ((jj / C::NVF) & 1) ^ 1);
      if (!ok) break;
      uint4 cur[C::LOADS];
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const int ci = i * 128 + tid, row = ci / CPR, c = ci % CPR;
        cur[i] = *reinterpret_cast<const uint4*>(s.vr[vs] + (c / (INNER / 16)) * (BKV * INNER) +
                                                 code_at<INNER>(row, c % (INNER / 16)));
        if (kv0 + row >= x.len || kv0 + row < x.lo) cur[i] = make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const int ci = i * 128 + tid, row = ci / CPR, c16 = ci % CPR;
        uint4 lo, hi;
        lo.x = c8_half2_lo(cur[i].x); lo.y = c8_half2_hi(cur[i].x); lo.z = c8_half2_lo(cur[i].y); lo.w = c8_half2_hi(cur[i].y);
        hi.x = c8_half2_lo(cur[i].z); hi.y = c8_half2_hi(cur[i].z); hi.z = c8_half2_lo(cur[i].w); hi.w = c8_half2_hi(cur[i].w);
        // two 16-byte chunks of the row's 128-byte slice; the threads of a warp that write the same chunk of two slices
        // take the two in opposite order (no bank conflict)
        uint8_t* base = s.vf[vd] + (c16 >> 2) * C::VF_SUB + row * 128;
        const int ch = (c16 & 3) * 2, sw = row & 7, flip = (c16 >> 2) & 1;
        *reinterpret_cast<uint4*>(base + (((ch + flip) ^ sw) << 4)) = flip ? hi : lo;
        *reinterpret_cast<uint4*>(base + (((ch + (flip ^ 1)) ^ sw) << 4)) = flip ? lo : hi;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s.vf_full[vd]);
        mbar_arrive(&s.vr_empty[vs]);
      }
    }
    if (!ok) A8_ABORT(s, status);
  } else {
    // ------------------------------------------------------------------ softmax warpgroups
    if constexpr (NQT == 2) regs_inc<176>();
    const int t = warp >> 2;
    const int quarter = warp & 3;
    const int row = quarter * 32 + lane;                  // row in the tile == TMEM lane
    const int ip_row = row_pos(x, row), i_row = x.q0 + t * x.per + ip_row;   // row of the sequence
    const bool used = row < x.per * x.heads && i_row < x.n;
    const int pos = used ? x.len - x.n + i_row : -1;      // its position; unused rows see nothing
    // positions of this tile's rows: keys up to pos_min need no causal mask, keys from pos_max - window on no window mask
    const int pos_min = x.pos0 + t * x.per;
    const int pos_max = pos_min + x.per - 1;
    const uint32_t lane_addr = uint32_t(quarter * 32) << 16;
    const uint32_t o_addr = tmem_base + lane_addr + C::O_COL + t * HD;
    const float c_row = s.crow[t * 128 + row];
    float m_run = -INFINITY;      // running (possibly stale) maximum of the exponent, ev included
    float l_run = 0.f;
    bool ok = true;
    auto wait_pv = [&](int jj) { return mbar_wait(&s.pv_done[t][jj / HPS & 1][jj % HPS], (jj / HPS >> 1) & 1); };

    for (int jj = 0; jj < n_tiles; ++jj) {
      const int kv0 = key0 + jj * BKV, set = jj / HPS, h = jj % HPS, grp = jj >> 3;
      const uint32_t sp_addr = tmem_base + lane_addr + t * 128 + (set & 1) * SK + h * BKV;
      if ((jj & 7) == 0 && !mbar_wait(&s.sc_full[grp & 1], (grp >> 1) & 1)) { ok = false; break; }
      float kf[4], lv[4], iv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 f = s.sc[grp & 1][(jj & 7) * 4 + k];
        kf[k] = fmaxf(f.x * c_row, 1e-37f);              // stays positive: a masked score times it stays -inf
        lv[k] = f.y;
        iv[k] = f.z;
      }
      if (h == 0) {
        if (!mbar_wait(&s.s_full[t][set & 1], (set >> 1) & 1)) { ok = false; break; }
        tc_fence_after();
      }
      float sv[BKV];
#pragma unroll
      for (int c = 0; c < BKV / 32; ++c)
        tmem_ld_32x32b_x32(sp_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[c * 32]));
      tmem_wait_ld();
      const bool masked = (kv0 + BKV - 1 > pos_min) || (p.window > 0 && kv0 <= pos_max - p.window);
      if (masked || !used) {
        const int lo = p.window > 0 ? pos - p.window : -1;   // seen keys: lo < j <= pos
#pragma unroll
        for (int i = 0; i < BKV; ++i) {
          const int j = kv0 + i;
          if (!(j <= pos && j > lo)) sv[i] = -INFINITY;
        }
      }
      // weights against the maximum the row already has; the tile's own maximum is reduced alongside and only checked
      // afterwards
      float l_tile, mx;
      uint32_t pk[BKV / 2];
      auto exps = [&](float m_use) {
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
        l_tile = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {                     // a block of 16 keys: one K scale, one V scale
          const float2 f2 = make_float2(kf[k], kf[k]);
          const float add = lv[k] - m_use;
          const float2 a2 = make_float2(add, add);
          float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const float* v = sv + k * 16 + c * 8;
            float2 x0 = __ffma2_rn(make_float2(v[0], v[1]), f2, a2);
            float2 x1 = __ffma2_rn(make_float2(v[2], v[3]), f2, a2);
            float2 x2 = __ffma2_rn(make_float2(v[4], v[5]), f2, a2);
            float2 x3 = __ffma2_rn(make_float2(v[6], v[7]), f2, a2);
            mx0 = max3(mx0, x0.x, x0.y);
            mx1 = max3(mx1, x1.x, x1.y);
            mx2 = max3(mx2, x2.x, x2.y);
            mx3 = max3(mx3, x3.x, x3.y);
            x0.x = ex2(x0.x); x0.y = ex2(x0.y);
            x1.x = ex2(x1.x); x1.y = ex2(x1.y);
            x2.x = ex2(x2.x); x2.y = ex2(x2.y);
            x3.x = ex2(x3.x); x3.y = ex2(x3.y);
            acc0 = __fadd2_rn(acc0, x0);
            acc1 = __fadd2_rn(acc1, x1);
            acc0 = __fadd2_rn(acc0, x2);
            acc1 = __fadd2_rn(acc1, x3);
            pk[k * 8 + c * 4 + 0] = pack_h2(x0.x, x0.y);
            pk[k * 8 + c * 4 + 1] = pack_h2(x1.x, x1.y);
            pk[k * 8 + c * 4 + 2] = pack_h2(x2.x, x2.y);
            pk[k * 8 + c * 4 + 3] = pack_h2(x3.x, x3.y);
          }
          l_tile = fmaf((acc0.x + acc0.y) + (acc1.x + acc1.y), iv[k], l_tile);
        }
        mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) + m_use;
      };
      exps((m_run == -INFINITY ? 0.f : m_run) - W_SHIFT);
      const float m_new = fmaxf(m_run, mx);
      const bool need = (m_new - m_run > 8.0f) || (m_run == -INFINITY && m_new > -INFINITY);
      if (__any_sync(0xffffffffu, need)) {
        // the maximum grew by more than 2^8 somewhere in this warp (in practice: a row's first tiles): rescale the
        // accumulator to the new maximum and take the exponentials again
        const float factor = (m_new == -INFINITY) ? 1.0f : ex2(m_run - m_new);   // ex2(-inf) = 0
        if (jj > 0) {
          if (!wait_pv(jj - 1)) { ok = false; break; }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(o_addr + c * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
            tmem_st_32x32b_x32(o_addr + c * 32, o);
          }
          tmem_wait_st();
        }
        l_run *= factor;
        m_run = m_new;
        exps((m_run == -INFINITY ? 0.f : m_run) - W_SHIFT);
      }
      l_run += l_tile;
      tmem_st_32x32b_x32(sp_addr, pk);      // over the scores this thread has just consumed
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s.p_ready[t][set & 1][h]);
        if ((jj & 7) == 7) mbar_arrive(&s.sc_empty[grp & 1]);
      }
    }
    if (ok && !s.abort) {
      if (!wait_pv(n_tiles - 1)) {
        ok = false;
      } else {
        tc_fence_after();
        const bool none = l_run == 0.f;                          // a row that sees nothing is a row of zeros
        const float inv = none ? 0.f : 1.0f / l_run;
        bf16* out = p.out + ((int64_t)x.row0 + i_row) * p.ldo + (int64_t)(x.h0 + row - ip_row * x.heads) * HD;
        float* pr = part != nullptr ? part + (int64_t)(t * 128 + row) * (HD + 4) : nullptr;
        if (pr != nullptr) *reinterpret_cast<float4*>(pr) = make_float4(m_run, l_run, 0.f, 0.f);
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(o_addr + c * 32, o);
          tmem_wait_ld();
          if (none) {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0;
          }
          if (pr != nullptr) {
#pragma unroll
            for (int v = 0; v < 8; ++v)
              *reinterpret_cast<uint4*>(pr + 4 + c * 32 + v * 4) = make_uint4(o[v * 4], o[v * 4 + 1], o[v * 4 + 2], o[v * 4 + 3]);
          } else if (used) {
            uint32_t w[16];
#pragma unroll
            for (int v = 0; v < 16; ++v)
              w[v] = pack_b2(__uint_as_float(o[v * 2]) * inv, __uint_as_float(o[v * 2 + 1]) * inv);
#pragma unroll
            for (int v = 0; v < 16; v += 8) {
              bf16* dst = out + c * 32 + v * 2;
              if (p.out32) {                             // a sector at once: half the stores, each of 32 different lines
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(w[v]), "r"(w[v + 1]),
                             "r"(w[v + 2]), "r"(w[v + 3]), "r"(w[v + 4]), "r"(w[v + 5]), "r"(w[v + 6]), "r"(w[v + 7]) : "memory");
              } else {
                *reinterpret_cast<uint4*>(dst) = make_uint4(w[v], w[v + 1], w[v + 2], w[v + 3]);
                *reinterpret_cast<uint4*>(dst + 8) = make_uint4(w[v + 4], w[v + 5], w[v + 6], w[v + 7]);
              }
            }
          }
        }
      }
    }
    if (!ok) A8_ABORT(s, status);
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (s.abort && threadIdx.x == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // let in-flight bulk copies land
  }
  __syncthreads();
  if (warp == C::SM_WARPS + 5) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

// Merge of the pieces of split rows: one warp per row, grid as the attention kernel's without the splits.
template <int HD, int NQT>
__global__ void __launch_bounds__(256) attn8_merge_kernel(const __grid_constant__ A8Dev p, int* __restrict__ status) {
  chain_trigger();
  chain_wait();
  // read once per CTA, while the lengths are on their way: 3 x 512 rows 238.8 us, with every warp's read of the one word 242.5
  const int word = threadIdx.x == 0 ? *reinterpret_cast<const volatile int*>(status) : 0;
  const int groups = NQT * 128 / 8;
  const int by = blockIdx.y / groups, r = (blockIdx.y % groups) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const Job x = job_of<NQT>(p, blockIdx.x, by, blockIdx.z, status);
  const int pieces = pieces_of(p, x);
  if (__syncthreads_or(gave_up(word)) || x.q0 < 0 || pieces == 1) return;   // gave up: there are pieces that nobody wrote
  const int in_tile = r & 127, ip = row_pos(x, in_tile), i = x.q0 + (r >> 7) * x.per + ip;
  if (in_tile >= x.per * x.heads || i >= x.n) return;
  constexpr int PER = HD / 32;
  float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) o[k] = 0.f;
  const int64_t stride = (int64_t)p.q_tiles * gridDim.x * (NQT * 128) * (HD + 4);           // from piece to piece
  const float* src = p.partial + (((int64_t)blockIdx.z * p.splits * p.q_tiles + by) * gridDim.x + blockIdx.x) *
                                     (int64_t)(NQT * 128) * (HD + 4) + (int64_t)r * (HD + 4);
  for (int s0 = 0; s0 < pieces; s0 += 32, src += 32 * stride) {
    // a lane per piece: its share in the sum; every piece has written its row, zeros where it saw nothing
    const int live = min(32, pieces - s0);
    float ms = -INFINITY, ls = 0.f;
    if (lane < live) {
      ms = __ldcg(src + lane * stride);
      ls = __ldcg(src + lane * stride + 1);
    }
    float n = fmaxf(m, ms);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, d));
    // no maximum so far: the pieces saw nothing (zeros), or scores that are all NaN, whose sums stay NaN
    const float z = n == -INFINITY ? 0.f : n;
    const float f = ex2(m - z), w = ex2(ms - z);
    float sum = w * ls;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    l = l * f + sum;
    m = n;
#pragma unroll
    for (int k = 0; k < PER; ++k) o[k] *= f;
#pragma unroll 4
    for (int q = 0; q < live; ++q) {
      const float wq = __shfl_sync(0xffffffffu, w, q);
#pragma unroll
      for (int k = 0; k < PER; k += 2) {
        const float2 v = __ldcg(reinterpret_cast<const float2*>(src + q * stride + 4 + lane * 2 + k * 32));
        o[k] = fmaf(v.x, wq, o[k]);
        o[k + 1] = fmaf(v.y, wq, o[k + 1]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;      // l 0: no piece saw a key, the sums are zeros
  bf16* dst = p.out + ((int64_t)x.row0 + i) * p.ldo + (int64_t)(x.h0 + in_tile - ip * x.heads) * HD + lane * 2;
#pragma unroll
  for (int k = 0; k < PER; k += 2)
    *reinterpret_cast<__nv_bfloat162*>(dst + k * 32) = __floats2bfloat162_rn(o[k] * inv, o[k + 1] * inv);
}

template <int HD, int NQT>
int launch_t(const Attn8Args& a, A8Dev& p, cudaStream_t s) {
  using C = A8<HD, NQT>;
  const size_t smem = sizeof(A8Smem<HD, NQT>) + 1024;
  static_assert(sizeof(A8Smem<HD, NQT>) + 1024 <= kSmemLimit, "shared memory budget");
  const int per = p.per;
  const int64_t q_tiles = ((int64_t)a.rows + NQT * per - 1) / (NQT * per);
  if (q_tiles > 65535) return POP_E_INVALID;
  p.q_tiles = (int)q_tiles;
  const int64_t base = (int64_t)a.n_kv * p.hg * q_tiles * a.batch;
  // Positions of a CTA at most: the last of several head groups may have fewer heads than the others, so more of them
  const int most = NQT * (128 / (p.G - (p.hg - 1) * 128)), reach = most < a.rows ? most : a.rows;
  // Pieces per tile: what takes the fewest turns of all SMs at the longest sequence's keys. The unit is a tile of 64 keys
  // (1.1 us at hd 128); beginning and ending a CTA costs eight, the merge four and its reads one per 96 pieces. Never more
  // than what POP_E4M3_WORKSPACE_BYTES holds, so that a workspace of that size covers every call.
  const int64_t span = p.window > 0 && (int64_t)p.window + reach < a.kv_len ? p.window + reach : a.kv_len;
  const int64_t sms = device_sms(), piece = (int64_t)NQT * 128 * (HD + 4) * 4;
  const int64_t tiles = span < 64 ? 1 : (span + 63) / 64 + (p.window > 0 ? 1 : 0);
  int64_t splits = 1, chunk = tiles, best = INT64_MAX;
  for (int64_t n = 1; n == 1 || (n <= sms && base * n <= 4 * sms && base * n * piece <= POP_E4M3_WORKSPACE_BYTES); ++n) {
    const int64_t c = n > 1 && tiles < 4 * n ? 4 : (tiles + n - 1) / n;         // four tiles or more to a piece
    const int64_t turns = (base * n + sms - 1) / sms, cost = turns * (c + 8) + (n > 1 ? 4 + base * n / 96 : 0);
    if (cost < best) {
      best = cost;
      chunk = c;
      splits = (tiles + c - 1) / c;
    }
    if (c <= 4) break;
  }
  p.splits = (int)splits;
  p.chunk = (int)chunk;
  if (splits > 1 && (size_t)(base * splits * piece) > a.workspace_bytes) return POP_E_NOSPACE;
  if (a.batch * splits > 65535) return POP_E_INVALID;
  static std::atomic<uint64_t> configured{0};
  if (!c8_allow_smem(configured, reinterpret_cast<const void*>(attn8_kernel<HD, NQT>), (int)smem)) return POP_E_CUDA;
  int* status = status_word();
  if (!status) return POP_E_CUDA;
  CUtensorMap tk, tv;
  if (make_tmap_u8_rows(&tk, a.c.k, HD, p.pool_rows, C::INNER, p.box) != POP_OK ||
      make_tmap_u8_rows(&tv, a.c.v, HD, p.pool_rows, C::INNER, p.box) != POP_OK)
    return POP_E_CUDA;
  ProfScope prof(PROF_ATTENTION, 4.0 * HD * a.n_q * a.batch * (double)a.rows * (span - (p.window > 0 ? 0.0 : 0.5 * a.rows)), s);
  if (launch_chained(attn8_kernel<HD, NQT>, dim3(a.n_kv * p.hg, (unsigned)q_tiles, (unsigned)(a.batch * splits)),
                     dim3(C::THREADS), smem, s, tk, tv, p, status) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  if (splits > 1) {
    if (launch_chained(attn8_merge_kernel<HD, NQT>, dim3(a.n_kv * p.hg, (unsigned)(q_tiles * (NQT * 16)), a.batch),
                       dim3(256), 0, s, p, status) != cudaSuccess)
      return POP_E_CUDA;
    count_launch();
  }
  return POP_OK;
}

}  // namespace

int launch_attention8(const Attn8Args& a, cudaStream_t s) {
  if (!a.q || !a.out || !c8_cache_ok(a.c)) return POP_E_INVALID;
  if (a.batch < 1 || a.batch > 65535 || a.n_kv < 1 || a.n_q < 1 || a.n_q % a.n_kv || a.n_q > 65536 || a.rows < 0 ||
      a.kv_len < 0 || a.kv_len > 0x7fff0000 || a.window < 0 || a.window > 0x7ffffff0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8)
    return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.workspace) % 16 || (int64_t)a.batch * a.rows > 0x7fffffff) return POP_E_INVALID;
  if (!a.seq_lens && a.rows > a.kv_len) return POP_E_INVALID;
  if ((int64_t)a.batch * a.rows > 1 && a.ldo < (int64_t)a.n_q * a.head_dim) return POP_E_INVALID;     // rows over each other
  // rows of the pool are 32-bit coordinates
  if (a.c.num_pages * (int64_t)a.n_kv > 0x7ffffff0 / a.c.page_size) return POP_E_INVALID;
  if ((int64_t)a.kv_len > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  if (a.rows == 0) return POP_OK;
  // few (row, head) columns per kv head: the kernel that streams the cache
  if ((int64_t)a.rows * (a.n_q / a.n_kv) <= FEW_COLUMNS && a.batch <= 4096) return launch_few8(a, s);
  A8Dev p{};
  p.q = a.q; p.ldq = a.ldq;
  p.c = a.c;
  p.box = a.c.page_size < 64 ? a.c.page_size : 64;
  p.pool_rows = (int)(a.c.num_pages * (int64_t)a.n_kv * a.c.page_size);
  p.cu = a.cu; p.rows = a.rows;
  p.seq_lens = a.seq_lens; p.kv_len = a.kv_len;
  p.out = a.out; p.ldo = a.ldo;
  p.out32 = reinterpret_cast<uintptr_t>(a.out) % 32 == 0 && a.ldo % 16 == 0;
  p.n_q = a.n_q; p.n_kv = a.n_kv; p.G = a.n_q / a.n_kv; p.hg = (p.G + 127) / 128;
  p.per = 128 / (p.G < 128 ? p.G : 128);
  p.inv = (65536 + p.G - 1) / p.G;
  p.window = a.window < a.kv_len ? a.window : 0;         // a longer one hides nothing
  p.partial = static_cast<float*>(a.workspace);
  p.scale_log2 = 1.4426950408889634f / sqrtf((float)a.head_dim);
  // one tile of 128 rows where no sequence has more
  const bool small = (int64_t)a.rows * (p.G < 128 ? p.G : 128) <= 128;
  switch (a.head_dim) {
    case 64: return small ? launch_t<64, 1>(a, p, s) : launch_t<64, 2>(a, p, s);
    case 128: return small ? launch_t<128, 1>(a, p, s) : launch_t<128, 2>(a, p, s);
    default: return launch_t<256, 1>(a, p, s);
  }
}

}  // namespace pop
