// Causal attention of many query rows over the 8-bit paged cache (paper Eq. 1, Attn(x_l, K, V)), with an optional
// sliding window: the prompt, a chunk of one, or a few drafted tokens behind a long cache.
//
// The last rows of a sequence are the queries: row i of n at position len - n + i sees positions j <= its own (and
// j > it - window). With codes k_j, v_j, block exponents ek, ev and c = log2(e) / sqrt(hd):
//   w_j = exp2(c q.k_j 2^(ek) + ev - m),  out = sum_j w_j v_j / sum_j w_j 2^(-ev)
// (m the running maximum of the exponent without -m): the block scales never touch the tensor cores' operands, which are
// the codes themselves as f16 (exact), the query as f16 after a power-of-two scale per row (exact down to 2^-36 of the
// row's largest element) and the weights as f16. Scores, statistics, sums and the accumulator are fp32.
//
// A CTA owns NQT tiles of 128 rows of one kv head; a row is a (position, query head) pair of that kv head, so that the
// keys are read and converted once for all heads that share them, however few the positions are. Keys are walked 64
// at a time. Warp roles:
//   NQT softmax warpgroups, one row per thread: place Q in shared memory, then read S = Q K^T from one of two TMEM
//       buffers, write the weights over it, rescale the TMEM accumulator when the maximum grew by more than 2^8;
//   4 converter warps: 16 codes per load straight from the paged cache, a tile ahead of its use, to f16 in the
//       128-byte-swizzled operand layout (K-major for K, MN-major for V: the same bytes); positions past the end become
//       zeros, the blocks' scales go to a small ring beside them;
//   1 MMA warp: scores two key tiles ahead of the softmax, then O += P V with P from TMEM.
// With fewer CTAs than SMs (few rows) the keys are split over several CTAs, which leave unnormalised rows in the
// workspace for a second, chained launch to merge.
#include "cache8.cuh"
#include "ptx.cuh"

namespace pop {
namespace {

constexpr int kSmemLimit = 227 * 1024;
constexpr float W_SHIFT = 7.f;        // weights are stored times 2^7; the lazy maximum lets them reach 2^15
constexpr int SC_RING = 16;           // key tiles whose scales are held: more than the ring of operand tiles can be ahead

template <int HD, int NQT>
struct A8 {
  static constexpr int BKV = 64;
  static constexpr int KV_TILE_BYTES = BKV * HD * 2;
  static constexpr int KV_SUB_BYTES = BKV * 128;     // one 64-wide slice of head_dim
  static constexpr int Q_TILE_BYTES = 128 * HD * 2;
  static constexpr int RING_BYTES = kSmemLimit - 4 * 1024 - NQT * Q_TILE_BYTES;   // alignment slack, scales, barriers
  static constexpr int STAGES = RING_BYTES / KV_TILE_BYTES < 8 ? RING_BYTES / KV_TILE_BYTES : 8;
  static constexpr int SM_WARPS = NQT * 4;
  static constexpr int THREADS = (SM_WARPS + 4 + 1) * 32;
  static constexpr int LOADS = BKV * HD / (16 * 128);          // 16-byte loads of a tile per converter thread
  static constexpr int S_COL = 0;                    // S_t[b] at (t * 2 + b) * 64
  static constexpr int O_COL = NQT * 2 * BKV;        // O_t at O_COL + t * HD
  static constexpr int COLS_USED = O_COL + NQT * HD;
  static constexpr uint32_t TMEM_COLS = COLS_USED <= 128 ? 128 : (COLS_USED <= 256 ? 256 : 512);
  static_assert(COLS_USED <= 512, "TMEM budget");
  static_assert(STAGES >= 4, "ring too shallow");
};

template <int HD, int NQT>
struct __align__(1024) A8Smem {
  using C = A8<HD, NQT>;
  uint8_t q[NQT][C::Q_TILE_BYTES];
  uint8_t kv[C::STAGES][C::KV_TILE_BYTES];
  float4 sc[SC_RING][4];        // per block of 16 keys: 2^ek, ev, 2^-ev
  uint64_t q_full;
  uint64_t kv_full[C::STAGES];
  uint64_t kv_empty[C::STAGES];
  uint64_t sc_full[SC_RING];
  uint64_t s_full[NQT][2];      // S_t[b] = Q_t K^T complete, b = key tile & 1, phase = key tile >> 1
  uint64_t p_ready[NQT][2];     // P_t[b] written over S_t[b] (one arrival per softmax warp)
  uint64_t pv_done[NQT][2];     // O_t += P_t[b] V complete
  uint32_t tmem_base;
  uint32_t raised;
  volatile uint32_t abort;
};

struct A8Dev {
  const bf16* q; int64_t ldq;
  Cache8 c;
  int ps_log2;                  // log2 of the page size, or -1
  const int32_t* cu; int rows;
  const int32_t* seq_lens; int kv_len;
  bf16* out; int64_t ldo;
  int n_q, n_kv, G, hg;         // query heads per kv head; head groups of at most 128 per kv head
  int window;
  int q_tiles;                  // CTAs along the rows of the longest sequence
  int splits;
  float* partial;               // [CTA][NQT * 128][hd + 4]: m, l, two unused, accumulator
  float scale_log2;
};

// The rows and keys of one CTA (without the split)
struct Job {
  int b, kvh, h0, heads, per;   // heads of this group; positions per tile
  int row0, n, q0;              // first packed row of the sequence, its rows, first row of the CTA
  int len, pos0;                // cached positions; position of row q0
  int j_lo, n_tiles;            // 64-key tiles that its rows see
};
template <int NQT>
__device__ __forceinline__ Job job_of(const A8Dev& p, int bx, int by, int b, int* status) {
  Job x;
  x.b = b;
  x.kvh = bx / p.hg;
  const int grp = bx - x.kvh * p.hg;
  x.h0 = x.kvh * p.G + grp * 128;
  x.heads = min(128, p.G - grp * 128);
  x.per = 128 / x.heads;
  x.row0 = p.cu ? p.cu[b] : b * p.rows;
  x.n = p.cu ? p.cu[b + 1] - x.row0 : p.rows;
  x.len = p.seq_lens ? p.seq_lens[b] : p.kv_len;
  if (x.len > p.kv_len || x.n > p.rows) {       // more than the caller said: nothing past it is touched
    atomicMin(status, (int)POP_E_INVALID);
    x.n = min(x.n, p.rows);
    x.len = min(x.len, p.kv_len);
  }
  x.len = max(x.len, 0);
  const int tile = (int)(((int64_t)x.n + (int64_t)NQT * x.per - 1) / (NQT * x.per)) - 1 - by;   // latest rows first
  x.q0 = tile * NQT * x.per;
  x.pos0 = x.len - x.n + x.q0;
  const int last = min(x.pos0 + NQT * x.per - 1, x.len - 1);
  x.j_lo = p.window > 0 ? max(0, x.pos0 - p.window + 1) / 64 : 0;
  x.n_tiles = last < 0 || tile < 0 ? 0 : last / 64 - x.j_lo + 1;
  return x;
}

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
__device__ __forceinline__ uint32_t pack_b2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Instruction descriptor for kind::f16 with f16 A and B (format 0 in both fields); see umma_idesc_bf16
__host__ __device__ constexpr uint32_t umma_idesc_f16(int m, int n, int b_mn_major) {
  return (1u << 4) | (uint32_t(b_mn_major) << 16) | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}

#define A8_ABORT(S, status)                           \
  do {                                                \
    (S).abort = 1;                                    \
    atomicMin((status), (int)POP_E_DEVICE_TIMEOUT);   \
  } while (0)

template <int HD, int NQT>
__global__ void __launch_bounds__(A8<HD, NQT>::THREADS, 1)
attn8_kernel(const __grid_constant__ A8Dev p, int* __restrict__ status) {
  using C = A8<HD, NQT>;
  constexpr int BKV = C::BKV, STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  A8Smem<HD, NQT>& s =
      *reinterpret_cast<A8Smem<HD, NQT>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  chain_trigger();
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  chain_wait();
  const int split = blockIdx.z % p.splits;
  const Job x = job_of<NQT>(p, blockIdx.x, blockIdx.y, blockIdx.z / p.splits, status);
  if (x.q0 < 0) return;                                  // past the rows of this sequence
  const int t_lo = (int)((int64_t)x.n_tiles * split / p.splits);
  const int n_tiles = (int)((int64_t)x.n_tiles * (split + 1) / p.splits) - t_lo;
  const int j_lo = x.j_lo + t_lo;
  float* part = p.splits > 1 ? p.partial + (((int64_t)(blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) *
                                            (NQT * 128)) * (HD + 4)
                             : nullptr;

  if (status_raised(status, &s.raised)) return;
  if (n_tiles <= 0) {                                    // rows that see nothing (here): zeros, or an empty piece
    for (int r = threadIdx.x; r < NQT * 128; r += blockDim.x) {
      if (part != nullptr) {
        part[(int64_t)r * (HD + 4)] = -INFINITY;
        part[(int64_t)r * (HD + 4) + 1] = 0.f;
        continue;
      }
      const int in_tile = r & 127, i = x.q0 + (r >> 7) * x.per + in_tile / x.heads;
      if (in_tile >= x.per * x.heads || i >= x.n) continue;
      uint4* dst = reinterpret_cast<uint4*>(p.out + ((int64_t)x.row0 + i) * p.ldo +
                                            (int64_t)(x.h0 + in_tile % x.heads) * HD);
      for (int c = 0; c < HD / 8; ++c) dst[c] = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  if (threadIdx.x == 0) {
    mbar_init(&s.q_full, C::SM_WARPS);
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(&s.kv_full[i], 4);
      mbar_init(&s.kv_empty[i], 1);
    }
    for (int i = 0; i < SC_RING; ++i) mbar_init(&s.sc_full[i], 1);
    for (int t = 0; t < NQT; ++t)
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s.s_full[t][i], 1);
        mbar_init(&s.p_ready[t][i], 4);
        mbar_init(&s.pv_done[t][i], 1);
      }
    s.abort = 0;
    fence_barrier_init();
  }
  if (warp == C::SM_WARPS + 4) {
    tmem_alloc(&s.tmem_base, C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s.tmem_base;

  if (warp >= C::SM_WARPS && warp < C::SM_WARPS + 4) {
    // ------------------------------------------------------------------ converters
    const int tid = threadIdx.x - C::SM_WARPS * 32;
    constexpr int CPR = HD / 16;                         // 16-code pieces per row
    const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;
    const int ps = p.c.page_size;
    // pool row (page * n_kv + head) * page_size + slot of a position below len, or -1
    auto pool_row = [&](int pos) -> int64_t {
      const int pi = p.ps_log2 >= 0 ? pos >> p.ps_log2 : pos / ps;
      const int page = bt[pi];
      if ((unsigned)page >= (unsigned)p.c.num_pages) {   // never turned into an address: reads as zeros
        atomicMin(status, (int)POP_E_INVALID);
        return -1;
      }
      return ((int64_t)page * p.n_kv + x.kvh) * ps + (pos - pi * ps);
    };
    auto load_tile = [&](const uint8_t* pool, int j, uint4 (&r)[C::LOADS]) {
      const int kv0 = (j_lo + j) * BKV;
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const int ci = i * 128 + tid, pos = kv0 + ci / CPR;
        r[i] = make_uint4(0, 0, 0, 0);
        if (pos < x.len) {
          const int64_t row = pool_row(pos);
          if (row >= 0) r[i] = *reinterpret_cast<const uint4*>(pool + row * HD + (ci % CPR) * 16);
        }
      }
    };
    int ke = 127, ve = 127;                              // threads 0..3: scales of the tile's four blocks
    auto load_scales = [&](int j) {
      ke = ve = 127;
      const int pos = (j_lo + j) * BKV + tid * C8_BLOCK;
      if (tid < 4 && pos < x.len) {
        const int64_t row = pool_row(pos);
        if (row >= 0) {
          ke = p.c.ks[row / C8_BLOCK];
          ve = p.c.vs[row / C8_BLOCK];
        }
      }
    };
    // ring order = the order the MMA warp consumes: K_0, K_1, then V_j, K_{j+2} for j = 0, 1, ...
    const int total = 2 * n_tiles;
    auto entry = [&](int r, bool& is_v, int& j) {
      if (r < 2 && r < n_tiles) { is_v = false; j = r; return; }
      // behind K_0, K_1: V_0 K_2 V_1 K_3 ... and the last two V without a K between
      const int k = r - (n_tiles < 2 ? n_tiles : 2);
      const int pairs = n_tiles > 2 ? n_tiles - 2 : 0;
      if (k < 2 * pairs) { is_v = !(k & 1); j = is_v ? k >> 1 : (k >> 1) + 2; }
      else { is_v = true; j = pairs + (k - 2 * pairs); }
    };
    uint4 cur[C::LOADS], nxt[C::LOADS];
    bool is_v;
    int j;
    entry(0, is_v, j);
    load_tile(p.c.k, j, cur);
    load_scales(j);
    bool ok = true;
    for (int r = 0; r < total && !s.abort; ++r) {
      const int ke_c = ke, ve_c = ve, j_c = j;
      const bool v_c = is_v;
      if (r + 1 < total) {
        entry(r + 1, is_v, j);
        load_tile(is_v ? p.c.v : p.c.k, j, nxt);
        if (!is_v) load_scales(j);
      }
      const int stage = r % STAGES;
      if (!mbar_wait_relaxed(&s.kv_empty[stage], ((r / STAGES) & 1) ^ 1)) { ok = false; break; }
      if (!v_c && tid < 4) s.sc[j_c % SC_RING][tid] = make_float4(c8_pow2(ke_c - 127), (float)(ve_c - 127), c8_pow2(127 - ve_c), 0.f);
      uint8_t* dst = s.kv[stage];
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) {
        const int ci = i * 128 + tid, row = ci / CPR, c16 = ci % CPR;
        uint4 lo, hi;
        lo.x = c8_half2_lo(cur[i].x); lo.y = c8_half2_hi(cur[i].x); lo.z = c8_half2_lo(cur[i].y); lo.w = c8_half2_hi(cur[i].y);
        hi.x = c8_half2_lo(cur[i].z); hi.y = c8_half2_hi(cur[i].z); hi.z = c8_half2_lo(cur[i].w); hi.w = c8_half2_hi(cur[i].w);
        // two 16-byte chunks of the row's 128-byte slice; the halves of a warp that write the same chunk of two
        // slices take the two in opposite order (no bank conflict)
        uint8_t* base = dst + (c16 >> 2) * C::KV_SUB_BYTES + row * 128;
        const int ch = (c16 & 3) * 2, sw = row & 7, flip = (c16 >> 2) & 1;
        *reinterpret_cast<uint4*>(base + (((ch + flip) ^ sw) << 4)) = flip ? hi : lo;
        *reinterpret_cast<uint4*>(base + (((ch + (flip ^ 1)) ^ sw) << 4)) = flip ? lo : hi;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&s.kv_full[stage]);
        if (!v_c && tid == 0) mbar_arrive(&s.sc_full[j_c % SC_RING]);
      }
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) cur[i] = nxt[i];
    }
    if (!ok) A8_ABORT(s, status);
  } else if (warp == C::SM_WARPS + 4) {
    // ------------------------------------------------------------------ MMA issuer (whole warp, elected lane)
    const uint32_t leader = elect_one();
    constexpr uint32_t idesc_s = umma_idesc_f16(128, BKV, 0);
    constexpr uint32_t idesc_o = umma_idesc_f16(128, HD, 1);
    uint64_t q_desc[NQT];
    for (int t = 0; t < NQT; ++t) q_desc[t] = umma_smem_desc(smem_u32(s.q[t]), 16, 1024);
    const uint64_t k_desc0 = umma_smem_desc(smem_u32(s.kv[0]), 16, 1024);                 // K-major
    const uint64_t v_desc0 = umma_smem_desc(smem_u32(s.kv[0]), C::KV_SUB_BYTES, 1024);    // MN-major
    auto issue_s = [&](int t, int j, int stage) {
      const uint64_t qd = q_desc[t];
      const uint64_t kd = k_desc0 + uint64_t(stage * (C::KV_TILE_BYTES >> 4));
      const uint32_t d = tmem_base + C::S_COL + (t * 2 + (j & 1)) * BKV;
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk) {
        const uint64_t ad = qd + uint64_t(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4);
        const uint64_t bd = kd + uint64_t(((kk >> 2) * C::KV_SUB_BYTES + (kk & 3) * 32) >> 4);
        umma_bf16_ss_w(leader, d, ad, bd, idesc_s, kk > 0 ? 1u : 0u);
      }
      umma_commit_w(leader, &s.s_full[t][j & 1]);
    };
    auto issue_pv = [&](int t, int j, int stage) {
      // A operand = P_t in TMEM: 16 keys are 8 packed 32-bit columns; B = V tile, MN-major
      const uint32_t pa = tmem_base + C::S_COL + (t * 2 + (j & 1)) * BKV;
      const uint64_t vd = v_desc0 + uint64_t(stage * (C::KV_TILE_BYTES >> 4));
      const uint32_t d = tmem_base + C::O_COL + t * HD;
#pragma unroll
      for (int kk = 0; kk < BKV / 16; ++kk)
        umma_bf16_ts_w(leader, d, pa + kk * 8, vd + uint64_t((kk * 2048) >> 4), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
      umma_commit_w(leader, &s.pv_done[t][j & 1]);
    };
    int ring = 0;
    auto wait_tile = [&](int& stage) {      // next ring entry, in the converters' order
      stage = ring % STAGES;
      const uint32_t phase = (ring / STAGES) & 1;
      ++ring;
      return mbar_wait_relaxed(&s.kv_full[stage], phase);
    };
    bool ok = mbar_wait_relaxed(&s.q_full, 0);
    for (int j = 0; j < 2 && j < n_tiles && ok; ++j) {
      int sk;
      ok = wait_tile(sk);
      if (!ok) break;
      tc_fence_after();
      for (int t = 0; t < NQT; ++t) issue_s(t, j, sk);
      umma_commit_w(leader, &s.kv_empty[sk]);
    }
    for (int jj = 0; jj < n_tiles && ok && !s.abort; ++jj) {
      int sv, sk = 0;
      ok = wait_tile(sv);
      const bool more = jj + 2 < n_tiles;
      for (int t = 0; t < NQT && ok; ++t) {
        ok = mbar_wait_relaxed(&s.p_ready[t][jj & 1], (jj >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        issue_pv(t, jj, sv);
        if (more) {
          // the scores of key tile jj+2 go into the buffer P_t(jj) occupies: the tensor pipe runs its instructions
          // in order, so the product above has read P before this overwrites it
          if (t == 0) {
            ok = wait_tile(sk);
            if (!ok) break;
            tc_fence_after();
          }
          issue_s(t, jj + 2, sk);
        }
      }
      if (ok) {
        umma_commit_w(leader, &s.kv_empty[sv]);
        if (more) umma_commit_w(leader, &s.kv_empty[sk]);
      }
    }
    if (!ok) A8_ABORT(s, status);
  } else {
    // ------------------------------------------------------------------ softmax warpgroups
    const int t = warp >> 2;
    const int quarter = warp & 3;
    const int row = quarter * 32 + lane;                  // row in the tile == TMEM lane
    const int i_row = x.q0 + t * x.per + row / x.heads;   // row of the sequence
    const bool used = row < x.per * x.heads && i_row < x.n;
    const int pos = used ? x.len - x.n + i_row : -1;      // its position; unused rows see nothing
    // positions of this tile's rows: keys up to `pos_min` need no causal mask, keys below `edge` a window mask
    const int pos_min = x.pos0 + t * x.per;
    const int pos_max = pos_min + x.per - 1;
    const uint32_t lane_addr = uint32_t(quarter * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_addr + C::S_COL + t * 2 * BKV;
    const uint32_t o_addr = tmem_base + lane_addr + C::O_COL + t * HD;
    // this thread's query row, scaled so that its largest element is in [2^12, 2^13)
    float c_row;
    {
      const uint4* src = reinterpret_cast<const uint4*>(p.q + ((int64_t)x.row0 + (used ? i_row : 0)) * p.ldq +
                                                        (int64_t)(x.h0 + (used ? row % x.heads : 0)) * HD);
      float am = 0.f;
#pragma unroll 4
      for (int c = 0; c < HD / 8; ++c) {
        const uint4 v = used ? src[c] : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          am = max3(am, fabsf(__uint_as_float(w[k] << 16)), fabsf(__uint_as_float(w[k] & 0xffff0000u)));
      }
      const int eb = max((int)(__float_as_uint(am) >> 23), 20);
      const float mul = c8_pow2(139 - eb);
      c_row = c8_pow2(eb - 139) * p.scale_log2;
#pragma unroll 4
      for (int c = 0; c < HD / 8; ++c) {
        const uint4 v = used ? src[c] : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          o[k] = pack_h2(__uint_as_float(w[k] << 16) * mul, __uint_as_float(w[k] & 0xffff0000u) * mul);
        *reinterpret_cast<uint4*>(s.q[t] + (c >> 3) * 16384 + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
            make_uint4(o[0], o[1], o[2], o[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.q_full);
    }
    float m_run = -INFINITY;      // running (possibly stale) maximum of the exponent, ev included
    float l_run = 0.f;
    bool ok = true;
    auto wait_pv = [&](int j) { return mbar_wait(&s.pv_done[t][j & 1], (j >> 1) & 1); };

    for (int jj = 0; jj < n_tiles && !s.abort; ++jj) {
      const int kv0 = (j_lo + jj) * BKV;
      const uint32_t sp_addr = s_addr + (jj & 1) * BKV;
      if (!mbar_wait(&s.sc_full[jj % SC_RING], (jj / SC_RING) & 1)) { ok = false; break; }
      float kf[4], lv[4], iv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 f = s.sc[jj % SC_RING][k];
        kf[k] = fmaxf(f.x * c_row, 1e-37f);              // stays positive: a masked score times it stays -inf
        lv[k] = f.y;
        iv[k] = f.z;
      }
      if (!mbar_wait(&s.s_full[t][jj & 1], (jj >> 1) & 1)) { ok = false; break; }
      tc_fence_after();
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
      if (lane == 0) mbar_arrive(&s.p_ready[t][jj & 1]);
    }
    if (ok && !s.abort) {
      if (!wait_pv(n_tiles - 1)) {
        ok = false;
      } else {
        tc_fence_after();
        const bool none = l_run == 0.f;                          // a row that sees nothing is a row of zeros
        const float inv = none ? 0.f : 1.0f / l_run;
        bf16* out = p.out + ((int64_t)x.row0 + i_row) * p.ldo + (int64_t)(x.h0 + row % x.heads) * HD;
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
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              uint4 w;
              w.x = pack_b2(__uint_as_float(o[v * 8 + 0]) * inv, __uint_as_float(o[v * 8 + 1]) * inv);
              w.y = pack_b2(__uint_as_float(o[v * 8 + 2]) * inv, __uint_as_float(o[v * 8 + 3]) * inv);
              w.z = pack_b2(__uint_as_float(o[v * 8 + 4]) * inv, __uint_as_float(o[v * 8 + 5]) * inv);
              w.w = pack_b2(__uint_as_float(o[v * 8 + 6]) * inv, __uint_as_float(o[v * 8 + 7]) * inv);
              *reinterpret_cast<uint4*>(out + c * 32 + v * 8) = w;
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
  if (warp == C::SM_WARPS + 4) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

// Merge of the pieces of split rows: one warp per row, grid as the attention kernel's without the splits.
template <int HD, int NQT>
__global__ void __launch_bounds__(256) attn8_merge_kernel(const __grid_constant__ A8Dev p, int* __restrict__ status) {
  chain_trigger();
  chain_wait();
  const int groups = NQT * 128 / 8;
  const int by = blockIdx.y / groups, r = (blockIdx.y % groups) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const Job x = job_of<NQT>(p, blockIdx.x, by, blockIdx.z, status);
  if (x.q0 < 0) return;
  const int in_tile = r & 127, i = x.q0 + (r >> 7) * x.per + in_tile / x.heads;
  if (in_tile >= x.per * x.heads || i >= x.n) return;
  constexpr int PER = HD / 32;
  float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) o[k] = 0.f;
  for (int sp = 0; sp < p.splits; ++sp) {
    const int64_t cta = ((int64_t)(blockIdx.z * p.splits + sp) * p.q_tiles + by) * gridDim.x + blockIdx.x;
    const float* src = p.partial + (cta * (NQT * 128) + r) * (HD + 4);
    const float ms = __ldcg(src), ls = __ldcg(src + 1);
    if (ms == -INFINITY) continue;                       // nothing seen there, its accumulator may not be written
    const float n = fmaxf(m, ms), fa = ex2(m - n), fb = ex2(ms - n);
    l = l * fa + ls * fb;
#pragma unroll
    for (int k = 0; k < PER; k += 2) {
      const float2 v = __ldcg(reinterpret_cast<const float2*>(src + 4 + lane * 2 + k * 32));
      o[k] = o[k] * fa + v.x * fb;
      o[k + 1] = o[k + 1] * fa + v.y * fb;
    }
    m = n;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;      // l 0: no piece was read, the sums are zeros
  bf16* dst = p.out + ((int64_t)x.row0 + i) * p.ldo + (int64_t)(x.h0 + in_tile % x.heads) * HD + lane * 2;
#pragma unroll
  for (int k = 0; k < PER; k += 2)
    *reinterpret_cast<__nv_bfloat162*>(dst + k * 32) = __floats2bfloat162_rn(o[k] * inv, o[k + 1] * inv);
}

template <int HD, int NQT>
int launch_t(const Attn8Args& a, A8Dev& p, cudaStream_t s) {
  using C = A8<HD, NQT>;
  const size_t smem = sizeof(A8Smem<HD, NQT>) + 1024;
  static_assert(sizeof(A8Smem<HD, NQT>) + 1024 <= kSmemLimit, "shared memory budget");
  const int per = 128 / (p.G < 128 ? p.G : 128);
  const int64_t q_tiles = ((int64_t)a.rows + NQT * per - 1) / (NQT * per);
  if (q_tiles > 65535) return POP_E_INVALID;
  p.q_tiles = (int)q_tiles;
  const int64_t base = (int64_t)a.n_kv * p.hg * q_tiles * a.batch;
  // fewer CTAs than SMs: split the keys, four 64-key tiles or more to a piece
  const int span = a.window > 0 && (int64_t)a.window + NQT * per < a.kv_len ? a.window + NQT * per : a.kv_len;
  int64_t splits = device_sms() / (base > 0 ? base : 1);
  const int64_t most = (span + 255) / 256;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  p.splits = (int)splits;
  if (splits > 1 && (size_t)(base * splits) * NQT * 128 * (HD + 4) * 4 > a.workspace_bytes) return POP_E_NOSPACE;
  if (a.batch * splits > 65535) return POP_E_INVALID;
  static bool configured = false;
  if (!configured) {
    if (cudaFuncSetAttribute(attn8_kernel<HD, NQT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
      return POP_E_CUDA;
    configured = true;
  }
  int* status = status_word();
  if (!status) return POP_E_CUDA;
  ProfScope prof(PROF_ATTENTION, 4.0 * HD * a.n_q * a.batch * (double)a.rows * (span - (a.window > 0 ? 0.0 : 0.5 * a.rows)), s);
  if (launch_chained(attn8_kernel<HD, NQT>, dim3(a.n_kv * p.hg, (unsigned)q_tiles, (unsigned)(a.batch * splits)),
                     dim3(C::THREADS), smem, s, p, status) != cudaSuccess)
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
      a.kv_len < 0 || a.kv_len > 0x7ffffff0 || a.window < 0 || a.window > 0x7ffffff0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8)
    return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.workspace) % 16 || (int64_t)a.batch * a.rows > 0x7fffffff) return POP_E_INVALID;
  if (!a.seq_lens && a.rows > a.kv_len) return POP_E_INVALID;
  if ((int64_t)a.kv_len > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  if (a.rows == 0) return POP_OK;
  A8Dev p{};
  p.q = a.q; p.ldq = a.ldq;
  p.c = a.c;
  p.ps_log2 = -1;
  for (int i = 4; i < 31; ++i)
    if (a.c.page_size == 1 << i) p.ps_log2 = i;
  p.cu = a.cu; p.rows = a.rows;
  p.seq_lens = a.seq_lens; p.kv_len = a.kv_len;
  p.out = a.out; p.ldo = a.ldo;
  p.n_q = a.n_q; p.n_kv = a.n_kv; p.G = a.n_q / a.n_kv; p.hg = (p.G + 127) / 128;
  p.window = a.window;
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
