// Attention of few query rows over the 8-bit paged cache (paper Eq. 1, Attn): the one position of a decode step, or a few
// drafted tokens at once.
//
// The queries of one kv head are columns: (row of the sequence, query head of that kv head). For column c at position pos_c
// and seen positions j in (pos_c - window, pos_c]:
//   out_c = sum_j p_j 2^(ev_j) v_j / sum_j p_j,   p_j = exp2(f q_c.k_j 2^(ek_j) - max),  f = log2(e) / sqrt(hd)
// with codes k_j, v_j and block exponents ek_j, ev_j. The V scale is folded into the exponent: with
// w_j = exp2(f q_c.k_j 2^(ek_j) + ev_j - m) and m the running maximum of that sum, out_c = sum w_j v_j / sum w_j 2^(-ev_j), so
// the weights that meet the tensor cores are at most 1 whatever the scales of the blocks are.
//
// Bound by the cache's bytes: 2 hd + 1/8 per kv head and position. A warp takes blocks of 16 positions of one item - a
// (sequence, kv head, group of at most 8 columns) - through its own small ring in shared memory (16-byte asynchronous
// copies; a block is one contiguous piece) and works on them with the warp-level MMA, the KEYS on the M side
// (S^T = K q^T, O^T = V^T P^T): a dot product does not see the order of its terms, so a lane's 16 consecutive bytes of a
// key feed the MMAs as they are. K codes meet the query as E4M3 operands: after a power-of-two scale per column an element
// is the sum of two codes, exactly for bf16 elements down to 2^-9 of the column's largest and to within 2^-17 of that
// below (half the smallest code). V codes become f16 exactly (two keys interleaved by a byte permute, one conversion per
// pair) and meet weights in f16 with 2^14 as the largest (half a step: 2^-11 relative); scores, statistics and sums are
// fp32. The 8-bit MMA runs at 3.5 times the f16 one's rate and needs no conversion.
//
// Who takes what:
//   - few items or short ones: a thread-block cluster of 1, 2, 4 or 8 CTAs per item, its blocks dealt to the warps in
//     equal stretches, the pieces merged in shared memory and over the cluster's. One launch.
//   - else all items form one line of blocks and every warp of a full GPU takes an equal stretch of it, whatever the
//     lengths are. An item that a warp has whole is finished by it; the pieces of the others go through the workspace to a
//     second, chained launch (a CTA that lies inside one item merges its eight in shared memory first).
// More than eight columns are several items, which read the same keys one after another from L2. (Two groups of columns
// per item, for one reading and conversion of the values, had one warp's registers full and were slower: five rows each of
// twelve sequences of up to 8000, 20 columns, 48.6 against 39.0 us.)
//
// Measured, hd 128, 32 heads over 8: 48 sequences of up to 16001 positions 142 us, 5.8 TB/s of the cache's bytes (0.88 of a
// copy's rate); one of 8192 11.1 us, where starting, one round through memory and merging are nearly all; hd 256, 20 windows
// of 1024 29.1 us: the blocks are read at the memory's rate in 11 us, the rest is the start (5.5 us: lengths, table, first
// blocks) and the second launch.
#include "../../include/pop_kernels.h"
#include "cache8.cuh"
#include "ptx.cuh"

namespace pop {
namespace {

constexpr uint32_t FULL = 0xffffffffu;
constexpr int WARPS = 8;
constexpr int MAX_BATCH = 4096;      // the block counts' prefix sums sit in shared memory
constexpr float W_SHIFT = 14.f;      // weights are stored times 2^14
constexpr int CLUSTER_BLOCKS = 16;   // one-launch form: blocks per warp at most

template <int HD>
struct D8 {
  static constexpr int NC = 8;                 // columns of an item: the N extent of an MMA
  static constexpr int NT = HD / 16;           // MMAs along the head
  static constexpr int KC = HD / 64;           // 16-byte pieces of a key row per lane
  static constexpr int VW = HD / 32;           // words of a value row per lane
  static constexpr int CH = HD / 16;           // 16-byte pieces of a row
  static constexpr int TILE = C8_BLOCK * HD;   // bytes of a block's keys; its values behind them
  // Blocks of one turn of the loop (their MMAs, exponentials and shuffles overlap, one maximum for all of them), and turns
  // in flight per warp: 192 KB per SM, two thirds of it always under way
  static constexpr int BPI = HD == 256 ? 1 : 2;
  static constexpr int NST = 3;
  static constexpr int STAGE = BPI * 2 * TILE;
  static constexpr int PER_SM = HD == 64 ? 2 : 1;
  static constexpr int HS = HD + 4;            // floats per column of a piece in shared memory: rows 4 banks apart
  static constexpr int SLOT = NC * HS + 2 * NC;         // m, l, then the sums
  static constexpr int PSLOT = NC * HD + 2 * NC;        // floats of a piece in the workspace
  static constexpr int RING = NST * STAGE;              // of a warp; a piece for the CTA's merge goes over the idle ring
  static constexpr int SMEM = WARPS * RING + SLOT * 4;  // and the CTA's merged piece, for its cluster
  static_assert(SLOT * 4 <= RING, "a piece goes over the ring");
  // two pieces of every warp: the stated workspace covers a GPU of up to 160 SMs
  static_assert(160 * PER_SM * WARPS * 2 * PSLOT * 4 <= POP_E4M3_WORKSPACE_BYTES, "workspace");
};

// Where 16-byte piece ch of row r of a block lies in its stage: permuted so that the eight lanes that read together (two
// keys at four pieces for K, four even or odd keys at two pieces for V) meet different banks.
template <int HD>
__device__ __forceinline__ int swz(int r, int ch) {
  const int f = HD == 64 ? (r >> 1) & 3 : (((r >> 1) & 3) << 1) ^ ((r & 1) << 2);
  return r * HD + ((ch ^ f) << 4);
}
// First of the two dims that tile j holds in lanes of group g: lanes read 8 (hd 64) or 16 bytes of a value row at once
template <int HD>
__device__ __forceinline__ int dim_of(int j, int g) {
  return HD == 64 ? g * 8 + 2 * j : (j >> 3) * 128 + g * 16 + (j & 7) * 2;
}

struct Dec8Dev {
  const bf16* q; int64_t ldq;
  Cache8 c;
  const int32_t* cu; int rows;       // query rows of each sequence (decode: one, row b)
  const int32_t* seq_lens; int kv_len, window;
  bf16* out; int64_t ldo;
  int batch, n_q, n_kv, G;
  int chunks;                        // column groups of a sequence with `rows` rows
  int cluster;                       // CTAs per item; 0: the line
  float* partial;                    // [warps][2][PSLOT]: the piece a warp begins with, and the one it ends with
  int* status;
  float scale_log2;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int src_bytes) {
  // src_bytes 0 writes 16 zero bytes and reads nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t movm_t(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// D[16x8] += A[16x32] . B[32x8], E4M3 operands, fp32 accumulate
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D[16x8] += A[16x16] . B[16x8], f16 operands, fp32 accumulate
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}


// Rows and seen positions of a sequence: blocks first .. first + n - 1 hold what its rows see
struct Seq { int row0, rows, len, lo, first, n, chunks; };
template <int NC>
__device__ __forceinline__ Seq seq_of(const Dec8Dev& p, int b) {
  Seq s;
  const int c0 = p.cu ? p.cu[b] : b * p.rows, c1 = p.cu ? p.cu[b + 1] : c0 + p.rows;
  s.len = p.seq_lens ? p.seq_lens[b] : p.kv_len;
  s.row0 = c0;
  s.rows = c1 - c0;
  if (s.len > p.kv_len || s.rows > p.rows) {    // more than the caller said: nothing past it is read
    s.len = min(s.len, p.kv_len);
    s.rows = min(s.rows, p.rows);
    atomicMin(p.status, (int)POP_E_INVALID);
  }
  s.len = max(s.len, 0);
  s.rows = max(s.rows, 0);
  s.chunks = s.rows == p.rows ? p.chunks : (s.rows * p.G + NC - 1) / NC;
  s.lo = p.window > 0 ? max(0, s.len - s.rows - p.window + 1) : 0;      // the first row's first
  s.first = s.lo / C8_BLOCK;
  s.n = s.chunks > 0 ? (s.len + C8_BLOCK - 1) / C8_BLOCK - s.first : 0;
  return s;
}

// Blocks of all items of the sequences before b. Up to 32 sequences: lane b of every warp knows its own, no shared memory;
// more: prefix[b] in shared memory, by all threads.
struct Prefix { int mine, total; const int* all; };
template <int NC>
__device__ __forceinline__ Prefix scan_blocks(const Dec8Dev& p, int* prefix, int* warp_sums) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto units = [&](int b) {
    const Seq s = seq_of<NC>(p, b);
    return s.n * s.chunks * p.n_kv;
  };
  Prefix x{0, 0, prefix};
  const bool small = p.batch <= 32;
  const int per = small ? 1 : (p.batch + blockDim.x - 1) / blockDim.x;
  const int b0 = min(p.batch, (small ? lane : (int)threadIdx.x) * per), b1 = min(p.batch, b0 + per);
  int sum = 0;
  for (int b = b0; b < b1; ++b) sum += units(b);
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(FULL, incl, o);
    if (lane >= o) incl += t;
  }
  if (small) {
    x.mine = incl - sum;
    x.total = __shfl_sync(FULL, incl, 31);
    return x;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int run = incl - sum;
  for (int w = 0; w < warp; ++w) run += warp_sums[w];
  for (int b = b0; b < b1; ++b) {
    prefix[b] = run;
    run += per == 1 ? sum : units(b);
  }
  if (b1 == p.batch && b0 < p.batch) prefix[p.batch] = run;
  __syncthreads();
  x.total = prefix[p.batch];
  return x;
}
// The line of all blocks, cut into W stretches that differ by at most one block (everything below 2^31: the host checks)
struct Line {
  int T, per, rest;
  __device__ __forceinline__ Line(int total, int W) {
    T = total;
    per = T / W;
    rest = T - per * W;
  }
  __device__ __forceinline__ int begin(int w) const { return w * per + min(w, rest); }
  __device__ __forceinline__ int owner(int u) const {      // the stretch that holds unit u
    const int big = rest * (per + 1);
    return u < big ? u / (per + 1) : rest + (u - big) / per;
  }
};
// Where unit u (< total) of the line lies: sequence, item of the sequence (kv head, column group), block of the item
struct Place { int b, kvh, chunk, blk; Seq s; };
template <int NC>
__device__ __forceinline__ Place locate(const Dec8Dev& p, const Prefix& pre, int u) {      // by whole warps
  Place x;
  int before;                                   // of the last b with prefix[b] <= u: it is not empty
  if (p.batch <= 32) {
    const int lane = threadIdx.x & 31;
    x.b = 31 - __clz(__ballot_sync(FULL, lane < p.batch && pre.mine <= u));
    before = __shfl_sync(FULL, pre.mine, x.b);
  } else {
    int lo = 0, hi = p.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (pre.all[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    x.b = lo;
    before = pre.all[lo];
  }
  x.s = seq_of<NC>(p, x.b);
  const int off = u - before, item = off / x.s.n;
  x.blk = off - item * x.s.n;
  x.kvh = item / x.s.chunks;
  x.chunk = item - x.kvh * x.s.chunks;
  return x;
}

template <int HD>
__global__ void __launch_bounds__(WARPS * 32, D8<HD>::PER_SM) dec8_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD>;
  constexpr int NC = C::NC, NT = C::NT, KC = C::KC, VW = C::VW, CH = C::CH, HS = C::HS, NST = C::NST, BPI = C::BPI;
  extern __shared__ __align__(128) uint8_t smem[];            // RING bytes of every warp, SLOT floats, the prefix sums
  __shared__ int warp_sums[WARPS];
  float* const xchg = reinterpret_cast<float*>(smem + WARPS * C::RING);
  int* const prefix = reinterpret_cast<int*>(xchg + C::SLOT);
  auto slot_of = [&](int w) { return reinterpret_cast<float*>(smem + w * C::RING); };     // the piece of warp w
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  chain_wait();
  chain_trigger();                   // after the wait: the merge reads the lengths before its own

  // this warp's stretch: places and count of blocks
  Place x;
  int left;                          // blocks of the stretch that are still to do
  int u = 0;                         // line form: the unit that x is at
  bool inside = false;               // line form: the CTA's stretch lies inside one item
  Prefix pre{};
  if (p.cluster) {
    const int item = blockIdx.x / p.cluster, rank = blockIdx.x - item * p.cluster;
    const int per_seq = p.n_kv * p.chunks;
    x.b = item / per_seq;
    const int in = item - x.b * per_seq;
    x.kvh = in / p.chunks;
    x.chunk = in - x.kvh * p.chunks;
    x.s = seq_of<NC>(p, x.b);
    const int w = rank * WARPS + warp, W = p.cluster * WARPS;
    x.blk = (int)((int64_t)x.s.n * w / W);
    left = x.chunk < x.s.chunks ? (int)((int64_t)x.s.n * (w + 1) / W) - x.blk : 0;
  } else {
    pre = scan_blocks<NC>(p, prefix, warp_sums);
    const Line line(pre.total, gridDim.x * WARPS);
    const int w = blockIdx.x * WARPS + warp;
    u = line.begin(w);
    left = line.begin(w + 1) - u;
    if (left > 0) x = locate<NC>(p, pre, u);
    if (left > 0) {                  // the same for all warps: an item that goes on behind the CTA leaves none without a block
      const int c0 = line.begin(blockIdx.x * WARPS), c1 = line.begin((blockIdx.x + 1) * WARPS), first = u - x.blk;
      inside = first < c0 && first + x.s.n > c1;
    }
  }
  // rows of sequences without a position: zeros
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const Seq s = seq_of<NC>(p, b);
    if (s.len == 0)
      for (int r = 0; r < s.rows; ++r)
        for (int e = threadIdx.x; e < p.n_q * HD; e += blockDim.x)
          p.out[(int64_t)(s.row0 + r) * p.ldo + e] = __float2bfloat16_rn(0.f);
  }

  uint8_t* const ring = smem + warp * C::RING;
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  const int ps = p.c.page_size;

  int stored = 0;                      // a piece of this warp is in shared memory
  while (left > 0) {
    const int n_blk = min(x.s.n - x.blk, left);
    const int col0 = x.chunk * NC, cols = min(NC, x.s.rows * p.G - col0), h0 = x.kvh * p.G;
    const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;

    // the query rows' loads go out first: a lane takes column g at dims 64 c + 16 t .. + 15
    uint4 raw[KC][2];
    const int col = col0 + g;
    const bool live = g < cols;
    const int row_of_col = live ? col / p.G : 0, h = live ? col - row_of_col * p.G : 0;
    const bf16* qrow = p.q + (int64_t)(x.s.row0 + row_of_col) * p.ldq + (int64_t)(h0 + h) * HD + 16 * t;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      raw[c][0] = *reinterpret_cast<const uint4*>(qrow + 64 * c);
      raw[c][1] = *reinterpret_cast<const uint4*>(qrow + 64 * c + 8);
    }

    // Places and scales of 32 blocks at a time, one per lane: block number in the pool (-1, read as zeros, for a table
    // entry that is no page of it) and both scale bytes
    auto fetch = [&](int i, int& id, int& sc) {
      id = -1;
      sc = 127 | 127 << 8;
      if (i + lane < n_blk) {
        const int pos = (x.s.first + x.blk + i + lane) * C8_BLOCK, pi = pos / ps, page = bt[pi];
        if ((unsigned)page < (unsigned)p.c.num_pages) {
          id = (page * p.n_kv + x.kvh) * (ps / C8_BLOCK) + (pos - pi * ps) / C8_BLOCK;
          sc = p.c.ks[id] | p.c.vs[id] << 8;
        } else {
          atomicMin(p.status, (int)POP_E_INVALID);
        }
      }
    };
    int base = 0, id_c, sc_c, id_n = -1, sc_n = 0;     // the 32 blocks from `base` on, and the 32 behind them
    fetch(0, id_c, sc_c);
    if (n_blk > 32) fetch(32, id_n, sc_n);
    auto issue = [&](int i, int stage) {               // blocks i .. i + BPI - 1; one that is not there reads as zeros
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        const int k = i + u2 - base, id = __shfl_sync(FULL, k < 32 ? id_c : id_n, k & 31);
        const int64_t off = id < 0 ? 0 : (int64_t)id * C::TILE;
        const int bytes = id < 0 ? 0 : 16;
        const uint32_t dst = ring_addr + stage * C::STAGE + u2 * 2 * C::TILE;
        const uint8_t *ks = p.c.k + off + lane * 16, *vs = p.c.v + off + lane * 16;
#pragma unroll
        for (int c = 0; c < C::TILE / 512; ++c) {
          const int e = c * 32 + lane;
          const uint32_t at = dst + swz<HD>(e / CH, e % CH);
          cp_async16(at, ks + c * 512, bytes);
          cp_async16(at + C::TILE, vs + c * 512, bytes);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (i * BPI < n_blk) issue(i * BPI, i);
      cp_async_commit();
    }

    // q^T as the B operand: a lane holds column g at dims 64 c + 16 t + 4 w .. + 3, scaled so that the
    // column's largest element is in [2^7, 2^8), as two codes: the nearest one and the nearest one of what is left.
    // Per column of this lane's scores (2t and 2t + 1): factor and position.
    uint32_t qh[KC][4], ql[KC][4];
    float am = 0.f;
    auto lo_f = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi_f = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t w[4] = {raw[c][k].x, raw[c][k].y, raw[c][k].z, raw[c][k].w};
#pragma unroll
        for (int m = 0; m < 4; ++m) am = fmaxf(am, fmaxf(fabsf(lo_f(w[m])), fabsf(hi_f(w[m]))));
      }
    am = fmaxf(am, __shfl_xor_sync(FULL, am, 1));
    am = fmaxf(am, __shfl_xor_sync(FULL, am, 2));
    const int eb = max((int)(__float_as_uint(am) >> 23), 20);
    // an infinite element makes the column NaN, as its softmax is
    const float mul = !live ? 0.f : eb == 255 ? NAN : c8_pow2(134 - eb), inv = c8_pow2(eb - 134) * p.scale_log2;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4& r = raw[c][k >> 1];
        const uint32_t w0 = (k & 1) ? r.z : r.x, w1 = (k & 1) ? r.w : r.y;
        const float e0 = lo_f(w0) * mul, e1 = hi_f(w0) * mul, e2 = lo_f(w1) * mul, e3 = hi_f(w1) * mul;
        const uint32_t hi = c8_codes4(e0, e1, e2, e3), f0 = c8_half2_lo(hi), f1 = c8_half2_hi(hi);
        const float2 r0 = __half22float2(*reinterpret_cast<const __half2*>(&f0));
        const float2 r1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
        qh[c][k] = hi;
        ql[c][k] = c8_codes4(e0 - r0.x, e1 - r0.y, e2 - r1.x, e3 - r1.y);
      }
    }
    const float c0 = __shfl_sync(FULL, inv, t * 8), c1 = __shfl_sync(FULL, inv, t * 8 + 4);
    const int pos = x.s.len - x.s.rows + row_of_col;
    const int pos0 = __shfl_sync(FULL, pos, t * 8), pos1 = __shfl_sync(FULL, pos, t * 8 + 4);
    // blocks up to key full_hi need no causal mask, from key full_lo on no window mask
    const int first_row = col0 / p.G, last_row = (col0 + cols - 1) / p.G;
    const int full_hi = x.s.len - x.s.rows + first_row;
    const int full_lo = p.window > 0 ? x.s.len - x.s.rows + last_row - p.window + 1 : 0;

    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f, o[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

    int stage = 0;
    for (int i = 0; i < n_blk; i += BPI) {
      const int at = (x.s.first + x.blk + i) * C8_BLOCK;       // first position of the first block
      cp_async_wait<NST - 1>();
      __syncwarp();
      if (i - base == 32) {
        base = i;
        id_c = id_n;
        sc_c = sc_n;
        if (i + 32 < n_blk) fetch(i + 32, id_n, sc_n);
      }
      const uint8_t* st = ring + stage * C::STAGE;
      float s[BPI][4];
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        float sb[4];                   // s and sb: of the two codes of q
#pragma unroll
        for (int k = 0; k < 4; ++k) s[u2][k] = sb[k] = 0.f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {                         // keys g and g + 8 at bytes 64 c + 16 t .. + 15
          const uint4 ka = *reinterpret_cast<const uint4*>(st + u2 * 2 * C::TILE + swz<HD>(g, 4 * c + t));
          const uint4 kb = *reinterpret_cast<const uint4*>(st + u2 * 2 * C::TILE + swz<HD>(g + 8, 4 * c + t));
          mma_e4m3(s[u2], ka.x, kb.x, ka.y, kb.y, qh[c][0], qh[c][1]);
          mma_e4m3(sb, ka.x, kb.x, ka.y, kb.y, ql[c][0], ql[c][1]);
          mma_e4m3(s[u2], ka.z, kb.z, ka.w, kb.w, qh[c][2], qh[c][3]);
          mma_e4m3(sb, ka.z, kb.z, ka.w, kb.w, ql[c][2], ql[c][3]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) s[u2][k] += sb[k];
      }
      float kf[BPI], lv[BPI], inv_v[BPI];
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        const int sc = __shfl_sync(FULL, sc_c, i + u2 - base), ke = sc & 255, ve = sc >> 8;
        kf[u2] = c8_pow2(ke - 127);
        lv[u2] = (float)(ve - 127);
        inv_v[u2] = c8_pow2(127 - ve);
      }
      const bool edge = at + BPI * C8_BLOCK - 1 > full_hi || at < full_lo || i + BPI > n_blk;
      const int end = (x.s.first + x.blk + n_blk) * C8_BLOCK;  // of this stretch: the blocks behind it are not its own
      uint32_t pb[BPI][2];
      float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        float* v = s[u2];
        const float k0 = c0 * kf[u2], k1 = c1 * kf[u2];
        v[0] = fmaf(v[0], k0, lv[u2]);
        v[1] = fmaf(v[1], k1, lv[u2]);
        v[2] = fmaf(v[2], k0, lv[u2]);
        v[3] = fmaf(v[3], k1, lv[u2]);
        if (edge) {                    // keys that a column does not see: no weight whatever is there
          const int a = at + u2 * C8_BLOCK + g, h0c = min(pos0, end - 1), h1c = min(pos1, end - 1);
          const int w0 = p.window > 0 ? pos0 - p.window : -1, w1 = p.window > 0 ? pos1 - p.window : -1;
          if (a > h0c || a <= w0) v[0] = -INFINITY;
          if (a > h1c || a <= w1) v[1] = -INFINITY;
          if (a + 8 > h0c || a + 8 <= w0) v[2] = -INFINITY;
          if (a + 8 > h1c || a + 8 <= w1) v[3] = -INFINITY;
        }
        x0 = fmaxf(x0, fmaxf(v[0], v[2]));
        x1 = fmaxf(x1, fmaxf(v[1], v[3]));
      }
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        x0 = fmaxf(x0, __shfl_xor_sync(FULL, x0, w));
        x1 = fmaxf(x1, __shfl_xor_sync(FULL, x1, w));
      }
      const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
      // a column that has seen nothing yet keeps its maximum of -inf and weights of 0
      const float b0 = n0 == -INFINITY ? 0.f : n0, b1 = n1 == -INFINITY ? 0.f : n1;
      const float f0 = ex2(m0 - b0), f1 = ex2(m1 - b1);
      const float e0 = b0 - W_SHIFT, e1 = b1 - W_SHIFT;
      l0 *= f0;
      l1 *= f1;
      m0 = n0;
      m1 = n1;
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        const float* v = s[u2];
        const float p0 = ex2(v[0] - e0), p1 = ex2(v[1] - e1), p2 = ex2(v[2] - e0), p3 = ex2(v[3] - e1);
        l0 = fmaf(p0 + p2, inv_v[u2], l0);
        l1 = fmaf(p1 + p3, inv_v[u2], l1);
        pb[u2][0] = movm_t(pack_half2(p0, p1));          // keys 0-7 of the block
        pb[u2][1] = movm_t(pack_half2(p2, p3));          // keys 8-15
      }
      if (__any_sync(FULL, f0 != 1.f || f1 != 1.f)) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          o[j][0] *= f0; o[j][1] *= f1; o[j][2] *= f0; o[j][3] *= f1;
        }
      }
#pragma unroll
      for (int u2 = 0; u2 < BPI; ++u2) {
        const uint8_t* sv = st + (u2 * 2 + 1) * C::TILE;
        uint32_t vr[4][VW];            // values of keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 2 * t + (k & 1) + (k >> 1) * 8;
          if constexpr (HD == 64) {
            const uint2 v = *reinterpret_cast<const uint2*>(sv + swz<HD>(r, g >> 1) + (g & 1) * 8);
            vr[k][0] = v.x; vr[k][1] = v.y;
          } else {
#pragma unroll
            for (int c = 0; c < VW / 4; ++c) {
              const uint4 v = *reinterpret_cast<const uint4*>(sv + swz<HD>(r, 8 * c + g));
              vr[k][4 * c] = v.x; vr[k][4 * c + 1] = v.y; vr[k][4 * c + 2] = v.z; vr[k][4 * c + 3] = v.w;
            }
          }
        }
        // behind the sequence, or in front of every row's window: no value whatever is there
        if (at + (u2 + 1) * C8_BLOCK > x.s.len || at + u2 * C8_BLOCK < x.s.lo) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int a = at + u2 * C8_BLOCK + 2 * t + (k & 1) + (k >> 1) * 8;
            if (a >= x.s.len || a < x.s.lo) {
#pragma unroll
              for (int w = 0; w < VW; ++w) vr[k][w] = 0;
            }
          }
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
          const uint32_t a = __byte_perm(vr[0][w], vr[1][w], 0x5140), b = __byte_perm(vr[0][w], vr[1][w], 0x7362);
          const uint32_t c = __byte_perm(vr[2][w], vr[3][w], 0x5140), d = __byte_perm(vr[2][w], vr[3][w], 0x7362);
          const uint32_t a0 = c8_half2_lo(a), a1 = c8_half2_hi(a), a2 = c8_half2_lo(c), a3 = c8_half2_hi(c);
          const uint32_t b0 = c8_half2_lo(b), b1 = c8_half2_hi(b), b2 = c8_half2_lo(d), b3 = c8_half2_hi(d);
          mma_f16(o[2 * w], a0, a1, a2, a3, pb[u2][0], pb[u2][1]);
          mma_f16(o[2 * w + 1], b0, b1, b2, b3, pb[u2][0], pb[u2][1]);
        }
      }
      __syncwarp();                    // every lane is done with the stage
      if (i + NST * BPI < n_blk) issue(i + NST * BPI, stage);
      cp_async_commit();
      stage = stage + 1 == NST ? 0 : stage + 1;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      l0 += __shfl_xor_sync(FULL, l0, w);
      l1 += __shfl_xor_sync(FULL, l1, w);
    }
    // lane (g, t) holds columns 2t ([0], [2]) and 2t + 1 ([1], [3]) at dims dim_of(j, g) and the one behind it
    const bool starts = x.blk == 0, ends = x.blk + n_blk == x.s.n;
    if (starts && ends && !p.cluster) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int k = 2 * t + hh;
        if (k >= cols) continue;
        const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
        const float l = hh ? l1 : l0, inv = l == 0.f ? 0.f : 1.f / l;
        bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(h0 + h) * HD;
#pragma unroll
        for (int j = 0; j < NT; ++j)
          *reinterpret_cast<__nv_bfloat162*>(dst + dim_of<HD>(j, g)) =
              __floats2bfloat162_rn(o[j][hh] * inv, o[j][2 + hh] * inv);
      }
    } else {
      // for the CTA's merge over the ring, which every lane has left; else to the workspace
      const bool local = p.cluster || inside;
      const int cs = local ? HS : HD;                          // floats per column
      float* sl = local ? slot_of(warp)
                        : p.partial + (((int64_t)blockIdx.x * WARPS + warp) * 2 + (starts ? 1 : 0)) * C::PSLOT;
      stored = local;
      __syncwarp();
      if (g == 0) {
        sl[2 * t] = m0; sl[2 * t + 1] = m1;
        sl[NC + 2 * t] = l0; sl[NC + 2 * t + 1] = l1;
      }
      float* so = sl + 2 * NC + 2 * t * cs + 2 * g;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<float2*>(so + 16 * j) = make_float2(o[j][0], o[j][2]);
        *reinterpret_cast<float2*>(so + cs + 16 * j) = make_float2(o[j][1], o[j][3]);
      }
    }
    left -= n_blk;
    if (left > 0) {                    // the line goes on with the next item
      u += n_blk;
      x = locate<NC>(p, pre, u);
    }
  }
  if (!p.cluster && !inside) return;
  // The CTA's pieces of its one item, by tasks of one column and 32 pairs of dims; lane k < 8 knows the piece of warp k. A
  // warp without a block leaves an empty piece.
  if (!stored) {
    float* sl = slot_of(warp);
    for (int e = lane; e < C::SLOT; e += 32) sl[e] = e < NC ? -INFINITY : 0.f;
  }
  __syncthreads();
  const bool has = lane < WARPS;
  const int col0 = x.chunk * NC, cols = x.s.len == 0 ? 0 : min(NC, x.s.rows * p.G - col0);
  constexpr int PARTS = HD / 64;       // tasks per column
  for (int task = warp; task < cols * PARTS; task += WARPS) {
    const int k = task / PARTS, pr = (task - k * PARTS) * 32 + lane;       // pair pr: dims dim_of(pr / 8, pr % 8) and the next
    const float mk = has ? slot_of(lane)[k] : -INFINITY;
    float m = mk;
#pragma unroll
    for (int w = 4; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, w));
    m = __shfl_sync(FULL, m, 0);       // lanes 8 .. 31 hold no piece
    const float f = mk == -INFINITY ? 0.f : ex2(mk - m);
    float l = has ? slot_of(lane)[NC + k] * f : 0.f;
#pragma unroll
    for (int w = 4; w > 0; w >>= 1) l += __shfl_xor_sync(FULL, l, w);
    l = __shfl_sync(FULL, l, 0);
    float2 v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float fk = __shfl_sync(FULL, f, w);
      const float2 ov = *reinterpret_cast<const float2*>(slot_of(w) + 2 * NC + k * HS + 2 * pr);
      v.x = fmaf(ov.x, fk, v.x);
      v.y = fmaf(ov.y, fk, v.y);
    }
    if (p.cluster == 1) {
      const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(x.kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
      *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
    } else {                           // for the cluster; or as the piece of the CTA's first warp
      float* dst = p.cluster ? xchg : p.partial + (int64_t)blockIdx.x * WARPS * 2 * C::PSLOT;
      *reinterpret_cast<float2*>(dst + 2 * NC + k * (p.cluster ? HS : HD) + 2 * pr) = v;
      if (pr == 0) {
        dst[k] = m;
        dst[NC + k] = l;
      }
    }
  }
  if (p.cluster > 1) {
    // every CTA of the cluster finishes a share of the item's pairs from all the CTAs' pieces
    cluster_arrive();
    cluster_wait();
    const int rank = (int)cluster_ctarank();
    const uint32_t xa = smem_u32(xchg);
    for (int e = rank * WARPS * 32 + threadIdx.x; e < cols * (HD / 2); e += p.cluster * WARPS * 32) {
      const int k = e / (HD / 2), pr = e - k * (HD / 2);
      float mr[8], lr[8], vx[8], vy[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        mr[r] = -INFINITY;
        lr[r] = vx[r] = vy[r] = 0.f;
        if (r < p.cluster) {
          const uint32_t a = mapa_u32(xa, (uint32_t)r);
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(mr[r]) : "r"(a + 4u * k));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(lr[r]) : "r"(a + 4u * (NC + k)));
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];"
                       : "=f"(vx[r]), "=f"(vy[r]) : "r"(a + 4u * (2 * NC + k * HS + 2 * pr)));
        }
      }
      float m = -INFINITY, l = 0.f, ox = 0.f, oy = 0.f;
#pragma unroll
      for (int r = 0; r < 8; ++r) m = fmaxf(m, mr[r]);
#pragma unroll
      for (int r = 0; r < 8; ++r)
        {
          const float f = mr[r] == -INFINITY ? 0.f : ex2(mr[r] - m);
          l = fmaf(lr[r], f, l);
          ox = fmaf(vx[r], f, ox);
          oy = fmaf(vy[r], f, oy);
        }
      const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(x.kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
      *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(ox * inv, oy * inv);
    }
    // nobody leaves while a neighbour may still read its shared memory
    cluster_arrive();
    cluster_wait();
  }
}

// Items that several warps have pieces of. Block w of this grid is for the border between warps w - 1 and w: if it lies
// inside an item, the blocks of all the borders inside it share its elements out. Reads the same lengths as the attention
// kernel, so it finds the same places. With few pieces every lane takes a pair of dims; with many, four neighbouring pairs (a
// 32-byte sector) go to four lanes, eight pieces at a time.
constexpr int MERGE_WARPS = 4;
template <int HD>
__global__ void __launch_bounds__(MERGE_WARPS * 32) dec8_merge_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD>;
  constexpr int NC = C::NC;
  extern __shared__ __align__(16) int prefix[];
  __shared__ int warp_sums[WARPS];
  chain_trigger();
  // this kernel starts behind the attention kernel's wait, so the lengths are there; only the pieces have to be waited for
  const Prefix pre = scan_blocks<NC>(p, prefix, warp_sums);
  const Line line(pre.total, gridDim.x);
  const int w = blockIdx.x, u = line.begin(w);
  Place x{};
  if (u < line.T) x = locate<NC>(p, pre, u);
  chain_wait();
  if (u >= line.T || x.blk == 0) return;       // behind the line's end, or the border is one between items
  const int first = u - x.blk, w0 = line.owner(first), w1 = line.owner(first + x.s.n - 1);
  // pieces: of the warps of the first CTA, of the CTAs inside the item (one each), of the warps of the last CTA
  const int q0 = w0 / WARPS, q1 = w1 / WARPS;
  const int n0 = min(w1, q0 * WARPS + WARPS - 1) - w0 + 1, n1 = max(0, q1 - q0 - 1), n = n0 + n1 + (q1 > q0 ? w1 - q1 * WARPS + 1 : 0);
  auto piece = [&](int i) {
    const int pw = i < n0 ? w0 + i : i < n0 + n1 ? (q0 + 1 + i - n0) * WARPS : q1 * WARPS + i - n0 - n1;
    return p.partial + ((int64_t)pw * 2 + (pw == w0 ? 1 : 0)) * C::PSLOT;
  };
  const int col0 = x.chunk * NC, cols = min(NC, x.s.rows * p.G - col0);
  const int lane = threadIdx.x & 31;
  const int rank = (w - w0 - 1) * MERGE_WARPS + (threadIdx.x >> 5), workers = (w1 - w0) * MERGE_WARPS;
  float m = -INFINITY, l = 0.f;
  float2 v = make_float2(0.f, 0.f);
  auto add = [&](int i, int k, int pr) {
    const float* sl = piece(i);
    const float mk = __ldcg(sl + k), lk = __ldcg(sl + NC + k);
    const float2 ov = __ldcg(reinterpret_cast<const float2*>(sl + 2 * NC + k * HD + 2 * pr));
    const float mx = fmaxf(m, mk), z = mx == -INFINITY ? 0.f : mx, fa = ex2(m - z), fb = ex2(mk - z);
    l = l * fa + lk * fb;
    v.x = v.x * fa + ov.x * fb;
    v.y = v.y * fa + ov.y * fb;
    m = mx;
  };
  auto finish = [&](int k, int pr) {
    const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(x.kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
    *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
  };
  if (n <= 24) {
    for (int task = rank; task < cols * (HD / 64); task += workers) {
      const int k = task / (HD / 64), pr = (task - k * (HD / 64)) * 32 + lane;
      m = -INFINITY;
      l = v.x = v.y = 0.f;
#pragma unroll 8
      for (int i = 0; i < n; ++i) add(i, k, pr);
      finish(k, pr);
    }
    return;
  }
  const int pk = lane >> 2, pe = lane & 3;
  for (int quad = rank; quad < cols * (HD / 8); quad += workers) {
    const int k = quad / (HD / 8), pr = (quad - k * (HD / 8)) * 4 + pe;
    m = -INFINITY;
    l = v.x = v.y = 0.f;
#pragma unroll 4
    for (int i = pk; i < n; i += 8) add(i, k, pr);
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      const float mk = __shfl_xor_sync(FULL, m, d), lk = __shfl_xor_sync(FULL, l, d);
      const float ox = __shfl_xor_sync(FULL, v.x, d), oy = __shfl_xor_sync(FULL, v.y, d);
      const float mx = fmaxf(m, mk), z = mx == -INFINITY ? 0.f : mx, fa = ex2(m - z), fb = ex2(mk - z);
      l = l * fa + lk * fb;
      v.x = v.x * fa + ox * fb;
      v.y = v.y * fa + oy * fb;
      m = mx;
    }
    if (pk == 0) finish(k, pr);
  }
}

// Clusters of n CTAs that the GPU holds at once (of the device that was current at the first call): fewer than its SMs
// would give, since a cluster lies within one group of SMs
template <int HD>
int max_clusters(int n) {
  using C = D8<HD>;
  static std::atomic<int> known[9];
  int most = known[n].load(std::memory_order_relaxed);
  if (most > 0) return most - 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n);
  cfg.blockDim = dim3(WARPS * 32);
  cfg.dynamicSmemBytes = C::SMEM;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = n;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&most, dec8_kernel<HD>, &cfg) != cudaSuccess) {
    cudaGetLastError();                          // no GPU: no clusters
    return 0;
  }
  known[n].store(most + 1, std::memory_order_relaxed);
  return most;
}

template <int HD>
int launch_t(const Attn8Args& a, Dec8Dev& p, cudaStream_t s) {
  using C = D8<HD>;
  p.chunks = (int)(((int64_t)a.rows * p.G + C::NC - 1) / C::NC);
  const int span = p.window > 0 && (int64_t)p.window + a.rows + C8_BLOCK < a.kv_len ? p.window + a.rows + C8_BLOCK : a.kv_len;
  const int64_t blocks = ((int64_t)span + C8_BLOCK - 1) / C8_BLOCK, items = (int64_t)a.batch * a.n_kv * p.chunks;
  // block numbers, of the call and of the pool, are 32-bit
  if (blocks > 0x7fffffff / (items + 1) ||
      (int64_t)a.c.num_pages * a.n_kv > 0x7fffffff / (a.c.page_size / C8_BLOCK))
    return POP_E_INVALID;
  const int ctas = device_sms() * C::PER_SM;
  static std::atomic<uint64_t> configured{0};
  const bool ready =                             // asked before the clusters are; counts when the kernel is launched
      c8_allow_smem(configured, reinterpret_cast<const void*>(dec8_kernel<HD>), C::SMEM + (MAX_BATCH + 1) * 4);
  // One launch, a CTA or a cluster per item, where no warp gets more than CLUSTER_BLOCKS blocks and the CTAs are resident
  // at once; two rounds of CTAs pay up to eight blocks per warp, any number up to four. Against the line and its second
  // launch, hd 128, 8 kv heads (us): 1 x 8192 positions 11.1 / 14.5, 1 x 2000 7.0 / 14.2, 9 x 2000 13.0 / 21.2, 18 x 1000 12.2
  // / 19.9, 18 x 2000 17.8 / 26.1; two rounds 20 x 1000 19.7 / 20.0 (unequal lengths 13.0 / 16.4), 30 x 1000 21.6 / 23.3, but 20 x
  // 2000 29.7 / 27.2. And 2 x 8192 in clusters of 8, which are not all resident, 21.2 against 16.5 in those of 4.
  int cs = 1;
  while (cs < 8 && blocks > (int64_t)cs * WARPS * 2 && items <= max_clusters<HD>(cs * 2)) cs *= 2;
  const bool one_launch = cs > 1 || items <= ctas || blocks <= WARPS * 4 || (items <= 2 * ctas && blocks <= WARPS * 8);
  p.cluster = one_launch && blocks <= (int64_t)cs * WARPS * CLUSTER_BLOCKS ? cs : 0;
  int64_t grid = items * cs;
  if (!p.cluster) {
    if (a.batch > MAX_BATCH) return POP_E_INVALID;
    grid = ctas;
    const int64_t most = (blocks * items + WARPS - 1) / WARPS;    // no fewer than one block per warp
    if (grid > most) grid = most;
    if ((size_t)grid * WARPS * 2 * C::PSLOT * 4 > a.workspace_bytes) return POP_E_NOSPACE;
  }
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  if (!ready) return POP_E_CUDA;
  const int scan_bytes = p.cluster ? 0 : (a.batch + 1) * 4;
  ProfScope prof(PROF_DECODE_ATTN, (double)a.batch * span * a.n_kv * (2.0 * HD + 0.125), s);
  const size_t smem = (size_t)(C::SMEM + scan_bytes);
  const cudaError_t rc = p.cluster > 1
                             ? launch_chained_cluster_x(dec8_kernel<HD>, dim3((unsigned)grid), dim3(WARPS * 32), smem, s,
                                                        (unsigned)p.cluster, p)
                             : launch_chained(dec8_kernel<HD>, dim3((unsigned)grid), dim3(WARPS * 32), smem, s, p);
  if (rc != cudaSuccess) return POP_E_CUDA;
  count_launch();
  if (!p.cluster) {
    if (launch_chained(dec8_merge_kernel<HD>, dim3((unsigned)grid * WARPS), dim3(MERGE_WARPS * 32), (size_t)scan_bytes, s, p) !=
        cudaSuccess)
      return POP_E_CUDA;
    count_launch();
  }
  return POP_OK;
}

}  // namespace

int launch_few8(const Attn8Args& a, cudaStream_t s) {
  Dec8Dev p{};
  p.q = a.q; p.ldq = a.ldq;
  p.c = a.c;
  p.cu = a.cu; p.rows = a.rows;
  p.seq_lens = a.seq_lens; p.kv_len = a.kv_len;
  p.window = a.window < a.kv_len ? a.window : 0;         // a longer one hides nothing
  p.out = a.out; p.ldo = a.ldo;
  p.batch = a.batch; p.n_q = a.n_q; p.n_kv = a.n_kv; p.G = a.n_q / a.n_kv;
  p.partial = static_cast<float*>(a.workspace);
  p.scale_log2 = 1.4426950408889634f / sqrtf((float)a.head_dim);
  switch (a.head_dim) {
    case 64: return launch_t<64>(a, p, s);
    case 128: return launch_t<128>(a, p, s);
    default: return launch_t<256>(a, p, s);
  }
}

int launch_decode_attention8(const Attn8Args& a, cudaStream_t s) {
  if (!a.q || !a.out || !c8_cache_ok(a.c)) return POP_E_INVALID;
  if (a.batch < 1 || a.batch > MAX_BATCH || a.n_kv < 1 || a.n_q < 1 || a.n_q % a.n_kv || a.n_q > 65536 || a.kv_len < 0 ||
      a.kv_len > 0x7fff0000 || a.window < 0 || a.window > 0x7ffffff0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8 ||
      reinterpret_cast<uintptr_t>(a.workspace) % 16)
    return POP_E_INVALID;
  if (a.batch > 1 && a.ldo < (int64_t)a.n_q * a.head_dim) return POP_E_INVALID;       // rows over each other
  if ((int64_t)a.kv_len > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  return launch_few8(a, s);
}

}  // namespace pop
