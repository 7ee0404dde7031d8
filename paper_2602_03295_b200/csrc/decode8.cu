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
// (sequence, kv head, group of at most 8 CG columns) - through its own small ring in shared memory (16-byte asynchronous
// copies; a block is one contiguous piece) and works on them with the warp-level MMA, the KEYS on the M side
// (S^T = K q^T, O^T = V^T P^T): a dot product does not see the order of its terms, so a lane's 16 consecutive bytes of a
// key feed the MMAs as they are. K codes meet the query as E4M3 operands: after a power-of-two scale per column an element
// is the sum of two codes, exactly for bf16 elements down to 2^-9 of the column's largest and to within 2^-17 of that
// below (half the smallest code). V codes become f16 exactly (two keys interleaved by a byte permute, one conversion per
// pair) and meet weights in f16 with 2^14 as the largest (half a step: 2^-11 relative); scores, statistics and sums are
// fp32. The 8-bit MMA runs at 3.5 times the f16 one's rate and needs no conversion.
//
// Who takes what:
//   - few items (a small batch): a thread-block cluster of 1, 2, 4 or 8 CTAs per item, its blocks dealt to the warps in
//     equal stretches, the pieces merged in shared memory and over the cluster's. One launch.
//   - else all items form one line of blocks and every warp of a full GPU takes an equal stretch of it, whatever the
//     lengths are. An item that a warp has whole is finished by it; pieces of one CTA are merged in shared memory, items
//     that cross CTAs through the workspace by a second, chained launch.
#include "cache8.cuh"
#include "ptx.cuh"

namespace pop {
namespace {

constexpr uint32_t FULL = 0xffffffffu;
constexpr int WARPS = 8;
constexpr int MAX_BATCH = 4096;      // the block counts' prefix sums sit in shared memory
constexpr float W_SHIFT = 14.f;      // weights are stored times 2^14
constexpr int CLUSTER_BLOCKS = 16;   // cluster form: blocks per warp at most

template <int HD, int CG>
struct D8 {
  static constexpr int NC = 8 * CG;            // columns of an item: the N extent of CG MMAs
  static constexpr int NT = HD / 16;           // MMAs along the head
  static constexpr int KC = HD / 64;           // 16-byte pieces of a key row per lane
  static constexpr int VW = HD / 32;           // words of a value row per lane
  static constexpr int CH = HD / 16;           // 16-byte pieces of a row
  static constexpr int TILE = C8_BLOCK * HD;   // bytes of a block's keys; its values behind them
  static constexpr int PER_SM = CG > 1 ? 1 : (HD == 64 ? 3 : (HD == 128 ? 2 : 1));
  static constexpr int NST = CG > 1 ? 3 : (HD == 64 ? 3 : 2);   // blocks in flight per warp: 96 KB and more per SM
  static constexpr int HS = HD + 4;            // floats per column of a piece in shared memory: rows 4 banks apart
  static constexpr int SLOT = NC * HS + 2 * NC;         // m, l, then the sums
  static constexpr int PSLOT = NC * HD + 2 * NC;        // floats of a piece in the workspace
  // a warp's memory: ring, the piece it begins with (the one it ends with goes over the idle ring), queries if CG > 1
  static constexpr int RING = NST * 2 * TILE;
  static constexpr int QB = CG > 1 ? CG * KC * 2 * 512 : 0;
  static constexpr int WARP_BYTES = RING + SLOT * 4 + QB;
  static constexpr int SMEM = WARPS * WARP_BYTES + SLOT * 4;    // and the CTA's merged piece, for its cluster
  static_assert(SLOT * 4 <= RING, "the last piece goes over the ring");
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
  float* partial;                    // [CTAs][2][PSLOT]
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

// prefix[b] = blocks of all items of the sequences before b, for b <= batch. By all threads.
template <int NC>
__device__ __forceinline__ void scan_blocks(const Dec8Dev& p, int* prefix, int* warp_sums) {
  const int per = (p.batch + blockDim.x - 1) / blockDim.x;
  const int b0 = min(p.batch, (int)threadIdx.x * per), b1 = min(p.batch, b0 + per);
  auto units = [&](int b) {
    const Seq s = seq_of<NC>(p, b);
    return s.n * s.chunks * p.n_kv;
  };
  int sum = 0;
  for (int b = b0; b < b1; ++b) sum += units(b);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(FULL, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int run = incl - sum;
  for (int w = 0; w < warp; ++w) run += warp_sums[w];
  for (int b = b0; b < b1; ++b) {
    prefix[b] = run;
    run += b + 1 == b1 && per == 1 ? sum : units(b);
  }
  if (b1 == p.batch && b0 < p.batch) prefix[p.batch] = run;
  __syncthreads();
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
__device__ __forceinline__ Place locate(const Dec8Dev& p, const int* prefix, int u) {
  Place x;
  int lo = 0, hi = p.batch - 1;                 // the last b with prefix[b] <= u: it is not empty
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  x.b = lo;
  x.s = seq_of<NC>(p, lo);
  const int off = u - prefix[lo], item = off / x.s.n;
  x.blk = off - item * x.s.n;
  x.kvh = item / x.s.chunks;
  x.chunk = item - x.kvh * x.s.chunks;
  return x;
}

template <int HD, int CG>
__global__ void __launch_bounds__(WARPS * 32, D8<HD, CG>::PER_SM) dec8_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD, CG>;
  constexpr int NC = C::NC, NT = C::NT, KC = C::KC, VW = C::VW, CH = C::CH, HS = C::HS, NST = C::NST;
  extern __shared__ __align__(128) uint8_t smem[];            // WARP_BYTES of every warp, SLOT floats, the prefix sums
  __shared__ int warp_sums[WARPS];
  __shared__ int hdr_item[2 * WARPS], hdr_flags[2 * WARPS], hdr_b[2 * WARPS];   // flags: 1 the item's first block, 2 its last
  float* const xchg = reinterpret_cast<float*>(smem + WARPS * C::WARP_BYTES);
  int* const prefix = reinterpret_cast<int*>(xchg + C::SLOT);
  auto slot_of = [&](int i) {        // slot 2 w: the piece that warp w began with, 2 w + 1: the one it ended with
    return reinterpret_cast<float*>(smem + (i >> 1) * C::WARP_BYTES + ((i & 1) ? 0 : C::RING));
  };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (threadIdx.x < 2 * WARPS) hdr_item[threadIdx.x] = -1;
  chain_wait();
  chain_trigger();                   // after the wait: the merge reads the lengths before its own

  // this warp's stretch: places and count of blocks
  Place x;
  int left;                          // blocks of the stretch that are still to do
  int u = 0;                         // line form: the unit that x is at
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
    __syncthreads();                 // the headers are empty
  } else {
    scan_blocks<NC>(p, prefix, warp_sums);
    const Line line(prefix[p.batch], gridDim.x * WARPS);
    const int w = blockIdx.x * WARPS + warp;
    u = line.begin(w);
    left = line.begin(w + 1) - u;
    if (left > 0) x = locate<NC>(p, prefix, u);
  }
  // rows of sequences without a position: zeros
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const Seq s = seq_of<NC>(p, b);
    if (s.len == 0)
      for (int r = 0; r < s.rows; ++r)
        for (int e = threadIdx.x; e < p.n_q * HD; e += blockDim.x)
          p.out[(int64_t)(s.row0 + r) * p.ldo + e] = __float2bfloat16_rn(0.f);
  }

  uint8_t* const ring = smem + warp * C::WARP_BYTES;
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  uint4* const q_sm = reinterpret_cast<uint4*>(ring + C::RING + C::SLOT * 4);      // CG > 1: [CG][KC][code][lane]
  const int ps = p.c.page_size;

  while (left > 0) {
    const int n_blk = min(x.s.n - x.blk, left);
    const int col0 = x.chunk * NC, cols = min(NC, x.s.rows * p.G - col0), h0 = x.kvh * p.G;
    const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;

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
    auto issue = [&](int i, int stage) {
      const int k = i - base, id = __shfl_sync(FULL, k < 32 ? id_c : id_n, k & 31);
      const int64_t off = id < 0 ? 0 : (int64_t)id * C::TILE;
      const int bytes = id < 0 ? 0 : 16;
      const uint32_t dst = ring_addr + stage * 2 * C::TILE;
#pragma unroll
      for (int c = 0; c < C::TILE / 512; ++c) {
        const int e = c * 32 + lane;
        const uint32_t at = dst + swz<HD>(e / CH, e % CH);
        cp_async16(at, p.c.k + off + e * 16, bytes);
        cp_async16(at + C::TILE, p.c.v + off + e * 16, bytes);
      }
    };
#pragma unroll
    for (int i = 0; i < NST; ++i) {
      if (i < n_blk) issue(i, i);
      cp_async_commit();
    }

    // q^T as the B operand: of column group cg a lane holds column g at dims 64 c + 16 t + 4 w .. + 3, scaled so that the
    // column's largest element is in [2^7, 2^8), as two codes: the nearest one and the nearest one of what is left.
    // Per column of this lane's scores (2t and 2t + 1 of each group): factor and position.
    uint32_t qh[CG == 1 ? KC : 1][4], ql[CG == 1 ? KC : 1][4];
    float c0[CG], c1[CG];
    int pos0[CG], pos1[CG];
#pragma unroll
    for (int cg = 0; cg < CG; ++cg) {
      const int col = col0 + cg * 8 + g;
      const bool live = cg * 8 + g < cols;
      const int i = live ? col / p.G : 0, h = live ? col - i * p.G : 0;
      const bf16* qrow = p.q + (int64_t)(x.s.row0 + i) * p.ldq + (int64_t)(h0 + h) * HD + 16 * t;
      uint4 raw[KC][2];
      float am = 0.f;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        raw[c][0] = *reinterpret_cast<const uint4*>(qrow + 64 * c);
        raw[c][1] = *reinterpret_cast<const uint4*>(qrow + 64 * c + 8);
      }
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
      const float mul = live ? c8_pow2(134 - eb) : 0.f, inv = c8_pow2(eb - 134) * p.scale_log2;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        uint32_t hi4[4], lo4[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4& r = raw[c][k >> 1];
          const uint32_t w0 = (k & 1) ? r.z : r.x, w1 = (k & 1) ? r.w : r.y;
          const float e0 = lo_f(w0) * mul, e1 = hi_f(w0) * mul, e2 = lo_f(w1) * mul, e3 = hi_f(w1) * mul;
          const uint32_t hi = c8_codes4(e0, e1, e2, e3), f0 = c8_half2_lo(hi), f1 = c8_half2_hi(hi);
          const float2 r0 = __half22float2(*reinterpret_cast<const __half2*>(&f0));
          const float2 r1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
          hi4[k] = hi;
          lo4[k] = c8_codes4(e0 - r0.x, e1 - r0.y, e2 - r1.x, e3 - r1.y);
        }
        if constexpr (CG == 1) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            qh[c][k] = hi4[k];
            ql[c][k] = lo4[k];
          }
        } else {                       // read back by the lane that wrote it
          q_sm[((cg * KC + c) * 2 + 0) * 32 + lane] = make_uint4(hi4[0], hi4[1], hi4[2], hi4[3]);
          q_sm[((cg * KC + c) * 2 + 1) * 32 + lane] = make_uint4(lo4[0], lo4[1], lo4[2], lo4[3]);
        }
      }
      c0[cg] = __shfl_sync(FULL, inv, t * 8);
      c1[cg] = __shfl_sync(FULL, inv, t * 8 + 4);
      const int pos = x.s.len - x.s.rows + i;
      pos0[cg] = __shfl_sync(FULL, pos, t * 8);
      pos1[cg] = __shfl_sync(FULL, pos, t * 8 + 4);
    }
    // blocks up to key full_hi need no causal mask, from key full_lo on no window mask
    const int first_row = col0 / p.G, last_row = (col0 + cols - 1) / p.G;
    const int full_hi = x.s.len - x.s.rows + first_row;
    const int full_lo = p.window > 0 ? x.s.len - x.s.rows + last_row - p.window + 1 : 0;

    float m0[CG], m1[CG], l0[CG], l1[CG], o[CG][NT][4];
#pragma unroll
    for (int cg = 0; cg < CG; ++cg) {
      m0[cg] = m1[cg] = -INFINITY;
      l0[cg] = l1[cg] = 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j) o[cg][j][0] = o[cg][j][1] = o[cg][j][2] = o[cg][j][3] = 0.f;
    }

    int stage = 0;
    for (int i = 0; i < n_blk; ++i) {
      const int at = (x.s.first + x.blk + i) * C8_BLOCK;       // first position of the block
      cp_async_wait<NST - 1>();
      __syncwarp();
      if (i - base == 32) {
        base = i;
        id_c = id_n;
        sc_c = sc_n;
        if (i + 32 < n_blk) fetch(i + 32, id_n, sc_n);
      }
      const int sc = __shfl_sync(FULL, sc_c, i - base), ke = sc & 255, ve = sc >> 8;
      const uint8_t* st = ring + stage * 2 * C::TILE;
      float s[CG][4], sb[CG][4];       // of the two codes of q
#pragma unroll
      for (int cg = 0; cg < CG; ++cg)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[cg][k] = sb[cg][k] = 0.f;
#pragma unroll
      for (int c = 0; c < KC; ++c) {                           // keys g and g + 8 at bytes 64 c + 16 t .. + 15
        const uint4 ka = *reinterpret_cast<const uint4*>(st + swz<HD>(g, 4 * c + t));
        const uint4 kb = *reinterpret_cast<const uint4*>(st + swz<HD>(g + 8, 4 * c + t));
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) {
          uint32_t qa[4], qz[4];
          if constexpr (CG == 1) {
#pragma unroll
            for (int k = 0; k < 4; ++k) { qa[k] = qh[c][k]; qz[k] = ql[c][k]; }
          } else {
            const uint4 a = q_sm[((cg * KC + c) * 2 + 0) * 32 + lane], z = q_sm[((cg * KC + c) * 2 + 1) * 32 + lane];
            qa[0] = a.x; qa[1] = a.y; qa[2] = a.z; qa[3] = a.w;
            qz[0] = z.x; qz[1] = z.y; qz[2] = z.z; qz[3] = z.w;
          }
          mma_e4m3(s[cg], ka.x, kb.x, ka.y, kb.y, qa[0], qa[1]);
          mma_e4m3(sb[cg], ka.x, kb.x, ka.y, kb.y, qz[0], qz[1]);
          mma_e4m3(s[cg], ka.z, kb.z, ka.w, kb.w, qa[2], qa[3]);
          mma_e4m3(sb[cg], ka.z, kb.z, ka.w, kb.w, qz[2], qz[3]);
        }
      }
      uint32_t vr[4][VW];              // values of keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = 2 * t + (k & 1) + (k >> 1) * 8;
        if constexpr (HD == 64) {
          const uint2 v = *reinterpret_cast<const uint2*>(st + C::TILE + swz<HD>(r, g >> 1) + (g & 1) * 8);
          vr[k][0] = v.x; vr[k][1] = v.y;
        } else {
#pragma unroll
          for (int c = 0; c < VW / 4; ++c) {
            const uint4 v = *reinterpret_cast<const uint4*>(st + C::TILE + swz<HD>(r, 8 * c + g));
            vr[k][4 * c] = v.x; vr[k][4 * c + 1] = v.y; vr[k][4 * c + 2] = v.z; vr[k][4 * c + 3] = v.w;
          }
        }
      }
      if (at + C8_BLOCK > x.s.len) {   // behind the sequence: no value whatever is there
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (at + 2 * t + (k & 1) + (k >> 1) * 8 >= x.s.len) {
#pragma unroll
            for (int w = 0; w < VW; ++w) vr[k][w] = 0;
          }
      }
      const float kf = c8_pow2(ke - 127), lv = (float)(ve - 127), inv_v = c8_pow2(127 - ve);
      const bool edge = at + C8_BLOCK - 1 > full_hi || at < full_lo;
      uint32_t pb0[CG], pb1[CG];
#pragma unroll
      for (int cg = 0; cg < CG; ++cg) {
        const float k0 = c0[cg] * kf, k1 = c1[cg] * kf;
        float s0 = fmaf(s[cg][0] + sb[cg][0], k0, lv), s1 = fmaf(s[cg][1] + sb[cg][1], k1, lv);
        float s2 = fmaf(s[cg][2] + sb[cg][2], k0, lv), s3 = fmaf(s[cg][3] + sb[cg][3], k1, lv);
        if (edge) {                    // keys that a column does not see: no weight whatever is there
          const int a = at + g, w0 = p.window > 0 ? pos0[cg] - p.window : -1, w1 = p.window > 0 ? pos1[cg] - p.window : -1;
          if (a > pos0[cg] || a <= w0) s0 = -INFINITY;
          if (a > pos1[cg] || a <= w1) s1 = -INFINITY;
          if (a + 8 > pos0[cg] || a + 8 <= w0) s2 = -INFINITY;
          if (a + 8 > pos1[cg] || a + 8 <= w1) s3 = -INFINITY;
        }
        float x0 = fmaxf(s0, s2), x1 = fmaxf(s1, s3);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          x0 = fmaxf(x0, __shfl_xor_sync(FULL, x0, w));
          x1 = fmaxf(x1, __shfl_xor_sync(FULL, x1, w));
        }
        const float n0 = fmaxf(m0[cg], x0), n1 = fmaxf(m1[cg], x1);
        // a column that has seen nothing yet keeps its maximum of -inf and weights of 0
        const float b0 = n0 == -INFINITY ? 0.f : n0, b1 = n1 == -INFINITY ? 0.f : n1;
        const float f0 = ex2(m0[cg] - b0), f1 = ex2(m1[cg] - b1);
        const float e0 = b0 - W_SHIFT, e1 = b1 - W_SHIFT;
        const float p0 = ex2(s0 - e0), p1 = ex2(s1 - e1), p2 = ex2(s2 - e0), p3 = ex2(s3 - e1);
        l0[cg] = fmaf(p0 + p2, inv_v, l0[cg] * f0);
        l1[cg] = fmaf(p1 + p3, inv_v, l1[cg] * f1);
        m0[cg] = n0;
        m1[cg] = n1;
        if (__any_sync(FULL, f0 != 1.f || f1 != 1.f)) {
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            o[cg][j][0] *= f0; o[cg][j][1] *= f1; o[cg][j][2] *= f0; o[cg][j][3] *= f1;
          }
        }
        pb0[cg] = movm_t(pack_half2(p0, p1));        // keys 0-7 of the block
        pb1[cg] = movm_t(pack_half2(p2, p3));        // keys 8-15
      }
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        const uint32_t a = __byte_perm(vr[0][w], vr[1][w], 0x5140), b = __byte_perm(vr[0][w], vr[1][w], 0x7362);
        const uint32_t c = __byte_perm(vr[2][w], vr[3][w], 0x5140), d = __byte_perm(vr[2][w], vr[3][w], 0x7362);
        const uint32_t a0 = c8_half2_lo(a), a1 = c8_half2_hi(a), a2 = c8_half2_lo(c), a3 = c8_half2_hi(c);
        const uint32_t b0 = c8_half2_lo(b), b1 = c8_half2_hi(b), b2 = c8_half2_lo(d), b3 = c8_half2_hi(d);
#pragma unroll
        for (int cg = 0; cg < CG; ++cg) {
          mma_f16(o[cg][2 * w], a0, a1, a2, a3, pb0[cg], pb1[cg]);
          mma_f16(o[cg][2 * w + 1], b0, b1, b2, b3, pb0[cg], pb1[cg]);
        }
      }
      __syncwarp();                    // every lane is done with the stage
      if (i + NST < n_blk) issue(i + NST, stage);
      cp_async_commit();
      stage = stage + 1 == NST ? 0 : stage + 1;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int cg = 0; cg < CG; ++cg)
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        l0[cg] += __shfl_xor_sync(FULL, l0[cg], w);
        l1[cg] += __shfl_xor_sync(FULL, l1[cg], w);
      }
    // lane (g, t) holds columns 2t ([0], [2]) and 2t + 1 ([1], [3]) at dims dim_of(j, g) and the one behind it
    const bool starts = x.blk == 0, ends = x.blk + n_blk == x.s.n;
    if (starts && ends && p.cluster <= 1) {
#pragma unroll
      for (int cg = 0; cg < CG; ++cg)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const int k = cg * 8 + 2 * t + hh;
          if (k >= cols) continue;
          const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
          const float l = hh ? l1[cg] : l0[cg], inv = l == 0.f ? 0.f : 1.f / l;
          bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(h0 + h) * HD;
#pragma unroll
          for (int j = 0; j < NT; ++j)
            *reinterpret_cast<__nv_bfloat162*>(dst + dim_of<HD>(j, g)) =
                __floats2bfloat162_rn(o[cg][j][hh] * inv, o[cg][j][2 + hh] * inv);
        }
    } else {
      const int si = 2 * warp + (starts ? 1 : 0);
      float* sl = slot_of(si);
      __syncwarp();                    // slot 2 w + 1 goes over the ring, which every lane has left
      if (lane == 0) {
        hdr_item[si] = x.kvh * p.chunks + x.chunk;             // with the sequence: which item
        hdr_b[si] = x.b;
        hdr_flags[si] = (starts ? 1 : 0) | (ends ? 2 : 0);
      }
#pragma unroll
      for (int cg = 0; cg < CG; ++cg) {
        if (g == 0) {
          sl[cg * 8 + 2 * t] = m0[cg]; sl[cg * 8 + 2 * t + 1] = m1[cg];
          sl[NC + cg * 8 + 2 * t] = l0[cg]; sl[NC + cg * 8 + 2 * t + 1] = l1[cg];
        }
        float* so = sl + 2 * NC + (cg * 8 + 2 * t) * HS + 2 * g;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          *reinterpret_cast<float2*>(so + 16 * j) = make_float2(o[cg][j][0], o[cg][j][2]);
          *reinterpret_cast<float2*>(so + HS + 16 * j) = make_float2(o[cg][j][1], o[cg][j][3]);
        }
      }
    }
    left -= n_blk;
    if (left > 0) {                    // the line goes on with the next item
      u += n_blk;
      x = locate<NC>(p, prefix, u);
    }
  }
  __syncthreads();

  // Pieces in the order of the line: slots 2 w and 2 w + 1 of warp w; lane k < 16 knows slot k. Those of one item are merged
  // by tasks of one column and 32 pairs of dims.
  const int my_item = lane < 2 * WARPS ? hdr_item[lane] : -1, my_b = my_item >= 0 ? hdr_b[lane] : -1;
  unsigned todo = __ballot_sync(FULL, my_item >= 0);
  if (p.cluster > 1) {
    if (todo == 0)                     // fewer blocks than CTAs: an empty piece
      for (int e = threadIdx.x; e < NC; e += blockDim.x) {
        xchg[e] = -INFINITY;
        xchg[NC + e] = 0.f;
      }
  }
  while (todo) {
    const int first = __ffs(todo) - 1, it = __shfl_sync(FULL, my_item, first), b = __shfl_sync(FULL, my_b, first);
    const unsigned mine = __ballot_sync(FULL, my_item == it && my_b == b);
    todo &= ~mine;
    const int last = 31 - __clz(mine);
    const bool starts = hdr_flags[first] & 1, ends = hdr_flags[last] & 2;
    const Seq s = seq_of<NC>(p, b);
    const int kvh = it / p.chunks, col0 = (it - kvh * p.chunks) * NC, cols = min(NC, s.rows * p.G - col0);
    constexpr int PARTS = HD / 64;     // tasks per column
    for (int task = warp; task < cols * PARTS; task += WARPS) {
      const int k = task / PARTS, pr = (task - k * PARTS) * 32 + lane;     // pair pr: dims dim_of(pr / 8, pr % 8) and the next
      const bool has = (mine >> lane) & 1;
      const float mk = has ? slot_of(lane)[k] : -INFINITY;
      float m = mk;
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, w));
      m = __shfl_sync(FULL, m, 0);     // lanes 16 .. 31 hold no slot
      const float f = mk == -INFINITY ? 0.f : ex2(mk - m);
      float l = has ? slot_of(lane)[NC + k] * f : 0.f;
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) l += __shfl_xor_sync(FULL, l, w);
      l = __shfl_sync(FULL, l, 0);
      float2 v = make_float2(0.f, 0.f);
      for (unsigned rem = mine; rem; rem &= rem - 1) {
        const int sl = __ffs(rem) - 1;
        const float fk = __shfl_sync(FULL, f, sl);
        const float2 ov = *reinterpret_cast<const float2*>(slot_of(sl) + 2 * NC + k * HS + 2 * pr);
        v.x = fmaf(ov.x, fk, v.x);
        v.y = fmaf(ov.y, fk, v.y);
      }
      if (p.cluster > 1) {
        *reinterpret_cast<float2*>(xchg + 2 * NC + k * HS + 2 * pr) = v;
        if (pr == 0) {
          xchg[k] = m;
          xchg[NC + k] = l;
        }
      } else if (starts && ends) {
        const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16* dst = p.out + (int64_t)(s.row0 + i) * p.ldo + (int64_t)(kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
        *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
      } else {                         // 1: the item starts in this CTA and goes on; 0: it came from an earlier one
        float* dst = p.partial + ((int64_t)blockIdx.x * 2 + (starts ? 1 : 0)) * C::PSLOT;
        *reinterpret_cast<float2*>(dst + 2 * NC + k * HD + 2 * pr) = v;
        if (pr == 0) {
          dst[k] = m;
          dst[NC + k] = l;
        }
      }
    }
  }
  if (p.cluster > 1) {
    // every CTA of the cluster finishes a share of the item's pairs from all the CTAs' pieces
    cluster_arrive();
    cluster_wait();
    const int rank = (int)cluster_ctarank();
    const int item = blockIdx.x / p.cluster, per_seq = p.n_kv * p.chunks;
    const int b = item / per_seq, in = item - b * per_seq, kvh = in / p.chunks;
    const Seq s = seq_of<NC>(p, b);
    const int col0 = (in - kvh * p.chunks) * NC, cols = s.len == 0 ? 0 : min(NC, s.rows * p.G - col0);
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
        if (mr[r] != -INFINITY) {                    // an empty piece's sums may not be written
          const float f = ex2(mr[r] - m);
          l = fmaf(lr[r], f, l);
          ox = fmaf(vx[r], f, ox);
          oy = fmaf(vy[r], f, oy);
        }
      const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* dst = p.out + (int64_t)(s.row0 + i) * p.ldo + (int64_t)(kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
      *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(ox * inv, oy * inv);
    }
    // nobody leaves while a neighbour may still read its shared memory
    cluster_arrive();
    cluster_wait();
  }
}

// Items that cross CTAs. The blocks of this grid are the CTAs of the attention kernel: those that hold pieces of an item
// share its elements out among them, so that few long items are merged by many CTAs. Reads the same lengths, so it finds
// the same places. Four neighbouring pairs of dims (a 32-byte sector) to four lanes, eight pieces at a time.
template <int HD, int CG>
__device__ __forceinline__ void merge_item(const Dec8Dev& p, const Line& line, const Place& x, int first) {
  using C = D8<HD, CG>;
  constexpr int NC = C::NC;
  const int c0 = line.owner(first) / WARPS, c1 = line.owner(first + x.s.n - 1) / WARPS;
  const int col0 = x.chunk * NC, cols = min(NC, x.s.rows * p.G - col0);
  const int lane = threadIdx.x & 31, pk = lane >> 2, pe = lane & 3;
  const int workers = (c1 - c0 + 1) * WARPS;
  for (int quad = (blockIdx.x - c0) * WARPS + (threadIdx.x >> 5); quad < cols * (HD / 8); quad += workers) {
    const int k = quad / (HD / 8), pr = (quad - k * (HD / 8)) * 4 + pe;
    float m = -INFINITY, l = 0.f;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = c0 + pk; c <= c1; c += 8) {
      const float* sl = p.partial + (2 * (int64_t)c + (c == c0 ? 1 : 0)) * C::PSLOT;
      const float mk = __ldcg(sl + k), lk = __ldcg(sl + NC + k);
      const float2 ov = __ldcg(reinterpret_cast<const float2*>(sl + 2 * NC + k * HD + 2 * pr));
      if (mk == -INFINITY) continue;
      const float n = fmaxf(m, mk), fa = ex2(m - n), fb = ex2(mk - n);
      l = l * fa + lk * fb;
      v.x = v.x * fa + ov.x * fb;
      v.y = v.y * fa + ov.y * fb;
      m = n;
    }
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      const float mk = __shfl_xor_sync(FULL, m, w), lk = __shfl_xor_sync(FULL, l, w);
      const float ox = __shfl_xor_sync(FULL, v.x, w), oy = __shfl_xor_sync(FULL, v.y, w);
      const float n = fmaxf(m, mk), fa = m == n ? 1.f : ex2(m - n), fb = mk == n ? 1.f : ex2(mk - n);   // both may be empty
      l = l * fa + lk * fb;
      v.x = v.x * fa + ox * fb;
      v.y = v.y * fa + oy * fb;
      m = n;
    }
    if (pk == 0) {
      const int i = (col0 + k) / p.G, h = col0 + k - i * p.G;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16* dst = p.out + (int64_t)(x.s.row0 + i) * p.ldo + (int64_t)(x.kvh * p.G + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
      *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
    }
  }
}
template <int HD, int CG>
__global__ void __launch_bounds__(WARPS * 32) dec8_merge_kernel(const __grid_constant__ Dec8Dev p) {
  constexpr int NC = D8<HD, CG>::NC;
  extern __shared__ __align__(16) int prefix[];
  __shared__ int warp_sums[WARPS];
  chain_trigger();
  // this kernel starts behind the attention kernel's wait, so the lengths are there; only the pieces have to be waited for
  scan_blocks<NC>(p, prefix, warp_sums);
  const Line line(prefix[p.batch], gridDim.x * WARPS);
  const int u0 = line.begin(blockIdx.x * WARPS), u1 = line.begin((blockIdx.x + 1) * WARPS);
  Place a{}, z{};
  if (u0 < u1) {
    a = locate<NC>(p, prefix, u0);
    z = locate<NC>(p, prefix, u1 - 1);
  }
  chain_wait();
  if (u0 >= u1) return;
  // the item that came from an earlier CTA, and the one that goes on in the next (they may be the same)
  if (a.blk > 0) merge_item<HD, CG>(p, line, a, u0 - a.blk);
  const int first = u1 - 1 - z.blk;
  if (z.blk + 1 < z.s.n && first >= u0) merge_item<HD, CG>(p, line, z, first);
}

template <int HD, int CG>
int launch_t(const Attn8Args& a, Dec8Dev& p, cudaStream_t s) {
  using C = D8<HD, CG>;
  p.chunks = (int)(((int64_t)a.rows * p.G + C::NC - 1) / C::NC);
  const int span = a.window > 0 && (int64_t)a.window + a.rows + C8_BLOCK < a.kv_len ? a.window + a.rows + C8_BLOCK : a.kv_len;
  const int64_t blocks = ((int64_t)span + C8_BLOCK - 1) / C8_BLOCK, items = (int64_t)a.batch * a.n_kv * p.chunks;
  // block numbers, of the call and of the pool, are 32-bit
  if (blocks > 0x7fffffff / (items + 1) ||
      (int64_t)a.c.num_pages * a.n_kv > 0x7fffffff / (a.c.page_size / C8_BLOCK))
    return POP_E_INVALID;
  const int ctas = device_sms() * C::PER_SM;
  // Clusters (one launch): one CTA per item while its warps have few blocks each; more per item while all of them are
  // resident at once and no warp gets more than CLUSTER_BLOCKS blocks.
  int cs = 1;
  while (cs < 8 && blocks > (int64_t)cs * WARPS * 2 && items * cs * 2 <= ctas) cs *= 2;
  p.cluster = blocks <= (int64_t)cs * WARPS * CLUSTER_BLOCKS && (cs > 1 || blocks <= WARPS * 4) ? cs : 0;
  int64_t grid = items * cs;
  if (!p.cluster) {
    if (a.batch > MAX_BATCH) return POP_E_INVALID;
    grid = ctas;
    const int64_t most = (blocks * items + WARPS - 1) / WARPS;    // no fewer than one block per warp
    if (grid > most) grid = most;
    if ((size_t)grid * 2 * C::PSLOT * 4 > a.workspace_bytes) return POP_E_NOSPACE;
  }
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  const int scan_bytes = p.cluster ? 0 : (a.batch + 1) * 4;
  static bool configured = false;
  if (!configured) {
    if (cudaFuncSetAttribute(dec8_kernel<HD, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             C::SMEM + (MAX_BATCH + 1) * 4) != cudaSuccess)
      return POP_E_CUDA;
    configured = true;
  }
  ProfScope prof(PROF_DECODE_ATTN, (double)a.batch * span * a.n_kv * (2.0 * HD + 0.125), s);
  const size_t smem = (size_t)(C::SMEM + scan_bytes);
  const cudaError_t rc = p.cluster > 1
                             ? launch_chained_cluster_x(dec8_kernel<HD, CG>, dim3((unsigned)grid), dim3(WARPS * 32), smem, s,
                                                        (unsigned)p.cluster, p)
                             : launch_chained(dec8_kernel<HD, CG>, dim3((unsigned)grid), dim3(WARPS * 32), smem, s, p);
  if (rc != cudaSuccess) return POP_E_CUDA;
  count_launch();
  if (!p.cluster) {
    if (launch_chained(dec8_merge_kernel<HD, CG>, dim3((unsigned)grid), dim3(WARPS * 32), (size_t)scan_bytes, s, p) !=
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
  p.seq_lens = a.seq_lens; p.kv_len = a.kv_len; p.window = a.window;
  p.out = a.out; p.ldo = a.ldo;
  p.batch = a.batch; p.n_q = a.n_q; p.n_kv = a.n_kv; p.G = a.n_q / a.n_kv;
  p.partial = static_cast<float*>(a.workspace);
  p.scale_log2 = 1.4426950408889634f / sqrtf((float)a.head_dim);
  // two column groups per item where there are more than eight columns: the keys are read from memory once for both. Not
  // for hd 256, whose accumulators alone would fill the registers.
  const bool wide = (int64_t)a.rows * p.G > 8;
  switch (a.head_dim) {
    case 64: return wide ? launch_t<64, 2>(a, p, s) : launch_t<64, 1>(a, p, s);
    case 128: return wide ? launch_t<128, 2>(a, p, s) : launch_t<128, 1>(a, p, s);
    default: return launch_t<256, 1>(a, p, s);
  }
}

int launch_decode_attention8(const Attn8Args& a, cudaStream_t s) {
  if (!a.q || !a.out || !c8_cache_ok(a.c)) return POP_E_INVALID;
  if (a.batch < 1 || a.batch > MAX_BATCH || a.n_kv < 1 || a.n_q < 1 || a.n_q % a.n_kv || a.n_q > 65536 || a.kv_len < 0 ||
      a.kv_len > 0x7ffffff0 || a.window < 0 || a.window > 0x7ffffff0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8 ||
      reinterpret_cast<uintptr_t>(a.workspace) % 16)
    return POP_E_INVALID;
  if ((int64_t)a.kv_len > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  return launch_few8(a, s);
}

}  // namespace pop
