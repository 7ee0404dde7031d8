// Single-query attention over the 8-bit paged cache (paper Eq. 1, Attn for the one position of a decode step).
//
// For sequence b with len positions, query head h of kv head g, and seen positions j in [max(0, len - window), len):
//   out[b][h] = sum_j p_j 2^(ev_j) v_j / sum_j p_j,   p_j = exp2(c q.k_j 2^(ek_j) - max),  c = log2(e) / sqrt(hd)
// with codes k_j, v_j and block exponents ek_j, ev_j. The V scale is folded into the exponent: with
// w_j = exp2(c q.k_j 2^(ek_j) + ev_j - m) and m the running maximum of that sum, out = sum w_j v_j / sum w_j 2^(-ev_j), so
// the weights that meet the tensor cores are at most 1 whatever the scales of the blocks are.
//
// Bound by the cache's bytes: 2 hd + 1/8 per kv head and position. A warp takes blocks of 16 positions of one (sequence,
// kv head, group of at most 8 query heads) through its own small ring in shared memory (16-byte asynchronous copies; a
// block is one contiguous piece) and works on them with the warp-level MMA, the KEYS on the M side (S^T = K q^T,
// O^T = V^T P^T): a dot product does not see the order of its terms, so a lane's 16 consecutive bytes of a key feed the
// MMAs as they are. K codes meet the query as E4M3 operands: after a power-of-two scale per head an element is the sum of
// two codes, exactly for bf16 elements down to 2^-9 of the head's largest and to within 2^-17 of that below (half the
// smallest code). V codes become f16 exactly (two keys interleaved by a byte permute, one conversion per pair) and meet
// weights in f16 with 2^14 as the largest (half a step: 2^-11 relative); scores, statistics and sums are fp32. The 8-bit
// MMA also runs at 3.5 times the f16 one's rate; with f16 on both sides the kernel was bound by instructions (measured
// with 48 sequences of up to 16001 positions: 154 us).
//
// Work is split evenly whatever the lengths are: all (sequence, kv head, head group) items form one line of 16-position
// blocks, every warp of the grid takes an equal stretch of it. An item that a warp has whole is finished by it; pieces
// of one CTA are merged in shared memory, items that cross CTAs through the workspace by a second, chained launch.
#include "cache8.cuh"

namespace pop {
namespace {

constexpr uint32_t FULL = 0xffffffffu;
constexpr int MAXG = 8;              // query heads per item: the N extent of one MMA
constexpr int WARPS = 8;
constexpr int MAX_BATCH = 8192;     // the block counts' prefix sums sit in shared memory
constexpr float W_SHIFT = 14.f;      // weights are stored times 2^14

template <int HD>
struct D8 {
  static constexpr int NT = HD / 16;           // MMAs along the head
  static constexpr int KC = HD / 64;           // 16-byte pieces of a key row per lane
  static constexpr int VW = HD / 32;           // words of a value row per lane
  static constexpr int CH = HD / 16;           // 16-byte pieces of a row
  static constexpr int TILE = C8_BLOCK * HD;   // bytes of a block's keys; its values behind them
  static constexpr int NST = HD == 64 ? 3 : 2; // blocks in flight per warp: with PER_SM CTAs 128 KB and more per SM
  static constexpr int PER_SM = HD == 64 ? 3 : (HD == 128 ? 2 : 1);
  static constexpr int HS = HD + 4;            // floats per head of a piece in shared memory: rows 4 banks apart
  static constexpr int SLOT = MAXG * HS + 2 * MAXG;
  static constexpr int PSLOT = MAXG * HD + 2 * MAXG;   // floats of a piece in the workspace
  // a warp's memory: ring, then the piece it begins with; the piece it ends with goes over the idle ring
  static constexpr int RING = NST * 2 * TILE;
  static constexpr int WARP_BYTES = RING + SLOT * 4;
  static constexpr int SMEM = WARPS * WARP_BYTES;
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
  const int32_t* seq_lens; int kv_len, window;
  bf16* out; int64_t ldo;
  int batch, n_q, n_kv, G, hg;       // G = n_q / n_kv, hg = head groups per kv head
  int whole;                         // 1: every CTA takes one whole item (short caches)
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

// Seen positions of a sequence: [lo, len), blocks first .. first + n - 1
struct Span { int len, lo, first, n; };
__device__ __forceinline__ Span span_of(const Dec8Dev& p, int b) {
  Span s;
  s.len = p.seq_lens ? p.seq_lens[b] : p.kv_len;
  if (s.len > p.kv_len) {                       // longer than the caller said: nothing past it is read
    s.len = p.kv_len;
    atomicMin(p.status, (int)POP_E_INVALID);
  }
  if (s.len < 0) s.len = 0;
  s.lo = (p.window > 0 && p.window < s.len) ? s.len - p.window : 0;
  s.first = s.lo / C8_BLOCK;
  s.n = (s.len + C8_BLOCK - 1) / C8_BLOCK - s.first;
  return s;
}

// prefix[b] = blocks of the sequences before b, for b <= batch. By all threads; nothing to do for equal lengths.
__device__ __forceinline__ void scan_blocks(const Dec8Dev& p, int* prefix, int* warp_sums) {
  if (p.seq_lens == nullptr) return;
  const int per = (p.batch + blockDim.x - 1) / blockDim.x;
  const int b0 = min(p.batch, (int)threadIdx.x * per), b1 = min(p.batch, b0 + per);
  int sum = 0;
  for (int b = b0; b < b1; ++b) sum += span_of(p, b).n;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(FULL, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < warp; ++w) base += warp_sums[w];
  int run = base + incl - sum;
  for (int b = b0; b < b1; ++b) {
    prefix[b] = run;
    run += span_of(p, b).n;
  }
  if (b1 == p.batch && b0 < p.batch) prefix[p.batch] = run;
  __syncthreads();
}
// The line of all blocks, cut into W stretches that differ by at most one block (everything below 2^31: the host checks)
struct Line {
  int T, per, rest;
  __device__ __forceinline__ Line(const Dec8Dev& p, const int* prefix, int H, int W) {
    T = (p.seq_lens == nullptr ? span_of(p, 0).n * p.batch : prefix[p.batch]) * H;
    per = T / W;
    rest = T - per * W;
  }
  __device__ __forceinline__ int begin(int w) const { return w * per + min(w, rest); }
  __device__ __forceinline__ int owner(int u) const {      // the stretch that holds unit u
    const int big = rest * (per + 1);
    return u < big ? u / (per + 1) : rest + (u - big) / per;
  }
};
// Where unit u (< total) of the line lies: sequence, item of the sequence (kv head and head group), block of the item
struct Place { int b, item, blk; Span s; };
__device__ __forceinline__ Place locate(const Dec8Dev& p, const int* prefix, int H, int u) {
  Place x;
  int off;
  if (p.seq_lens == nullptr) {
    const int per = span_of(p, 0).n * H;
    x.b = u / per;
    off = u - x.b * per;
  } else {
    int lo = 0, hi = p.batch - 1;               // the last b with prefix[b] * H <= u: its span is not empty
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prefix[mid] * H <= u) lo = mid;
      else hi = mid - 1;
    }
    x.b = lo;
    off = u - prefix[lo] * H;
  }
  x.s = span_of(p, x.b);
  x.item = off / x.s.n;
  x.blk = off - x.item * x.s.n;
  return x;
}

template <int HD>
__global__ void __launch_bounds__(WARPS * 32, D8<HD>::PER_SM) dec8_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD>;
  constexpr int NT = C::NT, KC = C::KC, VW = C::VW, CH = C::CH, HS = C::HS, NST = C::NST;
  extern __shared__ __align__(128) uint8_t smem[];            // WARP_BYTES of every warp, then the prefix sums
  __shared__ int warp_sums[WARPS];
  __shared__ int hdr_item[2 * WARPS], hdr_flags[2 * WARPS];   // flags: 1 holds the item's first block, 2 its last
  int* prefix = reinterpret_cast<int*>(smem + C::SMEM);
  auto slot_of = [&](int i) {        // slot 2 w: the piece that warp w began with, 2 w + 1: the one it ended with
    return reinterpret_cast<float*>(smem + (i >> 1) * C::WARP_BYTES + ((i & 1) ? 0 : C::RING));
  };
  chain_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (threadIdx.x < 2 * WARPS) hdr_item[threadIdx.x] = -1;
  chain_wait();
  scan_blocks(p, prefix, warp_sums);
  __syncthreads();
  const int H = p.n_kv * p.hg;

  // sequences without a position: rows of zeros
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x)
    if (span_of(p, b).n == 0)
      for (int e = threadIdx.x; e < p.n_q * HD; e += blockDim.x) p.out[(int64_t)b * p.ldo + e] = __float2bfloat16_rn(0.f);

  int u, u_end;
  if (p.whole) {                     // this CTA's item, its blocks dealt to the warps in stretches
    const int b = blockIdx.x / H, item = blockIdx.x - b * H;
    const Span s = span_of(p, b);
    const int base = (p.seq_lens ? prefix[b] * H : b * H * s.n) + item * s.n;
    u = base + s.n * warp / WARPS;
    u_end = base + s.n * (warp + 1) / WARPS;
  } else {
    const Line line(p, prefix, H, gridDim.x * WARPS);
    const int w = blockIdx.x * WARPS + warp;
    u = line.begin(w);
    u_end = line.begin(w + 1);
  }
  uint8_t* const ring = smem + warp * C::WARP_BYTES;
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);

  while (u < u_end) {
    const Place x = locate(p, prefix, H, u);
    const int n_blk = min(x.s.n - x.blk, u_end - u);
    const int kvh = x.item / p.hg, h0 = kvh * p.G + (x.item - kvh * p.hg) * MAXG;
    const int heads = min(MAXG, kvh * p.G + p.G - h0);
    const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;
    const int ps = p.c.page_size;

    // Places and scales of 32 blocks at a time, one per lane: block number in the pool (-1, read as zeros, for a table
    // entry that is no page of it) and both scale bytes
    auto fetch = [&](int i, int& id, int& sc) {
      id = -1;
      sc = 127 | 127 << 8;
      if (i + lane < n_blk) {
        const int pos = (x.s.first + x.blk + i + lane) * C8_BLOCK, pi = pos / ps, page = bt[pi];
        if ((unsigned)page < (unsigned)p.c.num_pages) {
          id = (page * p.n_kv + kvh) * (ps / C8_BLOCK) + (pos - pi * ps) / C8_BLOCK;
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

    // q^T as the B operand: lane holds head g at dims 64 c + 16 t + 4 w .. + 3, scaled so that the head's largest element is
    // in [2^7, 2^8), as two codes: the nearest one and the nearest one of what is left
    uint32_t qh[KC][4], ql[KC][4];
    float c0, c1;                      // score factors of heads 2t and 2t + 1
    {
      const bf16* qrow = p.q + (int64_t)x.b * p.ldq + (int64_t)(h0 + (g < heads ? g : 0)) * HD + 16 * t;
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
        for (int i = 0; i < 2; ++i) {
          const uint32_t w[4] = {raw[c][i].x, raw[c][i].y, raw[c][i].z, raw[c][i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) am = fmaxf(am, fmaxf(fabsf(lo_f(w[k])), fabsf(hi_f(w[k]))));
        }
      am = fmaxf(am, __shfl_xor_sync(FULL, am, 1));
      am = fmaxf(am, __shfl_xor_sync(FULL, am, 2));
      const int eb = max((int)(__float_as_uint(am) >> 23), 20);
      const float mul = g < heads ? c8_pow2(134 - eb) : 0.f, inv = c8_pow2(eb - 134) * p.scale_log2;
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t w[4] = {raw[c][i].x, raw[c][i].y, raw[c][i].z, raw[c][i].w};
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float e0 = lo_f(w[2 * k]) * mul, e1 = hi_f(w[2 * k]) * mul;
            const float e2 = lo_f(w[2 * k + 1]) * mul, e3 = hi_f(w[2 * k + 1]) * mul;
            const uint32_t hi = c8_codes4(e0, e1, e2, e3), f0 = c8_half2_lo(hi), f1 = c8_half2_hi(hi);
            const float2 r0 = __half22float2(*reinterpret_cast<const __half2*>(&f0));
            const float2 r1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
            qh[c][2 * i + k] = hi;
            ql[c][2 * i + k] = c8_codes4(e0 - r0.x, e1 - r0.y, e2 - r1.x, e3 - r1.y);
          }
        }
      c0 = __shfl_sync(FULL, inv, t * 8);
      c1 = __shfl_sync(FULL, inv, t * 8 + 4);
    }

    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    float o[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

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
      float s[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};   // of the two codes of q
#pragma unroll
      for (int c = 0; c < KC; ++c) {                           // keys g and g + 8 at bytes 64 c + 16 t .. + 15
        const uint4 ka = *reinterpret_cast<const uint4*>(st + swz<HD>(g, 4 * c + t));
        const uint4 kb = *reinterpret_cast<const uint4*>(st + swz<HD>(g + 8, 4 * c + t));
        mma_e4m3(s, ka.x, kb.x, ka.y, kb.y, qh[c][0], qh[c][1]);
        mma_e4m3(sb, ka.x, kb.x, ka.y, kb.y, ql[c][0], ql[c][1]);
        mma_e4m3(s, ka.z, kb.z, ka.w, kb.w, qh[c][2], qh[c][3]);
        mma_e4m3(sb, ka.z, kb.z, ka.w, kb.w, ql[c][2], ql[c][3]);
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
      const float kf = c8_pow2(ke - 127), k0 = c0 * kf, k1 = c1 * kf;
      const float lv = (float)(ve - 127), inv_v = c8_pow2(127 - ve);
      float s0 = fmaf(s[0] + sb[0], k0, lv), s1 = fmaf(s[1] + sb[1], k1, lv);
      float s2 = fmaf(s[2] + sb[2], k0, lv), s3 = fmaf(s[3] + sb[3], k1, lv);
      if (at < x.s.lo || at + C8_BLOCK > x.s.len) {  // positions outside the span: no weight, and no value whatever is there
        if (at + g < x.s.lo || at + g >= x.s.len) s0 = s1 = -INFINITY;
        if (at + g + 8 < x.s.lo || at + g + 8 >= x.s.len) s2 = s3 = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = at + 2 * t + (k & 1) + (k >> 1) * 8;
          if (key < x.s.lo || key >= x.s.len) {
#pragma unroll
            for (int w = 0; w < VW; ++w) vr[k][w] = 0;
          }
        }
      }
      float x0 = fmaxf(s0, s2), x1 = fmaxf(s1, s3);
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        x0 = fmaxf(x0, __shfl_xor_sync(FULL, x0, w));
        x1 = fmaxf(x1, __shfl_xor_sync(FULL, x1, w));
      }
      // a block of the span holds a seen position, so the new maxima are finite
      const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
      const float f0 = ex2(m0 - n0), f1 = ex2(m1 - n1);       // 0 on the first block
      const float e0 = n0 - W_SHIFT, e1 = n1 - W_SHIFT;
      const float p0 = ex2(s0 - e0), p1 = ex2(s1 - e1), p2 = ex2(s2 - e0), p3 = ex2(s3 - e1);
      l0 = fmaf(p0 + p2, inv_v, l0 * f0);
      l1 = fmaf(p1 + p3, inv_v, l1 * f1);
      m0 = n0;
      m1 = n1;
      if (__any_sync(FULL, f0 != 1.f || f1 != 1.f)) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          o[j][0] *= f0; o[j][1] *= f1; o[j][2] *= f0; o[j][3] *= f1;
        }
      }
      const uint32_t pb0 = movm_t(pack_half2(p0, p1));        // keys 0-7 of the block
      const uint32_t pb1 = movm_t(pack_half2(p2, p3));        // keys 8-15
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        const uint32_t a = __byte_perm(vr[0][w], vr[1][w], 0x5140), b = __byte_perm(vr[0][w], vr[1][w], 0x7362);
        const uint32_t c = __byte_perm(vr[2][w], vr[3][w], 0x5140), d = __byte_perm(vr[2][w], vr[3][w], 0x7362);
        mma_f16(o[2 * w], c8_half2_lo(a), c8_half2_hi(a), c8_half2_lo(c), c8_half2_hi(c), pb0, pb1);
        mma_f16(o[2 * w + 1], c8_half2_lo(b), c8_half2_hi(b), c8_half2_lo(d), c8_half2_hi(d), pb0, pb1);
      }
      __syncwarp();                    // every lane is done with the stage
      if (i + NST < n_blk) issue(i + NST, stage);
      cp_async_commit();
      stage = stage + 1 == NST ? 0 : stage + 1;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      l0 += __shfl_xor_sync(FULL, l0, w);
      l1 += __shfl_xor_sync(FULL, l1, w);
    }
    // lane (g, t) holds heads 2t ([0], [2]) and 2t + 1 ([1], [3]) at dims dim_of(j, g) and the one behind it
    const bool starts = x.blk == 0, ends = x.blk + n_blk == x.s.n;
    if (starts && ends) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        if (2 * t + hh >= heads) continue;
        const float inv = 1.f / (hh ? l1 : l0);
        bf16* dst = p.out + (int64_t)x.b * p.ldo + (int64_t)(h0 + 2 * t + hh) * HD;
#pragma unroll
        for (int j = 0; j < NT; ++j)
          *reinterpret_cast<__nv_bfloat162*>(dst + dim_of<HD>(j, g)) = __floats2bfloat162_rn(o[j][hh] * inv, o[j][2 + hh] * inv);
      }
    } else {
      const int si = 2 * warp + (starts ? 1 : 0);
      float* sl = slot_of(si);
      __syncwarp();                    // slot 2 w + 1 goes over the ring, which every lane has left
      if (lane == 0) {
        hdr_item[si] = x.b * H + x.item;
        hdr_flags[si] = (starts ? 1 : 0) | (ends ? 2 : 0);
      }
      if (g == 0) {
        sl[2 * t] = m0; sl[2 * t + 1] = m1;
        sl[MAXG + 2 * t] = l0; sl[MAXG + 2 * t + 1] = l1;
      }
      float* so = sl + 2 * MAXG + 2 * t * HS + 2 * g;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<float2*>(so + 16 * j) = make_float2(o[j][0], o[j][2]);
        *reinterpret_cast<float2*>(so + HS + 16 * j) = make_float2(o[j][1], o[j][3]);
      }
    }
    u += n_blk;
  }
  __syncthreads();

  // pieces in the order of the line: slots 2 w and 2 w + 1 of warp w; those of one item are neighbours
  for (int i = 0; i < 2 * WARPS;) {
    const int it = hdr_item[i];
    if (it < 0) { ++i; continue; }
    int last = i;
    for (int k = i + 1; k < 2 * WARPS; ++k)
      if (hdr_item[k] == it) last = k;
    const bool starts = hdr_flags[i] & 1, ends = hdr_flags[last] & 2;
    const int b = it / H, item = it - b * H, kvh = item / p.hg, h0 = kvh * p.G + (item - kvh * p.hg) * MAXG;
    const int heads = min(MAXG, kvh * p.G + p.G - h0);
    for (int e = threadIdx.x; e < heads * (HD / 2); e += blockDim.x) {
      const int h = e / (HD / 2), pr = e - h * (HD / 2);      // pair pr of the head: dims dim_of(pr / 8, pr % 8) and the next
      float m = -INFINITY, l = 0.f;
      float2 v = make_float2(0.f, 0.f);
      for (int k = i; k <= last; ++k)
        if (hdr_item[k] == it) m = fmaxf(m, slot_of(k)[h]);
      for (int k = i; k <= last; ++k) {
        if (hdr_item[k] != it) continue;
        const float* sl = slot_of(k);
        const float f = ex2(sl[h] - m);
        const float2 ov = *reinterpret_cast<const float2*>(sl + 2 * MAXG + h * HS + 2 * pr);
        l = fmaf(sl[MAXG + h], f, l);
        v.x = fmaf(ov.x, f, v.x);
        v.y = fmaf(ov.y, f, v.y);
      }
      if (starts && ends) {
        const float inv = 1.f / l;
        bf16* dst = p.out + (int64_t)b * p.ldo + (int64_t)(h0 + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
        *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
      } else {                       // 1: the item starts in this CTA and goes on; 0: it came from an earlier one
        float* dst = p.partial + ((int64_t)blockIdx.x * 2 + (starts ? 1 : 0)) * C::PSLOT;
        *reinterpret_cast<float2*>(dst + 2 * MAXG + h * HD + 2 * pr) = v;
        if (pr == 0) {
          dst[h] = m;
          dst[MAXG + h] = l;
        }
      }
    }
    i = last + 1;
  }
}

// Items that cross CTAs. The blocks of this grid are the CTAs of the attention kernel: those that hold pieces of an item
// share its elements out among them, so that few long items are merged by many CTAs. Reads the same lengths, so it finds
// the same places. Four neighbouring pairs of dims (a 32-byte sector) to four lanes, eight pieces at a time.
template <int HD>
__device__ __forceinline__ void merge_item(const Dec8Dev& p, const Line& line, int H, const Place& x, int first) {
  using C = D8<HD>;
  const int c0 = line.owner(first) / WARPS, c1 = line.owner(first + x.s.n - 1) / WARPS;
  const int kvh = x.item / p.hg, h0 = kvh * p.G + (x.item - kvh * p.hg) * MAXG;
  const int heads = min(MAXG, kvh * p.G + p.G - h0);
  const int lane = threadIdx.x & 31, pk = lane >> 2, pe = lane & 3;
  const int workers = (c1 - c0 + 1) * WARPS;
  for (int quad = (blockIdx.x - c0) * WARPS + (threadIdx.x >> 5); quad < heads * (HD / 8); quad += workers) {
    const int h = quad / (HD / 8), pr = (quad - h * (HD / 8)) * 4 + pe;
    float m = -INFINITY, l = 0.f;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int k = c0 + pk; k <= c1; k += 8) {
      const float* sl = p.partial + (2 * (int64_t)k + (k == c0 ? 1 : 0)) * C::PSLOT;
      const float mk = __ldcg(sl + h), lk = __ldcg(sl + MAXG + h);
      const float2 ov = __ldcg(reinterpret_cast<const float2*>(sl + 2 * MAXG + h * HD + 2 * pr));
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
      const float inv = 1.f / l;
      bf16* dst = p.out + (int64_t)x.b * p.ldo + (int64_t)(h0 + h) * HD + dim_of<HD>(pr >> 3, pr & 7);
      *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
    }
  }
}
template <int HD>
__global__ void __launch_bounds__(WARPS * 32) dec8_merge_kernel(const __grid_constant__ Dec8Dev p) {
  extern __shared__ __align__(16) int prefix[];
  __shared__ int warp_sums[WARPS];
  chain_trigger();
  chain_wait();
  scan_blocks(p, prefix, warp_sums);
  const int H = p.n_kv * p.hg;
  const Line line(p, prefix, H, gridDim.x * WARPS);
  const int u0 = line.begin(blockIdx.x * WARPS), u1 = line.begin((blockIdx.x + 1) * WARPS);
  if (u0 >= u1) return;
  // the item that came from an earlier CTA, and the one that goes on in the next (they may be the same)
  const Place a = locate(p, prefix, H, u0);
  if (a.blk > 0) merge_item<HD>(p, line, H, a, u0 - a.blk);
  const Place z = locate(p, prefix, H, u1 - 1);
  const int first = u1 - 1 - z.blk;
  if (z.blk + 1 < z.s.n && first >= u0) merge_item<HD>(p, line, H, z, first);
}

// Short caches: one CTA per item and no second launch, up to this many blocks of the longest span.
constexpr int WHOLE_BLOCKS = 32;

template <int HD>
int launch_t(const Attn8Args& a, Dec8Dev& p, cudaStream_t s) {
  using C = D8<HD>;
  constexpr int PER_SM = C::PER_SM;
  const int scan_bytes = a.seq_lens ? (a.batch + 1) * 4 : 0;
  const int H = p.n_kv * p.hg;
  const int span = a.window > 0 && a.window < a.kv_len ? a.window + C8_BLOCK - 1 : a.kv_len;
  const int64_t blocks = (span + C8_BLOCK - 1) / C8_BLOCK, items = (int64_t)a.batch * H;
  p.whole = blocks <= WHOLE_BLOCKS;
  int64_t grid = items;
  if (!p.whole) {
    grid = (int64_t)device_sms() * PER_SM;
    const int64_t most = (blocks * items + WARPS - 1) / WARPS;    // no fewer than one block per warp
    if (grid > most) grid = most;
    if ((size_t)grid * 2 * C::PSLOT * 4 > a.workspace_bytes) return POP_E_NOSPACE;
  }
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  static bool configured = false;
  if (!configured) {
    if (cudaFuncSetAttribute(dec8_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             C::SMEM + (MAX_BATCH + 1) * 4) != cudaSuccess ||
        cudaFuncSetAttribute(dec8_merge_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (MAX_BATCH + 1) * 4) !=
            cudaSuccess)
      return POP_E_CUDA;
    configured = true;
  }
  ProfScope prof(PROF_DECODE_ATTN, (double)a.batch * span * a.n_kv * (2.0 * HD + 0.125), s);
  if (launch_chained(dec8_kernel<HD>, dim3((unsigned)grid), dim3(WARPS * 32), (size_t)(C::SMEM + scan_bytes), s, p) !=
      cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  if (!p.whole) {
    if (launch_chained(dec8_merge_kernel<HD>, dim3((unsigned)grid), dim3(WARPS * 32), (size_t)scan_bytes, s, p) !=
        cudaSuccess)
      return POP_E_CUDA;
    count_launch();
  }
  return POP_OK;
}

}  // namespace

int launch_decode_attention8(const Attn8Args& a, cudaStream_t s) {
  if (!a.q || !a.out || !c8_cache_ok(a.c)) return POP_E_INVALID;
  if (a.batch < 1 || a.batch > MAX_BATCH || a.n_kv < 1 || a.n_q < 1 || a.n_q % a.n_kv || a.n_q > 65536 || a.kv_len < 0 ||
      a.kv_len > 0x7ffffff0 || a.window < 0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8)
    return POP_E_INVALID;
  if ((int64_t)a.kv_len > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  const int G = a.n_q / a.n_kv, hg = (G + MAXG - 1) / MAXG;
  const int64_t blocks = ((int64_t)a.kv_len + C8_BLOCK - 1) / C8_BLOCK;
  // block numbers, of the call and of the pool, are 32-bit
  if ((blocks > 0 ? blocks : 1) * a.batch > 0x7fffffff / ((int64_t)a.n_kv * hg) ||
      (int64_t)a.c.num_pages * a.n_kv > 0x7fffffff / (a.c.page_size / C8_BLOCK))
    return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.workspace) % 16) return POP_E_INVALID;
  Dec8Dev p{};
  p.q = a.q; p.ldq = a.ldq;
  p.c = a.c;
  p.seq_lens = a.seq_lens; p.kv_len = a.kv_len; p.window = a.window;
  p.out = a.out; p.ldo = a.ldo;
  p.batch = a.batch; p.n_q = a.n_q; p.n_kv = a.n_kv; p.G = G; p.hg = hg;
  p.partial = static_cast<float*>(a.workspace);
  p.scale_log2 = 1.4426950408889634f / sqrtf((float)a.head_dim);
  switch (a.head_dim) {
    case 64: return launch_t<64>(a, p, s);
    case 128: return launch_t<128>(a, p, s);
    default: return launch_t<256>(a, p, s);
  }
}

}  // namespace pop
