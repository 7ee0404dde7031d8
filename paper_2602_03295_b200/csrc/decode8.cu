// Single-query attention over the 8-bit paged cache (paper Eq. 1, Attn for the one position of a decode step).
//
// For sequence b with len positions, query head h of kv head g, and seen positions j in [max(0, len - window), len):
//   out[b][h] = sum_j p_j 2^(ev_j) v_j / sum_j p_j,   p_j = exp2(c q.k_j 2^(ek_j) - max),  c = log2(e) / sqrt(hd)
// with codes k_j, v_j and block exponents ek_j, ev_j. The V scale is folded into the exponent: with
// w_j = exp2(c q.k_j 2^(ek_j) + ev_j - m) and m the running maximum of that sum, out = sum w_j v_j / sum w_j 2^(-ev_j), so
// the weights that meet the tensor cores are at most 1 whatever the scales of the blocks are.
//
// Bound by the cache's bytes: 2 hd + 1/8 per kv head and position. A warp takes blocks of 16 positions of one (sequence,
// kv head, group of at most 8 query heads) and works on them straight from global memory: on the warp-level MMA the
// KEYS are the M side (S^T = K q^T, O^T = V^T P^T), a dot product does not see the order of its terms, so every lane
// loads 16 consecutive bytes of a key and two halves of a word feed one MMA; V codes of two keys are interleaved by byte
// permutes. Codes become f16 exactly (one conversion per pair), the query is scaled to f16 by a power of two per head
// (exact down to 2^-36 of its largest element), weights are f16 with 2^14 as the largest (half a step: 2^-12 relative);
// scores, statistics and sums are fp32. No shared memory is involved in the stream.
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
constexpr int MAX_BATCH = 16384;     // the block counts' prefix sums sit in shared memory
constexpr float W_SHIFT = 14.f;      // weights are stored times 2^14

template <int HD>
struct D8 {
  static constexpr int NT = HD / 16;           // MMAs along the head
  static constexpr int KC = HD / 64;           // 16-byte pieces of a key row per lane
  static constexpr int VW = HD / 32;           // words of a value row per lane
  static constexpr int HS = HD + 4;            // floats per head of a piece in shared memory: rows 4 banks apart
  static constexpr int SLOT = MAXG * HS + 2 * MAXG;
  static constexpr int PSLOT = MAXG * HD + 2 * MAXG;   // floats of a piece in the workspace
  static constexpr int SMEM = 2 * WARPS * SLOT * 4;
};

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

__device__ __forceinline__ uint4 ld_nc16(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld_nc8(const uint8_t* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
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
__device__ __forceinline__ int64_t total_units(const Dec8Dev& p, const int* prefix, int H) {
  if (p.seq_lens == nullptr) return (int64_t)span_of(p, 0).n * p.batch * H;
  return (int64_t)prefix[p.batch] * H;
}
// Where unit u (< total) of the line lies: sequence, item of the sequence (kv head and head group), block of the item
struct Place { int b, item, blk; Span s; };
__device__ __forceinline__ Place locate(const Dec8Dev& p, const int* prefix, int H, int64_t u) {
  Place x;
  int64_t before;
  if (p.seq_lens == nullptr) {
    const int64_t per = (int64_t)span_of(p, 0).n * H;
    x.b = (int)(u / per);
    before = x.b * per;
  } else {
    int lo = 0, hi = p.batch - 1;               // the last b with prefix[b] * H <= u: its span is not empty
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((int64_t)prefix[mid] * H <= u) lo = mid;
      else hi = mid - 1;
    }
    x.b = lo;
    before = (int64_t)prefix[lo] * H;
  }
  x.s = span_of(p, x.b);
  const int off = (int)(u - before);            // < 2^31: the host checks blocks * items
  x.item = off / x.s.n;
  x.blk = off - x.item * x.s.n;
  return x;
}

template <int HD>
__global__ void __launch_bounds__(WARPS * 32, HD == 64 ? 3 : (HD == 128 ? 2 : 1))
dec8_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD>;
  constexpr int NT = C::NT, KC = C::KC, VW = C::VW, HS = C::HS;
  extern __shared__ __align__(16) float slots[];              // [WARPS][2][SLOT], then the prefix sums
  __shared__ int warp_sums[WARPS];
  __shared__ int hdr_item[2 * WARPS], hdr_flags[2 * WARPS];   // flags: 1 holds the item's first block, 2 its last
  int* prefix = reinterpret_cast<int*>(slots + 2 * WARPS * C::SLOT);
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

  const int64_t T = total_units(p, prefix, H);
  int64_t u, u_end;
  if (p.whole) {                     // this CTA's item, its blocks dealt to the warps in stretches
    const int b = blockIdx.x / H, item = blockIdx.x - b * H;
    const Span s = span_of(p, b);
    const int64_t base = (p.seq_lens ? (int64_t)prefix[b] * H : (int64_t)b * H * s.n) + (int64_t)item * s.n;
    u = base + (int64_t)s.n * warp / WARPS;
    u_end = base + (int64_t)s.n * (warp + 1) / WARPS;
  } else {
    const int64_t W = (int64_t)gridDim.x * WARPS, w = (int64_t)blockIdx.x * WARPS + warp;
    u = T * w / W;
    u_end = T * (w + 1) / W;
  }

  while (u < u_end) {
    const Place x = locate(p, prefix, H, u);
    const int n_blk = (int)min((int64_t)(x.s.n - x.blk), u_end - u);
    const int kvh = x.item / p.hg, h0 = kvh * p.G + (x.item - kvh * p.hg) * MAXG;
    const int heads = min(MAXG, kvh * p.G + p.G - h0);
    const int32_t* bt = p.c.table + (int64_t)x.b * p.c.max_pages;
    const int last_page = (x.s.len - 1) / p.c.page_size;

    // coordinates of the block to load next; a table entry that is no page of the pool reads as zeros
    const int ps = p.c.page_size;
    int pos = (x.s.first + x.blk) * C8_BLOCK;
    int pi = pos / ps, slot = pos - pi * ps;
    auto entry = [&](int i) {
      const int page = i <= last_page ? bt[i] : 0;
      if ((unsigned)page < (unsigned)p.c.num_pages) return page;
      if (lane == 0) atomicMin(p.status, (int)POP_E_INVALID);
      return -1;
    };
    int page = entry(pi), ahead = entry(pi + 1);
    uint4 kr[2][KC];
    uint32_t vr[4][VW];
    int ke = 0, ve = 0;
    auto load_k = [&]() {              // keys g and g + 8 of the block, bytes 64 c + 16 t .. + 15
      if (page < 0) {
#pragma unroll
        for (int c = 0; c < KC; ++c) kr[0][c] = kr[1][c] = make_uint4(0, 0, 0, 0);
        return;
      }
      const int64_t tile = (int64_t)page * p.n_kv + kvh;
      const uint8_t* base = p.c.k + (tile * ps + slot + g) * HD + 16 * t;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        kr[0][c] = ld_nc16(base + 64 * c);
        kr[1][c] = ld_nc16(base + 8 * HD + 64 * c);
      }
      ke = p.c.ks[tile * (ps / C8_BLOCK) + slot / C8_BLOCK];
    };
    auto load_v = [&]() {              // values of keys 2t, 2t + 1, 2t + 8, 2t + 9, bytes g hd/8 .. + hd/8 - 1
      if (page < 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int w = 0; w < VW; ++w) vr[i][w] = 0;
        return;
      }
      const int64_t tile = (int64_t)page * p.n_kv + kvh;
      const uint8_t* base = p.c.v + (tile * ps + slot + 2 * t) * HD + g * (HD / 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint8_t* r = base + ((i & 1) + (i >> 1) * 8) * HD;
        if constexpr (VW == 2) {
          const uint2 v = ld_nc8(r);
          vr[i][0] = v.x; vr[i][1] = v.y;
        } else {
#pragma unroll
          for (int c = 0; c < VW / 4; ++c) {
            const uint4 v = ld_nc16(r + 16 * c);
            vr[i][4 * c] = v.x; vr[i][4 * c + 1] = v.y; vr[i][4 * c + 2] = v.z; vr[i][4 * c + 3] = v.w;
          }
        }
      }
      ve = p.c.vs[tile * (ps / C8_BLOCK) + slot / C8_BLOCK];
    };
    load_k();
    load_v();

    // q^T as the B operand: lane holds head g at dims 64 c + 16 t + 4 i + {0, 1} and {2, 3}, scaled so that the head's
    // largest element is in [2^12, 2^13)
    uint32_t qb[KC * 4][2];
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
      const float mul = g < heads ? c8_pow2(139 - eb) : 0.f, inv = c8_pow2(eb - 139) * p.scale_log2;
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t w[4] = {raw[c][i].x, raw[c][i].y, raw[c][i].z, raw[c][i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            qb[c * 4 + 2 * i + (k >> 1)][k & 1] = pack_half2(lo_f(w[k]) * mul, hi_f(w[k]) * mul);
        }
      c0 = __shfl_sync(FULL, inv, t * 8);
      c1 = __shfl_sync(FULL, inv, t * 8 + 4);
    }

    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    float o[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

    for (int i = 0; i < n_blk; ++i) {
      const bool more = i + 1 < n_blk;
      const int at = pos;                            // first position of the block in registers
      pos += C8_BLOCK;
      slot += C8_BLOCK;
      if (more && slot == ps) {
        slot = 0;
        ++pi;
        page = ahead;
        ahead = entry(pi + 1);
      }
      float s[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};   // two chains of dependent MMAs
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const uint32_t a[4] = {kr[0][c].x, kr[0][c].y, kr[0][c].z, kr[0][c].w};
        const uint32_t b[4] = {kr[1][c].x, kr[1][c].y, kr[1][c].z, kr[1][c].w};
#pragma unroll
        for (int w = 0; w < 4; ++w)
          mma_f16((w & 1) ? sb : s, c8_half2_lo(a[w]), c8_half2_lo(b[w]), c8_half2_hi(a[w]), c8_half2_hi(b[w]),
                  qb[c * 4 + w][0], qb[c * 4 + w][1]);
      }
      const float kf = c8_pow2(ke - 127), k0 = c0 * kf, k1 = c1 * kf;
      if (more) load_k();
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
      if (more) load_v();
    }
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      l0 += __shfl_xor_sync(FULL, l0, w);
      l1 += __shfl_xor_sync(FULL, l1, w);
    }
    // lane (g, t) holds heads 2t, 2t + 1 at dims g hd/8 .. + hd/8 - 1: o[j] is dims 2j ([0], [1]) and 2j + 1 ([2], [3])
    const bool starts = x.blk == 0, ends = x.blk + n_blk == x.s.n;
    if (starts && ends) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        if (2 * t + hh >= heads) continue;
        const float inv = 1.f / (hh ? l1 : l0);
        bf16* dst = p.out + (int64_t)x.b * p.ldo + (int64_t)(h0 + 2 * t + hh) * HD + g * (HD / 8);
#pragma unroll
        for (int j = 0; j < NT; ++j)
          *reinterpret_cast<__nv_bfloat162*>(dst + 2 * j) = __floats2bfloat162_rn(o[j][hh] * inv, o[j][2 + hh] * inv);
      }
    } else {
      const int si = 2 * warp + (starts ? 1 : 0);
      float* sl = slots + si * C::SLOT;
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
      const int h = e / (HD / 2), pr = e - h * (HD / 2);      // pair pr of the head: dims g hd/8 + 2 j, j = pr / 8, g = pr % 8
      float m = -INFINITY, l = 0.f;
      float2 v = make_float2(0.f, 0.f);
      for (int k = i; k <= last; ++k)
        if (hdr_item[k] == it) m = fmaxf(m, slots[k * C::SLOT + h]);
      for (int k = i; k <= last; ++k) {
        if (hdr_item[k] != it) continue;
        const float* sl = slots + k * C::SLOT;
        const float f = ex2(sl[h] - m);
        const float2 ov = *reinterpret_cast<const float2*>(sl + 2 * MAXG + h * HS + 2 * pr);
        l = fmaf(sl[MAXG + h], f, l);
        v.x = fmaf(ov.x, f, v.x);
        v.y = fmaf(ov.y, f, v.y);
      }
      if (starts && ends) {
        const float inv = 1.f / l;
        bf16* dst = p.out + (int64_t)b * p.ldo + (int64_t)(h0 + h) * HD + (pr & 7) * (HD / 8) + 2 * (pr >> 3);
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

// Items that cross CTAs: the CTA in which such an item starts (its number is this block's) merges the pieces of the
// CTAs behind it. Reads the same lengths, so it finds the same places.
template <int HD>
__global__ void __launch_bounds__(WARPS * 32) dec8_merge_kernel(const __grid_constant__ Dec8Dev p) {
  using C = D8<HD>;
  extern __shared__ __align__(16) float slots[];
  __shared__ int warp_sums[WARPS];
  int* prefix = reinterpret_cast<int*>(slots);
  chain_trigger();
  chain_wait();
  scan_blocks(p, prefix, warp_sums);
  const int H = p.n_kv * p.hg;
  const int64_t T = total_units(p, prefix, H), P = gridDim.x, c = blockIdx.x;
  const int64_t u0 = T * c / P, u1 = T * (c + 1) / P;
  if (u0 >= u1) return;
  const Place x = locate(p, prefix, H, u1 - 1);
  const int64_t first = u1 - 1 - x.blk;
  if (x.blk + 1 == x.s.n || first < u0) return;                 // nothing left over, or it started earlier
  const int64_t c1 = ((first + x.s.n) * P - 1) / T;             // CTA of the item's last block
  const int kvh = x.item / p.hg, h0 = kvh * p.G + (x.item - kvh * p.hg) * MAXG;
  const int heads = min(MAXG, kvh * p.G + p.G - h0);
  for (int e = threadIdx.x; e < heads * (HD / 2); e += blockDim.x) {
    const int h = e / (HD / 2), pr = e - h * (HD / 2);
    auto piece = [&](int64_t k) { return p.partial + (2 * k + (k == c ? 1 : 0)) * C::PSLOT; };
    float m = -INFINITY, l = 0.f;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int64_t k = c; k <= c1; ++k) {
      if (T * k / P == T * (k + 1) / P) continue;     // fewer blocks than CTAs: this one had none
      const float* sl = piece(k);
      const float mk = __ldcg(sl + h), lk = __ldcg(sl + MAXG + h);
      const float2 ov = __ldcg(reinterpret_cast<const float2*>(sl + 2 * MAXG + h * HD + 2 * pr));
      const float n = fmaxf(m, mk), fa = ex2(m - n), fb = ex2(mk - n);
      l = l * fa + lk * fb;
      v.x = v.x * fa + ov.x * fb;
      v.y = v.y * fa + ov.y * fb;
      m = n;
    }
    const float inv = 1.f / l;
    bf16* dst = p.out + (int64_t)x.b * p.ldo + (int64_t)(h0 + h) * HD + (pr & 7) * (HD / 8) + 2 * (pr >> 3);
    *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(v.x * inv, v.y * inv);
  }
}

// Short caches: one CTA per item and no second launch, up to this many blocks of the longest span.
constexpr int WHOLE_BLOCKS = 32;

template <int HD>
int launch_t(const Attn8Args& a, Dec8Dev& p, cudaStream_t s) {
  using C = D8<HD>;
  constexpr int PER_SM = HD == 64 ? 3 : (HD == 128 ? 2 : 1);
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
  if (blocks * a.n_kv * hg > 0x7fffffff || blocks * a.batch > 0x7fffffff || (int64_t)a.batch * a.n_kv * hg > 0x7fffffff)
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
