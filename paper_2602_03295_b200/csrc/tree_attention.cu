// Attention of drafted tokens over the bf16 paged cache (Attn of paper Eq. 1 for several rows of a sequence that form a tree):
// row i of a sequence sees the cached positions in front of the draft, and of the drafted slots those whose bit its mask has.
//
// A tile is 128 (row, head) pairs of one kv head: K and V are read once for all of them. Few rows over a long cache are bound
// by the cache's bytes, so what counts is that every SM reads all the time, whatever the sequences' lengths: the key tiles of
// all (sequence, kv head, row tile) items form one line, and each CTA takes an equal stretch of it. An item that lies in one
// stretch is finished there; the others leave (maximum, sum, output) of their part, and a second launch joins the parts. Short
// items that fit the CTAs are not cut at all.
// Warps of a CTA:
//   4 softmax warps, a thread per (row, head): scores of 64 keys from TMEM, mask, maximum, exponentials, P in bf16 back over
//       the scores. These dependent steps (1700 clocks) are what a CTA waits for; where a second CTA shares the SM that is
//       hidden, else (hd 256) 8 warps take half of the keys each, and join their maxima through shared memory (16 x 12 rows,
//       window 1024: 8 % less; with two CTAs on the SM it costs: 24 x 27 rows of up to 12001 9 % more);
//   1 TMA warp: the CTA's place in the line, then Q of an item and K and V tiles of 64 positions through a ring, in the order in
//       which they are used;
//   1 MMA warp: scores two tiles ahead of the softmax, across the ends of items too, and O += P V with P from TMEM.
#include "ptx.cuh"
#include "tree.cuh"

namespace pop {
namespace {

constexpr int BKV = 64;

template <int HD>
struct TC {
  static constexpr int KV_TILE_BYTES = BKV * HD * 2;
  static constexpr int KV_SUB_BYTES = BKV * 128;       // one 64-wide slice of head_dim
  static constexpr int Q_TILE_BYTES = 128 * HD * 2;
  static constexpr int O_COL = 2 * BKV;                // scores of tile f at (f & 1) * 64, O behind them
  static constexpr uint32_t TMEM_COLS = O_COL + HD <= 256 ? 256 : 512;
  static constexpr int PER_SM = TMEM_COLS == 256 ? 2 : 1;        // one CTA's beginnings and ends beside the other's keys
  static constexpr int RING_BYTES = (PER_SM == 2 ? 113 : 227) * 1024 - 4 * 1024 - Q_TILE_BYTES;
  static constexpr int STAGES = RING_BYTES / KV_TILE_BYTES < 12 ? RING_BYTES / KV_TILE_BYTES : 12;
  static constexpr int HALVES = PER_SM == 2 ? 1 : 2;   // threads that share a row's keys of a tile
  static constexpr int KEYS = BKV / HALVES;
  static constexpr int THREADS = HALVES * 128 + 64;
  static_assert(STAGES >= 4, "ring too shallow");
};

// One sequence of the line
struct Seq {
  int row0, n, start;           // packed rows, positions in front of them
  int j_lo, tiles, qts;         // first key tile, key tiles of an item, items per kv head
};

// Where a CTA's stretch of the line begins
struct Plan {
  int lo, hi;                   // its places in the line; nothing to do where they are equal
  int b, base;                  // the sequence at lo, and where that one begins
  Seq x;
};

template <int HD>
struct __align__(1024) TreeSmem {
  using C = TC<HD>;
  uint8_t q[C::Q_TILE_BYTES];
  uint8_t kv[C::STAGES][C::KV_TILE_BYTES];
  uint64_t q_full, q_empty;
  uint64_t kv_full[C::STAGES];
  uint64_t kv_empty[C::STAGES];
  uint64_t s_full[2];           // scores of tile f in buffer f & 1, phase f >> 1; the same for the two below
  uint64_t p_ready[2];          // P over the scores (one arrival per softmax warp)
  uint64_t pv_done[2];          // O += P V complete
  float half_max[2][2][128];    // [tile & 1][half of its keys][row]
  float half_sum[128];
  volatile uint32_t half_lost[4][2];      // [quarter][meeting & 1]: a half of the rows has given up
  Plan plan;
  uint32_t tmem_base;
  uint32_t raised;
  volatile uint32_t abort;
};

struct TreeDev {
  TreeAttnArgs a;
  int G, per;                   // query heads per kv head, rows of an item: a tile of 128 pairs
  int rows_per_load;            // positions of a TMA load: min(page_size, 64)
  int room;                     // positions that a row of the block table has pages for
  int ctas;
  int whole;                    // CTA c has item c and nothing else: no parts, and no second launch
  float scale_log2;             // log2(e) / sqrt(hd)
  float* partial;               // [2 per CTA] parts
  int* starts;                  // [batch + 1]: see plan_of
  int* status;
};

// Floats of a part: [hd / 4][128 rows][4] of the output, then maximum and sum as [128][4], two of them used. Neighbouring lanes
// have neighbouring rows, so that what they write and read together lies together.
__host__ __device__ constexpr int part_floats(int hd) { return (hd + 4) * 128; }

// Fewest tiles of a stretch: below, beginning and ending it costs more than its keys
constexpr int MIN_SHARE = 2;
// Where no item has more tiles than this and there are no more items than CTAs, each CTA has an item, and nothing is to be joined. us
// so / in stretches: 1 x 5 rows of 50 5.7 / 11.0, 8 x 16 of up to 100 8.0 / 12.8, 1 x 5 of 180 7.2 / 9.6 (pages of 16: 10.8 / 11.3); with
// four tiles 1 x 5 of 240 8.4 / 7.8 (13.3 / 10.2)
constexpr int WHOLE_TILES = 3;

__device__ __forceinline__ Seq seq_of(const TreeDev& p, int b, bool report) {
  const Drafts& d = p.a.d;
  Seq x;
  x.row0 = d.cu ? __ldg(d.cu + b) : b * d.max_rows;
  x.n = d.cu ? __ldg(d.cu + b + 1) - x.row0 : d.max_rows;
  x.start = d.start ? __ldg(d.start + b) : d.pos0;
  x.j_lo = x.tiles = x.qts = 0;
  if (x.n <= 0) return x;                                      // no rows: whatever the rest is
  if (x.n > d.max_rows || x.row0 < 0 || x.row0 > d.rows - x.n || x.start < 0 || x.start > d.pos0 ||
      x.start > p.room - x.n) {
    if (report) atomicMin(p.status, (int)POP_E_INVALID);
    x.n = 0;
    return x;
  }
  x.j_lo = p.a.window > 0 ? max(0, x.start - p.a.window + 1) / BKV : 0;
  x.tiles = (x.start + x.n - 1) / BKV - x.j_lo + 1;
  x.qts = (x.n + p.per - 1) / p.per;
  return x;
}
__device__ __forceinline__ int line_of(const TreeDev& p, const Seq& x) { return x.tiles * x.qts * p.a.n_kv; }
// places of a sequence in what the CTAs share out
__device__ __forceinline__ int places_of(const TreeDev& p, const Seq& x) { return p.whole ? x.qts * p.a.n_kv : line_of(p, x); }

__device__ __forceinline__ int warp_add(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// from the item that a CTA has to its tiles
__device__ __forceinline__ void item_of(Plan& r) {
  if (r.lo >= r.hi) return;
  r.lo = (r.lo - r.base) * r.x.tiles;
  r.hi = r.lo + r.x.tiles;
  r.base = 0;
}
// Finds the stretch of CTA `cta`, by a whole warp. `starts`, if given, gets the place where each sequence begins and, behind them,
// the tiles of a stretch: what the second launch asks for.
__device__ __forceinline__ Plan plan_of(const TreeDev& p, int cta, int* starts) {
  const int lane = threadIdx.x & 31, batch = p.a.d.batch;
  if (batch == 1) {                                            // nothing to add up (4 % of 1 x 5 rows of 300)
    Plan r;
    r.x = seq_of(p, 0, cta == 0 && lane == 0);
    const int total = places_of(p, r.x), share = p.whole ? 1 : max((total + p.ctas - 1) / p.ctas, MIN_SHARE);
    r.lo = (int)min((int64_t)cta * share, (int64_t)total);
    r.hi = min(r.lo + share, total);
    r.b = r.base = 0;
    if (starts != nullptr && lane == 0) {
      starts[0] = 0;
      starts[1] = share;
    }
    if (p.whole) item_of(r);
    return r;
  }
  Seq x;
  int mine = 0, total = 0;
  for (int b0 = 0; b0 < batch; b0 += 32) {
    mine = 0;
    if (b0 + lane < batch) {
      x = seq_of(p, b0 + lane, cta == 0);
      mine = places_of(p, x);
    }
    total += warp_add(mine);
  }
  const int share = p.whole ? 1 : max((total + p.ctas - 1) / p.ctas, MIN_SHARE);
  Plan r;
  r.lo = (int)min((int64_t)cta * share, (int64_t)total);
  r.hi = min(r.lo + share, total);
  r.b = -1;
  int base = 0;
  for (int b0 = 0; b0 < batch; b0 += 32) {
    if (batch > 32) {                                          // else the first loop's are still there
      mine = 0;
      if (b0 + lane < batch) {
        x = seq_of(p, b0 + lane, false);
        mine = places_of(p, x);
      }
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (starts != nullptr && b0 + lane < batch) starts[b0 + lane] = base + incl - mine;
    const uint32_t past = __ballot_sync(0xffffffffu, base + incl > r.lo);
    if (past != 0 && r.b < 0) {
      const int at = __ffs(past) - 1;
      r.b = b0 + at;
      r.base = base + __shfl_sync(0xffffffffu, incl - mine, at);
      r.x.row0 = __shfl_sync(0xffffffffu, x.row0, at);
      r.x.n = __shfl_sync(0xffffffffu, x.n, at);
      r.x.start = __shfl_sync(0xffffffffu, x.start, at);
      r.x.j_lo = __shfl_sync(0xffffffffu, x.j_lo, at);
      r.x.tiles = __shfl_sync(0xffffffffu, x.tiles, at);
      r.x.qts = __shfl_sync(0xffffffffu, x.qts, at);
      if (starts == nullptr) break;
    }
    base += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (starts != nullptr && lane == 0) starts[batch] = share;
  if (p.whole) item_of(r);
  return r;
}

// A walk over a stretch of the line, tile by tile, the same for all lanes
struct Walk {
  Seq x;
  int b, left;                  // sequence; its tiles from here on
  int pos, hi;                  // place in the line, end of the stretch
  int kvh, q0;                  // the item: kv head, first row
  int j, j_end;                 // key tile (absolute), end of the segment
  int j_item_end;
  __device__ __forceinline__ void item(const TreeDev& p, int off) {
    const int it = off / x.tiles, r = off - it * x.tiles;
    kvh = it / x.qts;
    q0 = (it - kvh * x.qts) * p.per;
    j = x.j_lo + r;
    j_item_end = x.j_lo + x.tiles;
    j_end = min(j_item_end, j + hi - pos);
    left = line_of(p, x) - off;
  }
  __device__ __forceinline__ void begin(const TreeDev& p, const Plan& at) {
    x = at.x;
    b = at.b;
    pos = at.lo;
    hi = at.hi;
    item(p, at.lo - at.base);
  }
  // to the next tile; true where another segment begins there
  __device__ __forceinline__ bool next(const TreeDev& p) {
    if (j + 1 < j_end) {
      ++pos;
      --left;
      ++j;
      return false;
    }
    return segment(p);
  }
  // to the next segment
  __device__ __forceinline__ bool segment(const TreeDev& p) {
    pos += j_end - j;
    left -= j_end - j;
    if (pos >= hi) return true;
    if (left == 0) {
      do {
        x = seq_of(p, ++b, false);
      } while (x.tiles == 0);                                  // pos lies in front of the line's end, so one follows
      item(p, 0);
    } else {
      item(p, line_of(p, x) - left);
    }
    return true;
  }
};

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
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint64_t ones(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ __forceinline__ bool gave_up(int status) { return status <= (int)POP_E_DEVICE_TIMEOUT; }

// The first words of a row's mask, asked for where its segment begins: a tile of the draft comes long after
struct Words {
  uint32_t w[4];
};

// Which of the 64 positions from kv0 on row i (packed row `row`) of the sequence sees. One body, not unrolled by halves: its
// instructions are met cold, and a launch waits for the CTAs that have the drafts.
__device__ __forceinline__ uint64_t seen_of(const TreeDev& p, const Seq& x, int i, int64_t row, const Words& first, int depth, int kv0) {
  const int ctx = x.start - kv0;                               // positions of these in front of the draft
  const int window = p.a.window;
  uint64_t vis = ~0ull;
  if (ctx < 64) {
    if (p.a.mask == nullptr) {
      vis = ones(ctx + i + 1);
    } else {
      const int slot0 = ctx < 0 ? -ctx : 0, w = slot0 >> 5;
      uint32_t a = first.w[0], b = first.w[1], c = first.w[2];
      if (w == 1) {
        a = b;
        b = c;
        c = first.w[3];
      } else if (w > 1) {
        const uint32_t* m = p.a.mask + row * p.a.mask_words;
        auto word = [&](int k) { return k < p.a.mask_words ? __ldg(m + k) : 0u; };
        a = word(w);
        b = word(w + 1);
        c = word(w + 2);
      }
      vis = ((uint64_t)__funnelshift_r(b, c, slot0 & 31) << 32) | __funnelshift_r(a, b, slot0 & 31);
      if (ctx > 0) vis = (vis << ctx) | ones(ctx);
    }
    vis &= ones(ctx + x.n);
  }
  if (window > 0) {
    const int hidden = ctx > 0 ? ctx + depth - window + 1 : 0; // positions in front of the window
    if (hidden > 0) vis &= ~ones(min(hidden, ctx));
    if (ctx < 64 && depth >= window) {                         // drafted slots that lie so far up the tree
      for (uint64_t m = vis & ~ones(ctx); m != 0; m &= m - 1) {
        const int k = __ffsll((long long)m) - 1, slot = k - ctx;
        const int d = p.a.d.depth ? __ldg(p.a.d.depth + x.row0 + slot) : slot;
        if (d <= depth - window) vis &= ~(1ull << k);
      }
    }
  }
  return vis;
}

#define TREE_ABORT(S, status)                         \
  do {                                                \
    (S).abort = 1;                                    \
    atomicMin((status), (int)POP_E_DEVICE_TIMEOUT);   \
  } while (0)

// waits for, or only counts towards, a barrier of `n` threads
__device__ __forceinline__ void named_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void named_arrive(int id, int n) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(n) : "memory"); }

template <int HD>
__global__ void __launch_bounds__(TC<HD>::THREADS, TC<HD>::PER_SM)
tree_attn_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeDev p) {
  using C = TC<HD>;
  constexpr int STAGES = C::STAGES, HALVES = C::HALVES, KEYS = C::KEYS, TMA_WARP = 4 * HALVES, MMA_WARP = TMA_WARP + 1, PLAN_BAR = 1, PAIR_BAR = 2;     // PAIR_BAR + quarter
  extern __shared__ uint8_t smem_raw[];
  TreeSmem<HD>& s = *reinterpret_cast<TreeSmem<HD>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  chain_trigger();
  Plan plan;
  plan.lo = plan.hi = 0;
  if (warp == TMA_WARP) {
    if (lane == 0) {
      mbar_init(&s.q_full, 1);
      mbar_init(&s.q_empty, 1);
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(&s.kv_full[i], 1);
        mbar_init(&s.kv_empty[i], 1);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s.s_full[i], 1);
        mbar_init(&s.p_ready[i], 4 * HALVES);
        mbar_init(&s.pv_done[i], 1);
      }
      s.abort = 0;
      for (int i = 0; i < 8; ++i) s.half_lost[i >> 1][i & 1] = 0;
      fence_barrier_init();
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      prefetch_tmap(&tmV);
    }
    __syncwarp();
    chain_wait();
    const int raised = lane == 0 ? *reinterpret_cast<const volatile int*>(p.status) : 0;
    plan = plan_of(p, blockIdx.x, blockIdx.x == 0 && !p.whole ? p.starts : nullptr);
    if (__shfl_sync(0xffffffffu, gave_up(raised) ? 1 : 0, 0)) plan.hi = plan.lo;     // a call that is not to run
    if (lane == 0) s.plan = plan;
    __syncwarp();
    named_arrive(PLAN_BAR, C::THREADS);
  } else {
    chain_wait();
    if (warp == MMA_WARP) {
      // columns that a CTA of another call has not given back yet are waited for: that CTA waits for nobody
      tmem_alloc(&s.tmem_base, C::TMEM_COLS);
      tmem_relinquish();
    }
    tc_fence_before();
    named_sync(PLAN_BAR, C::THREADS);
    tc_fence_after();
  }
  const uint32_t tmem_base = s.tmem_base;
  const int lo = warp == TMA_WARP ? plan.lo : s.plan.lo, hi = warp == TMA_WARP ? plan.hi : s.plan.hi, n_tiles = hi - lo;
  const bool nothing = n_tiles <= 0;

  if (nothing) {
    // beyond the line's end
  } else if (warp == TMA_WARP) {
    // ------------------------------------------------------------------ TMA: K_0, K_1, then V_f, K_{f+2}
    Walk kw, vw;
    kw.begin(p, plan);
    vw = kw;
    const int log_rows = p.rows_per_load == 64 ? 6 : p.rows_per_load == 32 ? 5 : 4, log_loads = 6 - log_rows, loads = 1 << log_loads;
    int ring = 0, items = 0;
    bool ok = true;
    // Pages of the next 32 loads of a sequence, an entry per lane, and of the 32 behind them
    struct Ahead {
      int b = -1, first = 0, pg0 = 0, pg1 = 0;
    } k_ahead, v_ahead;
    auto entry = [&](const Walk& w, int load) {
      const int at = load << log_rows;
      return at < w.x.start + w.x.n ? __ldg(p.a.c.table + (int64_t)w.b * p.a.c.max_pages + (uint32_t)at / (uint32_t)p.a.c.page_size) : 0;
    };
    auto load_tile = [&](const Walk& w, Ahead& ahead, const CUtensorMap* tm) {
      const int stage = ring % STAGES;
      const uint32_t phase = (ring / STAGES) & 1;
      ++ring;
      const int l0 = w.j << log_loads;
      if (ahead.b != w.b || l0 < ahead.first || l0 >= ahead.first + 64) {
        ahead.b = w.b;
        ahead.first = l0;
        ahead.pg0 = entry(w, l0 + lane);
        ahead.pg1 = entry(w, l0 + 32 + lane);
      } else if (l0 >= ahead.first + 32) {
        ahead.first += 32;
        ahead.pg0 = ahead.pg1;
        ahead.pg1 = entry(w, ahead.first + 32 + lane);
      }
      const int kv0 = w.j * BKV, live = min(loads, (w.x.start + w.x.n - kv0 + p.rows_per_load - 1) >> log_rows);
      // Pages in front of every row's window may have been given back: they are not looked at. What the ring has in their
      // places is masked (K) and cleared (V); the load that has the window's first position is always among the live ones.
      const int from = p.a.window > 0 ? max(0, max(0, w.x.start - p.a.window + 1) - kv0) >> log_rows : 0;
      if (!warp_agrees(mbar_wait_relaxed(&s.kv_empty[stage], phase ^ 1))) {
        ok = false;
        return;
      }
      if (lane == 0) mbar_expect_tx(&s.kv_full[stage], (live - from) * p.rows_per_load * HD * 2);
      for (int r = from; r < live; ++r) {
        const int k = l0 + r - ahead.first;
        const int page = k < 32 ? __shfl_sync(0xffffffffu, ahead.pg0, k) : __shfl_sync(0xffffffffu, ahead.pg1, k - 32);
        if (lane == 0) {
          // an entry outside the pool is clipped by the tensor map (it reads as zeros), but it is an error
          if ((unsigned)page >= (unsigned)p.a.c.num_pages) atomicMin(p.status, (int)POP_E_INVALID);
          for (int c = 0; c < HD / 64; ++c)
            tma_load_4d(s.kv[stage] + c * C::KV_SUB_BYTES + r * p.rows_per_load * 128, tm, &s.kv_full[stage], c * 64,
                        w.kvh, (uint32_t)(kv0 + r * p.rows_per_load) % (uint32_t)p.a.c.page_size, page);
        }
      }
    };
    auto load_q = [&](const Walk& w) {
      if (items > 0 && !warp_agrees(mbar_wait_relaxed(&s.q_empty, (items - 1) & 1))) {
        ok = false;
        return;
      }
      ++items;
      if (lane == 0) {
        mbar_expect_tx(&s.q_full, p.per * p.G * HD * 2);
        for (int c = 0; c < HD / 64; ++c)
          tma_load_3d(s.q + c * 16384, &tmQ, &s.q_full, c * 64, w.kvh * p.G, w.x.row0 + w.q0);
      }
    };
    bool fresh = true;
    int kf = 0;
    auto load_k = [&] {
      if (fresh) load_q(kw);
      if (ok) load_tile(kw, k_ahead, &tmK);
      ++kf;
      fresh = kw.next(p);
    };
    load_k();
    if (ok && kf < n_tiles) load_k();
    for (int f = 0; f < n_tiles && ok; ++f) {
      load_tile(vw, v_ahead, &tmV);
      vw.next(p);
      if (ok && kf < n_tiles) load_k();
    }
    if (!ok) TREE_ABORT(s, p.status);
  } else if (warp == MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuer (whole warp, elected lane)
    Walk sw, pw;
    sw.begin(p, s.plan);
    pw = sw;
    const uint32_t leader = elect_one();
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, BKV, 0, 0);
    constexpr uint32_t idesc_o = umma_idesc_bf16(128, HD, 0, 1);
    const uint64_t q_desc = umma_smem_desc(smem_u32(s.q), 16, 1024);
    const uint64_t k_desc0 = umma_smem_desc(smem_u32(s.kv[0]), 16, 1024);                 // K-major
    const uint64_t v_desc0 = umma_smem_desc(smem_u32(s.kv[0]), C::KV_SUB_BYTES, 1024);    // MN-major
    auto issue_s = [&](int f, int stage) {
      const uint64_t kd = k_desc0 + uint64_t(stage * (C::KV_TILE_BYTES >> 4));
      const uint32_t d = tmem_base + (f & 1) * BKV;
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk)
        umma_bf16_ss_w(leader, d, q_desc + uint64_t(((kk >> 2) * 16384 + (kk & 3) * 32) >> 4),
                       kd + uint64_t(((kk >> 2) * C::KV_SUB_BYTES + (kk & 3) * 32) >> 4), idesc_s, kk > 0 ? 1u : 0u);
      umma_commit_w(leader, &s.s_full[f & 1]);
    };
    auto issue_pv = [&](int f, int stage, bool begins) {
      const uint32_t pa = tmem_base + (f & 1) * BKV;
      const uint64_t vd = v_desc0 + uint64_t(stage * (C::KV_TILE_BYTES >> 4));
#pragma unroll
      for (int kk = 0; kk < BKV / 16; ++kk)
        umma_bf16_ts_w(leader, tmem_base + C::O_COL, pa + kk * 8, vd + uint64_t((kk * 2048) >> 4), idesc_o, (!begins || kk > 0) ? 1u : 0u);
      umma_commit_w(leader, &s.pv_done[f & 1]);
    };
    int ring = 0, sf = 0, items = 0;
    bool ok = true, s_fresh = true, p_fresh = true;
    auto wait_tile = [&](int& stage) {
      stage = ring % STAGES;
      const uint32_t phase = (ring / STAGES) & 1;
      ++ring;
      return mbar_wait(&s.kv_full[stage], phase);
    };
    // Scores of the next tile into the buffer that the tile two in front of it has left: its product is issued, and the
    // tensor pipe runs in order. The first wait of an item is for its queries.
    auto scores = [&] {
      if (s_fresh) ok = mbar_wait(&s.q_full, items++ & 1);
      int stage = 0;
      if (ok) ok = wait_tile(stage);
      if (!ok) return;
      tc_fence_after();
      issue_s(sf, stage);
      umma_commit_w(leader, &s.kv_empty[stage]);
      ++sf;
      s_fresh = sw.next(p);
      if (s_fresh) umma_commit_w(leader, &s.q_empty);
    };
    scores();
    if (ok && sf < n_tiles) scores();
    for (int f = 0; f < n_tiles && ok && !s.abort; ++f) {
      int stage = 0;
      ok = wait_tile(stage);
      if (ok) ok = mbar_wait(&s.p_ready[f & 1], (f >> 1) & 1);
      if (!ok) break;
      tc_fence_after();
      issue_pv(f, stage, p_fresh);
      umma_commit_w(leader, &s.kv_empty[stage]);
      p_fresh = pw.next(p);
      if (sf < n_tiles) scores();
    }
    if (!ok) TREE_ABORT(s, p.status);
  } else {
    // ------------------------------------------------------------------ softmax
    Walk w;
    w.begin(p, s.plan);
    const int half = warp >> 2, quarter = warp & 3;       // half of a tile's keys
    const int row = quarter * 32 + lane;                  // pair of the tile == TMEM lane
    const int ip = row / p.G, h = row - ip * p.G;         // row of the tile, head of the kv head
    const uint32_t lane_addr = uint32_t(quarter * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_addr;
    const uint32_t o_addr = tmem_base + lane_addr + C::O_COL + half * (HD / HALVES);
    bool ok = true;
    // Where two warps share rows, they meet at a barrier that knows no limit: neither leaves except behind a meeting, at which each
    // tells whether it goes on. The word of a meeting is written again two meetings later, when the other half has read it.
    int meetings = 0;
    auto meet = [&](bool fine) {
      volatile uint32_t& lost = s.half_lost[quarter][meetings++ & 1];
      if (!fine) lost = 1;
      named_sync(PAIR_BAR + quarter, 64);
      return lost == 0;
    };
    auto wait_pv = [&](int f) { return warp_agrees(mbar_wait(&s.pv_done[f & 1], (f >> 1) & 1)); };
    int f = 0;
    while (f < n_tiles && ok) {
      // ---- a segment: the tiles of one item that lie in this stretch
      const Seq x = w.x;
      const int kvh = w.kvh, j0 = w.j, nt = w.j_end - w.j, i = w.q0 + ip;
      const bool whole = j0 == x.j_lo && w.j_end == w.j_item_end;
      const int slot = 2 * (int)blockIdx.x + (f > 0 ? 1 : 0);
      const bool used = ip < p.per && i < x.n;
      const bool idle = !__any_sync(0xffffffffu, used);   // a warp without rows only keeps the barriers going
      const bool paired = HALVES == 2 && !idle;
      const int64_t prow = (int64_t)x.row0 + i;
      const int depth = !used || p.a.window == 0 ? 0 : p.a.d.depth ? min(max(__ldg(p.a.d.depth + prow), 0), 0xffff) : i;
      const int win_lo = p.a.window > 0 ? x.start - p.a.window + 1 : 0;      // in front of every row's window
      const int len = x.start + x.n;
      Words first = {{0, 0, 0, 0}};
      if (used && p.a.mask != nullptr && w.j_end * BKV > x.start) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < p.a.mask_words) first.w[k] = __ldg(p.a.mask + prow * p.a.mask_words + k);
      }
      float m_run = -INFINITY, l_run = 0.f;
      for (int jj = 0; jj < nt; ++jj, ++f) {
        const int kv0 = (j0 + jj) * BKV;
        const uint32_t sp_addr = s_addr + (f & 1) * BKV;
        uint32_t vis[KEYS / 32];
#pragma unroll
        for (int c = 0; c < KEYS / 32; ++c) vis[c] = used ? ~0u : 0u;
        if (used && (kv0 + BKV > x.start || (p.a.window > 0 && kv0 <= x.start + depth - p.a.window))) {
          const uint64_t v = seen_of(p, x, i, prow, first, depth, kv0);
          if constexpr (HALVES == 2) {
            vis[0] = half ? (uint32_t)(v >> 32) : (uint32_t)v;
          } else {
            vis[0] = (uint32_t)v;
            vis[KEYS / 32 - 1] = (uint32_t)(v >> 32);
          }
        }
        if (ok) ok = warp_agrees(mbar_wait(&s.s_full[f & 1], (f >> 1) & 1));
        if (!ok && !paired) break;
        if (!idle) {
          tc_fence_after();
          float sv[KEYS];
#pragma unroll
          for (int c = 0; c < KEYS / 32; ++c)
            tmem_ld_32x32b_x32(sp_addr + half * KEYS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[c * 32]));
          tmem_wait_ld();
          if ((vis[0] & vis[KEYS / 32 - 1]) != ~0u) {
#pragma unroll
            for (int k = 0; k < KEYS; ++k)
              if (!((vis[k / 32] >> (k & 31)) & 1u)) sv[k] = -INFINITY;
          }
          float mx0 = sv[0], mx1 = sv[2], mx2 = sv[4], mx3 = sv[6];
#pragma unroll
          for (int c = 0; c < KEYS / 8; ++c) {
            mx0 = max3(mx0, sv[c * 8 + 0], sv[c * 8 + 1]);
            mx1 = max3(mx1, sv[c * 8 + 2], sv[c * 8 + 3]);
            mx2 = max3(mx2, sv[c * 8 + 4], sv[c * 8 + 5]);
            mx3 = max3(mx3, sv[c * 8 + 6], sv[c * 8 + 7]);
          }
          float mine = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
          if constexpr (HALVES == 2) {
            // the other half's maximum; behind this barrier both halves have their scores, and P may overwrite them
            s.half_max[f & 1][half][row] = mine;
            tc_fence_before();
            ok = meet(ok);
            if (!ok) break;
            tc_fence_after();
            mine = fmaxf(mine, s.half_max[f & 1][half ^ 1][row]);
          }
          const float m_new = fmaxf(m_run, mine * p.scale_log2);
          const bool need = (m_new - m_run > 8.0f) || (m_run == -INFINITY && m_new > -INFINITY);
          if (__any_sync(0xffffffffu, need)) {
            // the maximum grew by more than 2^8 somewhere in these rows: bring the accumulator to the new one
            const float factor = (m_new == -INFINITY) ? 1.0f : ex2(m_run - m_new);   // ex2(-inf) = 0
            if (jj > 0) {
              ok = wait_pv(f - 1);
              if (!ok && !paired) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < HD / HALVES / 32; ++c) {
                uint32_t o[32];
                tmem_ld_32x32b_x32(o_addr + c * 32, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * factor);
                tmem_st_32x32b_x32(o_addr + c * 32, o);
              }
              tmem_wait_st();
            }
            l_run *= factor;
            m_run = m_new;
          }
          // P = exp2(S * scale - m): enters the product as bf16, its sum is taken in fp32 before that rounding
          const float m_use = m_run == -INFINITY ? 0.f : m_run;
          const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nm2 = make_float2(-m_use, -m_use);
          float2 acc0 = make_float2(0.f, 0.f), acc1 = make_float2(0.f, 0.f);
          uint32_t pk[KEYS / 2];
#pragma unroll
          for (int c = 0; c < KEYS / 4; ++c) {
            float2 x0 = __ffma2_rn(make_float2(sv[c * 4 + 0], sv[c * 4 + 1]), sc2, nm2);
            float2 x1 = __ffma2_rn(make_float2(sv[c * 4 + 2], sv[c * 4 + 3]), sc2, nm2);
            x0.x = ex2(x0.x); x0.y = ex2(x0.y);
            x1.x = ex2(x1.x); x1.y = ex2(x1.y);
            acc0 = __fadd2_rn(acc0, x0);
            acc1 = __fadd2_rn(acc1, x1);
            pk[c * 2 + 0] = pack2(x0.x, x0.y);
            pk[c * 2 + 1] = pack2(x1.x, x1.y);
          }
          l_run += (acc0.x + acc0.y) + (acc1.x + acc1.y);
          if constexpr (HALVES == 2) tmem_st_32x32b_x16(sp_addr + half * 16, pk);
          else tmem_st_32x32b_x32(sp_addr, pk);
          tmem_wait_st();
        }
        // positions behind the sequence's end or in front of every window may hold anything: zeros in the staged V tile, so
        // that 0 * garbage cannot reach the accumulator. V_f is entry min(f + 2, n_tiles) + f of the ring.
        if (warp < 2 && (kv0 + BKV > len || kv0 < win_lo)) {
          const int rv = min(f + 2, n_tiles) + f;
          if (ok) ok = warp_agrees(mbar_wait(&s.kv_full[rv % STAGES], (rv / STAGES) & 1));
          if (!ok && !paired) break;
          if (kv0 + row >= len || kv0 + row < win_lo) {
#pragma unroll 1
            for (int c = 0; c < HD / 64; ++c) {
              uint4* dst = reinterpret_cast<uint4*>(s.kv[rv % STAGES] + c * C::KV_SUB_BYTES + row * 128);
#pragma unroll
              for (int q = 0; q < 8; ++q) dst[q ^ (row & 7)] = make_uint4(0, 0, 0, 0);       // neighbours in other banks
            }
          }
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.p_ready[f & 1]);
      }
      if (ok) ok = wait_pv(f - 1);
      if (!ok && !paired) break;
      if (!idle) {
        tc_fence_after();
        if constexpr (HALVES == 2) {                      // the sum of both halves, the first half's first
          if (half == 1) s.half_sum[row] = l_run;
          ok = meet(ok);
          if (!ok) break;
          if (half == 0) {
            l_run += s.half_sum[row];
            s.half_sum[row] = l_run;
          }
          meet(true);
          l_run = s.half_sum[row];
        }
        const bool none = l_run == 0.f;                   // a row that sees nothing is a row of zeros
        const float inv = none ? 0.f : 1.0f / l_run;
        bf16* out = p.a.out + prow * p.a.ldo + (int64_t)(kvh * p.G + h) * HD + half * (HD / HALVES);
        float* part = p.partial + (int64_t)slot * part_floats(HD) + row * 4;     // four columns of all rows, then the next
        if (used && !whole && half == 0) *reinterpret_cast<float2*>(part + HD * 128) = make_float2(m_run, l_run);
        part += half * (HD / HALVES / 4) * 512;
#pragma unroll 1
        for (int c = 0; c < HD / HALVES / 32; ++c) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(o_addr + c * 32, o);
          tmem_wait_ld();
          if (none) {
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = 0;
          }
          if (!used) continue;
          if (whole) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              uint4 o4;
              o4.x = pack2(__uint_as_float(o[v * 8 + 0]) * inv, __uint_as_float(o[v * 8 + 1]) * inv);
              o4.y = pack2(__uint_as_float(o[v * 8 + 2]) * inv, __uint_as_float(o[v * 8 + 3]) * inv);
              o4.z = pack2(__uint_as_float(o[v * 8 + 4]) * inv, __uint_as_float(o[v * 8 + 5]) * inv);
              o4.w = pack2(__uint_as_float(o[v * 8 + 6]) * inv, __uint_as_float(o[v * 8 + 7]) * inv);
              *reinterpret_cast<uint4*>(out + c * 32 + v * 8) = o4;
            }
          } else {
#pragma unroll
            for (int v = 0; v < 8; ++v)
              *reinterpret_cast<uint4*>(part + (c * 8 + v) * 512) = make_uint4(o[v * 4], o[v * 4 + 1], o[v * 4 + 2], o[v * 4 + 3]);
          }
        }
      }
      w.segment(p);
      // the next item's first product overwrites O: it waits for P of all warps, which they write after this
    }
    if (!ok) TREE_ABORT(s, p.status);
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (!nothing && s.abort && threadIdx.x == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);   // let in-flight bulk copies land
  }
  __syncthreads();
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

// Joins the parts of the items that lie in several stretches: a thread per (row, head) and COLS columns, out = sum_c w_c o_c /
// sum_c w_c l_c with w_c = exp2(m_c - max m), the stretches in their order, the loads of PARTS of them in flight together.
template <int HD, int COLS, int PARTS>
__global__ void __launch_bounds__(128) tree_merge_kernel(const __grid_constant__ TreeDev p) {
  chain_trigger();
  chain_wait();
  const int b = blockIdx.z, kvh = blockIdx.x % p.a.n_kv, qt = blockIdx.x / p.a.n_kv, col = blockIdx.y * COLS, row = threadIdx.x;
  const int word = *reinterpret_cast<const volatile int*>(p.status), share = p.starts[p.a.d.batch], first = p.starts[b];
  const Seq x = seq_of(p, b, false);
  if (qt >= x.qts || gave_up(word)) return;                                     // gave up: there are parts that nobody wrote
  const int a = first + (kvh * x.qts + qt) * x.tiles, c0 = a / share, c1 = (a + x.tiles - 1) / share;
  const int ip = row / p.G, i = qt * p.per + ip;
  if (c0 == c1 || ip >= p.per || i >= x.n) return;
  // a stretch's first segment is in its first slot; the item's own beginning may lie behind another item in its stretch
  constexpr int64_t step = 2 * part_floats(HD);
  const float* at = p.partial + row * 4 + c0 * step;
  const float* head = at + (a > c0 * share ? part_floats(HD) : 0);
  constexpr int N = COLS / 4;
  float m = -INFINITY, l = 0.f, o[COLS];
#pragma unroll
  for (int k = 0; k < COLS; ++k) o[k] = 0.f;
  for (int c = c0; c <= c1; c += PARTS) {
    float2 ml[PARTS];
    float4 v[PARTS][N];
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const float* src = c + u == c0 ? head : at + (c + u - c0) * step;
      const bool in = c + u <= c1;
      ml[u] = in ? __ldcg(reinterpret_cast<const float2*>(src + HD * 128)) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < N; ++k)
        v[u][k] = in ? __ldcg(reinterpret_cast<const float4*>(src + (col / 4 + k) * 512)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float n = m;
#pragma unroll
    for (int u = 0; u < PARTS; ++u) n = fmaxf(n, ml[u].x);
    // no maximum so far: the parts saw nothing (zeros), or scores that are all NaN, whose sums stay NaN
    const float z = n == -INFINITY ? 0.f : n, f = ex2(m - z);
    m = n;
    l *= f;
#pragma unroll
    for (int k = 0; k < COLS; ++k) o[k] *= f;
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      const float w = ex2(ml[u].x - z);
      l = fmaf(w, ml[u].y, l);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        o[k * 4 + 0] = fmaf(v[u][k].x, w, o[k * 4 + 0]);
        o[k * 4 + 1] = fmaf(v[u][k].y, w, o[k * 4 + 1]);
        o[k * 4 + 2] = fmaf(v[u][k].z, w, o[k * 4 + 2]);
        o[k * 4 + 3] = fmaf(v[u][k].w, w, o[k * 4 + 3]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16* dst = p.a.out + ((int64_t)x.row0 + i) * p.a.ldo + (int64_t)(kvh * p.G + row - ip * p.G) * HD + col;
  if constexpr (COLS == 8)
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv), pack2(o[4] * inv, o[5] * inv),
                                                pack2(o[6] * inv, o[7] * inv));
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv));
}

bool allow_smem(std::atomic<uint64_t>& done, const void* kernel, int bytes) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

template <int HD>
int launch_t(const TreeAttnArgs& a, TreeDev& p, cudaStream_t s) {
  using C = TC<HD>;
  const size_t smem = sizeof(TreeSmem<HD>) + 1024;
  static_assert(sizeof(TreeSmem<HD>) + 1024 <= (C::PER_SM == 2 ? 113 : 227) * 1024, "shared memory budget");
  p.ctas = device_sms() * C::PER_SM;
  const int64_t qts = ceil_div(a.d.max_rows, p.per);
  const int64_t line = (int64_t)a.d.batch * a.n_kv * qts * (((int64_t)a.d.pos0 + a.d.max_rows + BKV - 1) / BKV);
  if (line > 0x3fffffff || a.n_kv * qts > 0x7fffffff) return POP_E_INVALID;          // places in the line are 32-bit numbers
  // two parts per CTA at most: of the item that it begins with and of the one that it ends with
  const size_t parts = (size_t)2 * p.ctas * part_floats(HD), need = (parts + a.d.batch + 1) * 4;
  p.starts = reinterpret_cast<int*>(p.partial + parts);
  const int64_t tiles = ((int64_t)a.d.pos0 + a.d.max_rows + BKV - 1) / BKV, items = (int64_t)a.d.batch * a.n_kv * qts;
  p.whole = tiles <= WHOLE_TILES && items <= p.ctas;
  if (a.workspace_bytes < need) return POP_E_NOSPACE;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  static std::atomic<uint64_t> configured{0};
  if (!allow_smem(configured, reinterpret_cast<const void*>(tree_attn_kernel<HD>), (int)smem)) return POP_E_CUDA;
  CUtensorMap tq, tk, tv;
  {
    // Q [rows][heads][hd]: a box is `per` rows of the G heads of a kv head; rows behind the last are zeros
    const uint64_t dims[5] = {(uint64_t)HD, (uint64_t)a.n_q, (uint64_t)a.d.rows, 1, 1};
    const uint64_t str[4] = {(uint64_t)HD, (uint64_t)a.ldq, (uint64_t)a.ldq * a.d.rows, (uint64_t)a.ldq * a.d.rows};
    const uint32_t box[5] = {64, (uint32_t)p.G, (uint32_t)p.per, 1, 1};
    if (make_tmap_bf16_nd(&tq, a.q, 3, dims, str, box) != POP_OK) return POP_E_CUDA;
  }
  {
    const uint64_t row = (uint64_t)HD * a.n_kv;
    const uint64_t dims[5] = {(uint64_t)HD, (uint64_t)a.n_kv, (uint64_t)a.c.page_size, (uint64_t)a.c.num_pages, 1};
    const uint64_t str[4] = {(uint64_t)HD, row, row * a.c.page_size, row * a.c.page_size * a.c.num_pages};
    const uint32_t box[5] = {64, 1, (uint32_t)p.rows_per_load, 1, 1};
    if (make_tmap_bf16_nd(&tk, a.c.k, 4, dims, str, box) != POP_OK || make_tmap_bf16_nd(&tv, a.c.v, 4, dims, str, box) != POP_OK)
      return POP_E_CUDA;
  }
  ProfScope prof(PROF_ATTENTION, 4.0 * HD * a.n_q * a.d.rows * ((double)a.d.pos0 + a.d.max_rows), s);
  if (launch_chained(tree_attn_kernel<HD>, dim3(p.whole ? (int)items : p.ctas), dim3(C::THREADS), smem, s, tq, tk, tv, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  if (p.whole) return POP_OK;
  const int pairs = a.d.max_rows < p.per ? a.d.max_rows * p.G : p.per * p.G;
  // Few items of many parts are joined by more threads, which each have more loads in flight: 1 x 64 rows of 8192 26.8 us against
  // 27.5, 1 x 16 of 2000 13.3 against 14.1. Many items (16 x 12 rows, window 1024: 48.2 against 43.4) or few parts (1 x 5 of 300: 11.3
  // against 11.0) would lose.
  const int64_t share = (line + p.ctas - 1) / p.ctas;
  const bool wide = tiles > 8 * (share < MIN_SHARE ? MIN_SHARE : share) && a.n_kv * qts * (HD / 8) * a.d.batch <= 2 * device_sms();
  if (launch_chained(wide ? tree_merge_kernel<HD, 4, 16> : tree_merge_kernel<HD, 8, 8>,
                     dim3((unsigned)(a.n_kv * qts), HD / (wide ? 4 : 8), a.d.batch), dim3((pairs + 31) & ~31), 0, s, p) != cudaSuccess)
    return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

}  // namespace

int launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s) {
  if (!a.q || !a.out || !pages_ok(a.c)) return POP_E_INVALID;
  if (a.d.batch < 1 || a.d.batch > 4096 || a.n_kv < 1 || a.n_q < 1 || a.n_q % a.n_kv || a.n_q > 65536 || a.n_q / a.n_kv > 128 ||
      a.d.max_rows < 0 || a.d.max_rows > 65536 || a.d.rows < 0 || a.d.pos0 < 0 || a.d.pos0 > 0x7fff0000 - 65536 || a.window < 0 ||
      a.window > 0x7ffffff0)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.q) % 16 || reinterpret_cast<uintptr_t>(a.out) % 16 || a.ldq % 8 || a.ldo % 8 ||
      reinterpret_cast<uintptr_t>(a.workspace) % 16 || !words_ok(a.d.cu, a.d.start, a.d.depth, a.mask))
    return POP_E_INVALID;
  if (!a.d.cu && (int64_t)a.d.batch * a.d.max_rows > a.d.rows) return POP_E_INVALID;
  if (a.mask && (int64_t)a.mask_words * 32 < a.d.max_rows) return POP_E_INVALID;
  if (a.ldq < (int64_t)a.n_q * a.head_dim || (a.d.rows > 1 && a.ldo < (int64_t)a.n_q * a.head_dim)) return POP_E_INVALID;
  const int64_t room = (int64_t)a.c.max_pages * a.c.page_size;
  if (a.d.pos0 > room || (!a.d.start && !a.d.cu && (int64_t)a.d.pos0 + a.d.max_rows > room)) return POP_E_NOSPACE;
  if (a.d.max_rows == 0 || a.d.rows == 0) return POP_OK;
  TreeDev p{};
  p.a = a;
  if (a.window - 65536 >= a.d.pos0) p.a.window = 0;            // beyond the reach of every row: depths are below 65536
  p.G = a.n_q / a.n_kv;
  p.per = 128 / p.G;
  p.room = room < 0x7fff0000 ? (int)room : 0x7fff0000;
  p.rows_per_load = a.c.page_size < BKV ? a.c.page_size : BKV;
  p.scale_log2 = 1.4426950408889634f / sqrtf((float)a.head_dim);
  p.partial = static_cast<float*>(a.workspace);
  switch (a.head_dim) {
    case 64: return launch_t<64>(a, p, s);
    case 128: return launch_t<128>(a, p, s);
    default: return launch_t<256>(a, p, s);
  }
}

}  // namespace pop
