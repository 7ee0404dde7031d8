// Drafted tokens and the bf16 paged cache: the append of a tree's rows (paper Eq. 2-3 for several rows of a sequence, whose
// rotary position is their depth in the tree and not their cache slot), and keeping of the accepted path.
#include "heads.cuh"
#include "tree.cuh"

namespace pop {
namespace {

// ------------------------------------------------------------------------------ norm + rotation + append
// hd / 8 lanes per row and HPG consecutive heads, each with four rotation pairs: place, position, page and rotary entries are
// found once for the heads, whose rows are all asked for before the first is used. Every value is read and written once: bound
// by the bytes, and for few rows by the chain of loads (prefix sums and start, then page, depth and rows, then the rotary
// entries).
struct TreeAppendDev {
  TreeAppendArgs a;
  int* status;
};

template <int HD, bool IN_BF16, int HPG>
__global__ void __launch_bounds__(256) tree_append_kernel(const __grid_constant__ TreeAppendDev p) {
  constexpr int LPR = HD / 8, HALF = HD / 2;
  const TreeAppendArgs& a = p.a;
  chain_trigger();
  const int lane = threadIdx.x & 31, j0 = (lane % LPR) * 4, b = blockIdx.y;
  const uint32_t heads = a.n_q + 2 * a.n_kv, groups = (heads + HPG - 1) / HPG;
  const uint32_t item = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;             // below 2^29
  const int i = item / groups, h0 = (item - i * groups) * HPG;
  chain_wait();
  const int row0 = a.d.cu ? __ldg(a.d.cu + b) : b * a.d.max_rows;
  const int n = a.d.cu ? __ldg(a.d.cu + b + 1) - row0 : a.d.max_rows;
  const int start = a.d.start ? __ldg(a.d.start + b) : a.d.pos0;
  if (n <= 0) return;                                                             // no rows: whatever the start is
  if (n > a.d.max_rows || row0 < 0 || row0 > a.d.rows - n || start < 0 || start > 0x7fff0000 - n) {
    if (threadIdx.x == 0) atomicMin(p.status, (int)POP_E_INVALID);
    return;
  }
  if (blockIdx.x * (256 / LPR) >= n * groups) return;
  // The lanes behind the last item work on the last row and store nothing: the warp stays whole for the norm's shuffles
  const bool idle = i >= n;
  const int ii = idle ? n - 1 : i;
  const int64_t row = row0 + ii;
  const uint32_t slot = start + ii, page_at = slot / (uint32_t)a.dst.page_size, in_page = slot - page_at * a.dst.page_size;
  bool bad = false;
  int page = -1;
  if (h0 + HPG > a.n_q && page_at < (uint32_t)a.dst.max_pages) page = __ldg(a.dst.table + (int64_t)b * a.dst.max_pages + page_at);
  float x[HPG][8];
#pragma unroll
  for (int u = 0; u < HPG; ++u) load_row8<HD, IN_BF16>(a.in, row * a.ld_in + (int64_t)min(h0 + u, (int)heads - 1) * HD + j0, x[u]);
  float2 cs[4];
  if (h0 < a.n_q + a.n_kv) {
    int64_t at = (int64_t)start + (a.d.depth ? __ldg(a.d.depth + row) : ii);
    if (at < 0 || at >= a.table_rows) {                                           // never turned into an address
      bad = true;
      at = 0;
    }
    const float4* t = reinterpret_cast<const float4*>(a.table + at * HALF + j0);
    const float4 t0 = __ldg(t), t1 = __ldg(t + 1);
    cs[0] = make_float2(t0.x, t0.y); cs[1] = make_float2(t0.z, t0.w);
    cs[2] = make_float2(t1.x, t1.y); cs[3] = make_float2(t1.z, t1.w);
  }
  if (a.q_gain != nullptr || a.k_gain != nullptr) {                               // by all lanes: heads of a warp may differ
    const float* have = nullptr;
    float4 g0, g1;
#pragma unroll
    for (int u = 0; u < HPG; ++u) {
      const int h = h0 + u;
      const float* gain = h < a.n_q ? a.q_gain : h < a.n_q + a.n_kv ? a.k_gain : nullptr;
      if (gain != nullptr && gain != have) {
        if (reinterpret_cast<uintptr_t>(gain) % 16 == 0) {
          g0 = __ldg(reinterpret_cast<const float4*>(gain + j0));
          g1 = __ldg(reinterpret_cast<const float4*>(gain + j0 + HALF));
        } else {
          g0 = make_float4(__ldg(gain + j0), __ldg(gain + j0 + 1), __ldg(gain + j0 + 2), __ldg(gain + j0 + 3));
          g1 = make_float4(__ldg(gain + j0 + HALF), __ldg(gain + j0 + HALF + 1), __ldg(gain + j0 + HALF + 2), __ldg(gain + j0 + HALF + 3));
        }
        have = gain;
      }
      float y[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) y[v] = x[u][v];
      norm_row8<HD>(y, g0, g1, a.eps);
      if (gain != nullptr) {
#pragma unroll
        for (int v = 0; v < 8; ++v) x[u][v] = y[v];
      }
    }
  }
  if (idle) return;
#pragma unroll
  for (int u = 0; u < HPG; ++u) {
    const int h = h0 + u;
    if (h >= (int)heads) break;
    if (h < a.n_q + a.n_kv) turn_row8(x[u], cs);
    if (h < a.n_q) {
      store_q8<HD>(a.q_out + row * a.ldq + (int64_t)h * HD + j0, x[u]);
    } else if ((unsigned)page < (unsigned)a.dst.num_pages) {                      // else never turned into an address
      const bool is_v = h >= a.n_q + a.n_kv;
      const int head = h - a.n_q - (is_v ? a.n_kv : 0);
      store_q8<HD>((is_v ? a.dst.v : a.dst.k) + (((int64_t)page * a.dst.page_size + in_page) * a.n_kv + head) * HD + j0, x[u]);
    } else {
      bad = true;
    }
  }
  if (bad) atomicMin(p.status, (int)POP_E_INVALID);
}

// ------------------------------------------------------------------------------ the accepted path
// Entry of slot start + kept[i] -> slot start + i for rising kept. A thread owns 16 bytes of an entry in one layer of K or V
// and walks the path: eight entries are read, then written. As kept[i] >= i and the list rises, what a later batch reads lies
// behind everything that an earlier one wrote, so the path may be moved where it lies. Entries that stay are not touched.
struct KeepDev {
  KeepArgs a;
  int cols;                     // 16-byte pieces of an entry: n_kv hd / 8
  int* status;
};
constexpr int KEEP_THREADS = 128, KEEP_LIST = 1024;

__global__ void __launch_bounds__(KEEP_THREADS) cache_keep_kernel(const __grid_constant__ KeepDev p) {
  const KeepArgs& a = p.a;
  __shared__ int src_at[KEEP_LIST], dst_at[KEEP_LIST];          // pool rows (page * page_size + slot in it)
  __shared__ int moved;
  chain_trigger();
  chain_wait();
  const int b = blockIdx.z, tid = threadIdx.x;
  const int n = a.n_kept ? __ldg(a.n_kept + b) : a.max_kept;
  const int start = a.start ? __ldg(a.start + b) : a.pos0;
  if (n <= 0) return;
  if (tid == 0) moved = n;
  bool bad = n > a.max_kept || start < 0;
  if (!bad) {
    const int32_t* list = a.kept + (int64_t)b * a.ld_kept;
    const int64_t room = min((int64_t)a.c.max_pages * a.c.page_size, (int64_t)0x7fff0000) - start;
    for (int i = tid; i < n; i += KEEP_THREADS) {
      const int from = __ldg(list + i), before = i > 0 ? __ldg(list + i - 1) : -1;
      int sp = -1, dp = -1;
      if (from > before && from >= 0 && from < room) {
        sp = __ldg(a.c.table + (int64_t)b * a.c.max_pages + (start + from) / a.c.page_size);
        dp = __ldg(a.c.table + (int64_t)b * a.c.max_pages + (start + i) / a.c.page_size);
      }
      if ((unsigned)sp >= (unsigned)a.c.num_pages || (unsigned)dp >= (unsigned)a.c.num_pages) {
        bad = true;                                             // never turned into an address
      } else {
        src_at[i] = sp * a.c.page_size + (start + from) % a.c.page_size;
        dst_at[i] = dp * a.c.page_size + (start + i) % a.c.page_size;
      }
    }
  }
  if (__syncthreads_or(bad)) {                                  // one wrong entry: the sequence stays as it is
    if (tid == 0) atomicMin(p.status, (int)POP_E_INVALID);
    return;
  }
  for (int i = tid; i < n; i += KEEP_THREADS)
    if (src_at[i] != dst_at[i]) atomicMin(&moved, i);           // the first that moves; all behind it do too
  __syncthreads();
  const int col = blockIdx.x * KEEP_THREADS + tid;
  if (col >= p.cols) return;
  const int layer = blockIdx.y >> 1;
  bf16* pool = (blockIdx.y & 1 ? a.c.v : a.c.k) + (int64_t)layer * a.layer_stride + (int64_t)col * 8;
  const int64_t entry = (int64_t)p.cols * 8;
  for (int i = moved; i < n; i += 8) {
    uint4 w[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u < n) w[u] = *reinterpret_cast<const uint4*>(pool + src_at[i + u] * entry);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u < n) *reinterpret_cast<uint4*>(pool + dst_at[i + u] * entry) = w[u];
  }
}

template <int HD>
auto kernel_of(bool in_bf16, bool four) {
  return in_bf16 ? (four ? tree_append_kernel<HD, true, 4> : tree_append_kernel<HD, true, 1>)
                 : (four ? tree_append_kernel<HD, false, 4> : tree_append_kernel<HD, false, 1>);
}

}  // namespace

int launch_tree_append(const TreeAppendArgs& a, cudaStream_t s) {
  if (!a.in || !a.table || !pages_ok(a.dst) || (a.n_q > 0 && !a.q_out)) return POP_E_INVALID;
  if (a.d.batch < 1 || a.d.batch > 65535 || a.d.max_rows < 0 || a.d.max_rows > 65536 || a.d.rows < 0 || a.n_q < 0 || a.n_kv < 1 || a.n_q > 4096 ||
      a.n_kv > 1024 || a.d.pos0 < 0 || a.table_rows < 1)
    return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  if (reinterpret_cast<uintptr_t>(a.in) % 16 || reinterpret_cast<uintptr_t>(a.table) % 16 || a.ld_in % 4 ||
      (a.n_q > 0 && (reinterpret_cast<uintptr_t>(a.q_out) % 8 || a.ldq % 4)))
    return POP_E_INVALID;
  if (!words_ok(a.d.cu, a.d.start, a.d.depth, a.q_gain, a.k_gain)) return POP_E_INVALID;
  if (!a.d.cu && (int64_t)a.d.batch * a.d.max_rows > a.d.rows) return POP_E_INVALID;
  if (a.n_q > 0 && a.d.rows > 1 && a.ldq < (int64_t)a.n_q * a.head_dim) return POP_E_INVALID;       // rows over each other
  if (!a.d.start && !a.d.cu && (int64_t)a.d.pos0 + a.d.max_rows > (int64_t)a.dst.max_pages * a.dst.page_size) return POP_E_NOSPACE;
  if (a.d.max_rows == 0 || a.d.rows == 0) return POP_OK;
  TreeAppendDev p{};
  p.a = a;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  // Four heads at a time where there are more blocks of one than the SMs hold, else one. us for one / four: 48 x up to 33 rows of
  // 48 heads, normalised 10.3 / 8.8, 16 x up to 64 rows of 32 heads of 256 8.7 / 7.1; 24 x up to 20 rows of 48 heads 3.9 / 4.2,
  // 8 rows of 48 heads 1.7 / 2.2
  const int heads = a.n_q + 2 * a.n_kv, per = 2048 / a.head_dim;
  const bool four = (int64_t)a.d.rows * heads >= (int64_t)device_sms() * 8 * per;
  const int groups = four ? ceil_div(heads, 4) : heads;
  const dim3 grid(ceil_div(a.d.max_rows * groups, per), a.d.batch);
  ProfScope prof(PROF_ELEMENTWISE, (double)a.d.rows * a.head_dim * heads * ((a.in_bf16 ? 2.0 : 4.0) + 2.0), s);
  void (*kernel)(TreeAppendDev);
  switch (a.head_dim) {
    case 64: kernel = kernel_of<64>(a.in_bf16, four); break;
    case 128: kernel = kernel_of<128>(a.in_bf16, four); break;
    default: kernel = kernel_of<256>(a.in_bf16, four); break;
  }
  if (launch_chained(kernel, grid, dim3(256), 0, s, p) != cudaSuccess) return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

int launch_cache_keep(const KeepArgs& a, cudaStream_t s) {
  if (!pages_ok(a.c) || !a.kept || a.layers < 1 || a.layers > 32767 || a.batch < 1 || a.batch > 65535 || a.n_kv < 1 ||
      a.n_kv > 1024 || a.max_kept < 0 || a.max_kept > KEEP_LIST || a.pos0 < 0 || (a.batch > 1 && a.ld_kept < a.max_kept))
    return POP_E_INVALID;
  if (!words_ok(a.kept, a.n_kept, a.start)) return POP_E_INVALID;
  if (a.head_dim != 64 && a.head_dim != 128 && a.head_dim != 256) return POP_E_INVALID;
  const int64_t page = (int64_t)a.c.page_size * a.n_kv * a.head_dim;
  if (a.layers > 1 && (a.layer_stride % 8 || (a.layer_stride > -page && a.layer_stride < page))) return POP_E_INVALID;  // layers over each other
  if ((int64_t)a.c.num_pages * a.c.page_size > 0x7fffffff) return POP_E_INVALID;                    // pool rows are 32-bit numbers
  if (!a.start && (int64_t)a.pos0 + a.max_kept > (int64_t)a.c.max_pages * a.c.page_size) return POP_E_NOSPACE;
  if (a.max_kept == 0) return POP_OK;
  KeepDev p{};
  p.a = a;
  p.cols = a.n_kv * a.head_dim / 8;
  p.status = status_word();
  if (!p.status) return POP_E_CUDA;
  const dim3 grid(ceil_div(p.cols, KEEP_THREADS), a.layers * 2, a.batch);
  ProfScope prof(PROF_ELEMENTWISE, (double)a.layers * a.batch * a.max_kept * a.n_kv * a.head_dim * 8.0, s);
  if (launch_chained(cache_keep_kernel, grid, dim3(KEEP_THREADS), 0, s, p) != cudaSuccess) return POP_E_CUDA;
  count_launch();
  return POP_OK;
}

}  // namespace pop
