// A step that checks drafted tokens (internal): append of a tree's rows to the bf16 paged cache, attention of the rows over
// the cache and their ancestors, and moving the accepted path's entries together.
#pragma once
#include "common.cuh"

#include <atomic>

namespace pop {

// One layer of the bf16 cache: [pages][page_size][n_kv][hd]
struct Pages {
  bf16* k; bf16* v;
  const int32_t* table;                // [batch][max_pages]
  int page_size, num_pages, max_pages;
};
// arrays of 32-bit words (null ones too) begin at one
template <typename... T>
inline bool words_ok(const T*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 3) == 0; }
inline bool pages_ok(const Pages& c) {
  return c.k && c.v && c.table && words_ok(c.table) && page_size_ok(c.page_size) && c.num_pages >= 1 && c.max_pages >= 1 &&
         reinterpret_cast<uintptr_t>(c.k) % 16 == 0 && reinterpret_cast<uintptr_t>(c.v) % 16 == 0;
}

// The drafted rows of the sequences: packed rows cu[b] .. cu[b + 1] - 1, or max_rows each; start[b] (or pos0) positions in
// front of them. Row i of a sequence has cache slot start + i and position start + depth (depth i without the array).
struct Drafts {
  const int32_t* cu; int max_rows; int rows;           // rows: all packed rows there are
  const int32_t* start; int pos0;
  const int32_t* depth;
  int batch;
};

struct TreeAppendArgs {
  const void* in; bool in_bf16; int64_t ld_in;         // rows [q heads | k heads | v heads] * hd
  Drafts d;
  bf16* q_out; int64_t ldq;
  Pages dst;
  const float* q_gain; const float* k_gain; float eps;
  const float2* table; int table_rows;
  int n_q, n_kv, head_dim;
};
int launch_tree_append(const TreeAppendArgs& a, cudaStream_t s);

struct KeepArgs {
  Pages c; int64_t layer_stride; int layers;           // elements between the layers of a pool
  const int32_t* kept; int64_t ld_kept; const int32_t* n_kept; int max_kept;
  const int32_t* start; int pos0;
  int batch, n_kv, head_dim;
};
int launch_cache_keep(const KeepArgs& a, cudaStream_t s);

struct TreeAttnArgs {
  const bf16* q; int64_t ldq;
  Drafts d;                                            // pos0: the largest start where d.start is given
  const uint32_t* mask; int mask_words;                // [rows][mask_words], or null: rows in front and the row itself
  Pages c;
  bf16* out; int64_t ldo;
  int n_q, n_kv, head_dim, window;
  void* workspace; size_t workspace_bytes;
};
int launch_tree_attention(const TreeAttnArgs& a, cudaStream_t s);

int device_sms();                                      // SMs of the device that was current at the first call

}  // namespace pop
