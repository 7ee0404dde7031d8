/* pop_kernels.h - kernel-level entry points of the POP prefill library (C ABI).
 *
 * Each call runs ONE step of the path declared in pop.h on caller-owned device buffers, so that
 * every kernel can be checked against the oracle's statement of the same step and timed alone.
 * Conventions are those of pop.h: device pointers are borrowed, `stream` is a cudaStream_t, calls
 * are asynchronous, the return value is a pop_status, and an error enqueues nothing.
 */
#ifndef POP_KERNELS_H_
#define POP_KERNELS_H_

#include "pop.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Projection GEMM of a decoder layer (paper Eq. 1-2: the "x W" products), batched:
 *   D[g][m][n] = sum_k A[g][m][k] * B[g][n][k],  g < batch, bf16 operands, fp32 accumulation.
 * A: device bf16, row stride lda, batch stride a_bs (elements; 0 = densely packed); B likewise.
 * epilogue: 0 store bf16, 1 store fp32, 2 fp32 out += D (residual add of Eq. 1),
 *           3 gated FFN: rows of B come in blocks of 256 (128 gate rows, then the 128 matching up
 *             rows), out bf16 column f = act(gate_f) * up_f for f < n_valid (act 0 SiLU, 1 tanh-GELU).
 * out: row stride ldo, batch stride o_bs, in elements of the output type.
 * Requires K, lda, ldb multiples of 8, 16-byte aligned pointers, N a multiple of 8 (256 for epilogue 3). */
int pop_k_gemm(const void* A, int64_t lda, int64_t a_bs, const void* B, int64_t ldb, int64_t b_bs, void* out,
               int64_t ldo, int64_t o_bs, int32_t M, int32_t N, int32_t K, int32_t batch, int32_t epilogue,
               int32_t act, int32_t n_valid, void* stream);

/* pop_k_gemm (batch 1, epilogues 0-3) with the layer's RMSNorm (the LN of paper Eq. 1-2) folded
 * around it, so that no separate pass over the residual stream is needed:
 *  - producer side, epilogue 2 only, when hn_out != NULL: besides out += D the call writes
 *    hn_out[m][n] = bf16(out_new[m][n] * gain_next[n]) (row stride ld_hn) -- the next GEMM's operand,
 *    not yet normalised -- and ss_out[m * ss_ld + n / 256] = sum over that 256-column tile of
 *    out_new[m][n]^2 (ss_ld >= ceil(N / 256));
 *  - consumer side, when ss_in != NULL: every row m of D is multiplied by
 *    rsqrt(sum_{i < ss_cnt} ss_in[m * ss_in_ld + i] / norm_d + norm_eps) before the epilogue acts
 *    (for epilogue 3 before the activation). The partial sums are added in index order, so the
 *    result does not depend on scheduling.
 * Pass NULL for the side not wanted. */
int pop_k_gemm_norm(const void* A, int64_t lda, const void* B, int64_t ldb, void* out, int64_t ldo, int32_t M,
                    int32_t N, int32_t K, int32_t epilogue, int32_t act, int32_t n_valid, void* hn_out, int64_t ld_hn,
                    const float* gain_next, float* ss_out, int32_t ss_ld, const float* ss_in, int32_t ss_cnt,
                    int32_t ss_in_ld, int32_t norm_d, float norm_eps, void* stream);

/* The fused form of the QKV projection and pop_k_rope_cache (paper Eq. 2-3; Eq. 14 for pruned
 * layers): D[g] = A[g] W[g]^T with W's rows ordered [q heads | k heads | v heads] * hd, and in the
 * GEMM's epilogue the optional per-head RMSNorm (q, k), RoPE (q, k), rounding to bf16, q -> q_out
 * [M][ldq] (n_q may be 0: no query, as for pruned layers), k and v -> cache layer layer0 + g.
 * A bf16 [batch][M][lda] (batch stride a_bs, 0 = packed), W bf16 [batch][(n_q+2 n_kv) hd][ldw].
 * Row / position / cache conventions and the remaining arguments are those of pop_k_rope_cache;
 * M must be a multiple of rows_per_seq. Nothing of the fp32 projection goes through memory. */
int pop_k_gemm_qkv_rope(const void* A, int64_t lda, int64_t a_bs, const void* W, int64_t ldw, int64_t w_bs, int32_t M,
                        int32_t K, int32_t batch, void* q_out, int64_t ldq, void* k_pool, void* v_pool,
                        int64_t pool_layer_stride, int32_t layer0, const int32_t* block_table,
                        int32_t max_pages_per_seq, int32_t page_size, const float* q_gain, const float* k_gain,
                        int64_t gain_gs, const void* table, int32_t n_q, int32_t n_kv, int32_t head_dim,
                        int32_t rows_per_seq, int32_t rows_written, int32_t pos0, float eps, void* stream);

/* Causal GQA attention of a decoder layer over the paged cache (paper Eq. 1, Attn(x_l, K, V) after
 * the append of Eq. 3): for sequence b, query row i (absolute position q_pos0 + i) and head h,
 *   out[b][i][h] = sum_j softmax_j(q[b][i][h] . k[b][j][g] / sqrt(hd)) v[b][j][g],  g = h*n_kv/n_q,
 * over cache positions j <= q_pos0 + i, and j > q_pos0 + i - window when window > 0.
 * q: device bf16 [batch*seq_len][ldq] (head h at column h*hd); k_pool/v_pool: ONE layer of the
 * cache, bf16 [num_pages][page_size][n_kv][hd]; block_table as in pop_kv_cache_t; out: bf16
 * [batch*seq_len][ldo]. kv_len = valid cache positions (>= q_pos0 + seq_len). hd in {64,128,256}; page_size as in pop.h. */
int pop_k_attention(const void* q, int64_t ldq, const void* k_pool, const void* v_pool, const int32_t* block_table,
                    void* out, int64_t ldo, int32_t batch, int32_t seq_len, int32_t q_pos0, int32_t kv_len,
                    int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                    int32_t max_pages_per_seq, int32_t window, void* stream);

/* FP8 operands for the projections of paper Eq. 1-2. The paper fixes no number format and names
 * stage-aware quantisation as a direction (Sec. 6); this is the OCP E4M3 format (1-4-3 bits, bias 7,
 * largest value 448, no infinities), round to nearest even, saturating, with one scale per
 * activation row and one per weight matrix: value = code * scale.
 *
 * pop_k_rmsnorm_e4m3: y = LN(x[r]) as pop_k_rmsnorm computes it in fp32; out[r][:] = e4m3(y * 448 /
 *   max|y|) as bytes (row stride ldo bytes, a multiple of 16), scale[r] = max|y| / 448 (1 for a zero row).
 * pop_k_quant_rows_e4m3: rows of stored bf16 values (row stride ld_in elements, d <= 16384 a multiple of 8):
 *   out[r][:] = e4m3(in[r][:] * 448 / max|in[r]|) (row stride ld_out bytes, a multiple of 16), scale[r] as
 *   above. out may be in itself (each row's codes then fill the first d bytes of the row).
 * pop_k_quantize_e4m3: the same for a whole bf16 array of n elements (n a multiple of 8) with one
 *   scale: out[i] = e4m3(w[i] * 448 / max|w|), *scale = max|w| / 448. scratch4: 4 device bytes.
 * pop_k_gemm_e4m3: D[m][n] = a_scale[m] * *b_scale * sum_k A[m][k] * B[n][k] on the codes (fp32
 *   accumulation on the tensor cores, kind f8f6f4), then epilogue 0, 1, 2 or 3 of pop_k_gemm. lda,
 *   ldb, K count codes and are multiples of 16; pointers 16-byte aligned; a_scale, b_scale device fp32. */
/* pop_k_gemv with E4M3 weights (the single-position passes of Sec. 3.3 / the decode stage stream half the
 * bytes): out[b][n] = *w_scale * sum_k x[b][k] * W[n][k], x bf16 [B][ldx] unquantised, W codes [N][ldw]
 * (K and ldw multiples of 16), w_scale device fp32. Modes as pop_k_gemv. */
int pop_k_gemv_e4m3(const void* x, int64_t ldx, const void* w, int64_t ldw, const float* w_scale, void* out,
                    int64_t ldo, int32_t B, int32_t N, int32_t K, int32_t mode, int32_t act, int32_t n_valid,
                    void* stream);
int pop_k_rmsnorm_e4m3(const float* x, int64_t ldx, const float* gain, void* out, int64_t ldo, float* scale,
                       int32_t rows, int32_t d, float eps, void* stream);
int pop_k_quant_rows_e4m3(const void* in, int64_t ld_in, void* out, int64_t ld_out, float* scale, int32_t rows,
                          int32_t d, void* stream);
int pop_k_quantize_e4m3(const void* w, int64_t n, void* out, float* scale, void* scratch4, void* stream);
int pop_k_gemm_e4m3(const void* A, int64_t lda, const float* a_scale, const void* B, int64_t ldb,
                    const float* b_scale, void* out, int64_t ldo, int32_t M, int32_t N, int32_t K, int32_t epilogue,
                    int32_t act, int32_t n_valid, void* stream);

/* RMSNorm, the LN of paper Eq. 2 / Eq. 14: out[g][r][:] = x[r][:] * rsqrt(mean(x[r]^2)+eps) * gain[g][:].
 * x fp32 [rows][ldx]; gain fp32, group g at gain + g*gain_stride; out bf16 (out_f32 = 0) or fp32,
 * group stride out_gs elements. */
int pop_k_rmsnorm(const float* x, int64_t ldx, const float* gain, int64_t gain_stride, void* out, int64_t ldo,
                  int64_t out_gs, int32_t rows, int32_t d, int32_t groups, float eps, int32_t out_f32, void* stream);

/* Rotary table: table[pos][j] = (cos, sin)(pos * theta^(-2j/hd)) as float2, pos < n_pos, j < hd/2. */
int pop_k_rope_table(void* table, int32_t n_pos, int32_t head_dim, float theta, void* stream);

/* KV generation and append (paper Eq. 2-3; Eq. 14 when applied to a pruned layer): rows of fp32
 * projections [q heads | k heads | v heads] * hd get the optional per-head RMSNorm (q, k), RoPE
 * (q, k), rounding to bf16; q goes to q_out [rows][ldq], k and v into cache layer layer0 + g of
 * the pools [layer][page][slot][n_kv][hd] (pool_layer_stride elements per layer). Row r belongs to
 * sequence r / rows_per_seq at position pos0 + r % rows_per_seq; rows with r % rows_per_seq >=
 * rows_written are skipped. n_q may be 0 (pruned layers: no query). */
int pop_k_rope_cache(const float* in, int64_t ld_in, int64_t in_gs, void* q_out, int64_t ldq, void* k_pool,
                     void* v_pool, int64_t pool_layer_stride, int32_t layer0, const int32_t* block_table,
                     int32_t max_pages_per_seq, int32_t page_size, const float* q_gain, const float* k_gain,
                     int64_t gain_gs, const void* table, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t rows,
                     int32_t rows_per_seq, int32_t rows_written, int32_t pos0, int32_t groups, float eps,
                     void* stream);

/* Weight-streaming GEMV of the boundary-token path (paper Sec. 3.3) and of the output head:
 * out[b][n] = sum_k x[b][k] * W[n][k] for a few rows b. x bf16 or fp32 (x_f32) [B][ldx]; W bf16
 * [N][ldw]. mode 0: fp32 store; 2: fp32 +=; 3: gated (W rows in 128-gate/128-up blocks) -> bf16. */
int pop_k_gemv(const void* x, int64_t ldx, int32_t x_f32, const void* w, int64_t ldw, void* out, int64_t ldo,
               int32_t B, int32_t N, int32_t K, int32_t mode, int32_t act, int32_t n_valid, void* stream);

/* Single-query attention of the boundary token (paper Sec. 3.3; one query per sequence at position
 * kv_len-1) over one cache layer, split over the keys. n_q / n_kv <= 8; head_dim 64, 128 or 256.
 * partial: device scratch of batch * n_q * 64 * (hd + 2) floats, contents irrelevant before and after.
 * counters: optional device int32 [batch * n_kv]. If given they must all be zero when the call's
 * kernels start and are all zero again when they end (so one zeroed array serves any number of
 * calls on one stream); the attention kernel then merges its own splits and the call is a single
 * launch. Null: a second kernel merges them. Both ways give the same bits. With few splits per sequence
 * and kv head (short caches, several sequences) the splits run as one thread-block cluster and merge
 * through distributed shared memory; partial and counters are then not touched (POP_DEC_CLUSTER=0 in the
 * environment turns that form off). */
int pop_k_decode_attention(const void* q, int64_t ldq, const void* k_pool, const void* v_pool,
                           const int32_t* block_table, int32_t max_pages_per_seq, int32_t page_size, float* partial,
                           int32_t* counters, void* out, int64_t ldo, int32_t batch, int32_t n_q, int32_t n_kv,
                           int32_t head_dim, int32_t kv_len, int32_t window, void* stream);

/* pop_k_decode_attention with the end of the projection folded in (paper Eq. 2-3 for the one new
 * position, then Attn of Eq. 1; Sec. 3.3): instead of finished queries the kernel takes the fp32 row
 * qkv[b] = [q heads | k heads | v heads] * head_dim of every sequence (ld_qkv floats apart), applies the
 * per-head RMSNorm (q_gain / k_gain: fp32 [head_dim], or both NULL for none; eps) and the rotary row
 * of position kv_len - 1 (table: device float2 [head_dim / 2] pairs (cos, sin) of that one position) to
 * the queries and the key, appends key and value at position kv_len - 1 of the cache (k_pool and
 * v_pool are WRITTEN here: one layer, [num_pages][page_size][n_kv][head_dim]), and attends over
 * positions max(0, kv_len - window) .. kv_len - 1 (window 0: all). counters (device int32
 * [batch * n_kv], zero before and after) are required: the call is a single launch. A block-table
 * entry outside [0, num_pages) is never dereferenced; the status word is raised to POP_E_INVALID.
 * This is the form the boundary-token / decode path of pop_prefill and pop_decode_step runs. */
int pop_k_decode_attention_qkv(const float* qkv, int64_t ld_qkv, const float* q_gain, const float* k_gain, float eps,
                               const void* rope_row, void* k_pool, void* v_pool, const int32_t* block_table,
                               int32_t max_pages_per_seq, int32_t page_size, int32_t num_pages, float* partial,
                               int32_t* counters, void* out, int64_t ldo, int32_t batch, int32_t n_q, int32_t n_kv,
                               int32_t head_dim, int32_t kv_len, int32_t window, void* stream);

/* The same single-query attention as pop_k_decode_attention for callers that have no way to hand
 * over a scratch buffer because they cannot allocate device memory at the point of the call: code
 * running inside a host callback or a real-time serving loop where cudaMalloc is forbidden, or a
 * process that received all its device buffers (inputs and outputs only) from another owner and
 * has no allocator of its own. (The paper has no counterpart: this is a packaging variant, not a
 * step of the method.) The split-KV partials go to a fixed array of POP_STATIC_SCRATCH_FLOATS
 * floats (16 MiB) that is part of the library image, so every GPU that loads the library holds it
 * until the process ends. The call allocates and frees nothing, neither through CUDA nor any other
 * library. Arguments, layouts and results are those of pop_k_decode_attention minus `partial`.
 *  - Limit: batch * n_q * splits * (head_dim + 2) <= POP_STATIC_SCRATCH_FLOATS, where splits =
 *    min(64, SMs / (n_kv * batch), ceil(span / 64)), at least 1, and span = min(kv_len, window or
 *    kv_len); a larger problem is refused with POP_E_NOSPACE and nothing is enqueued (e.g. 512
 *    sequences x 32 heads x hd 128 fit at any length; 1024 such sequences do not).
 *  - The first call on each device looks up the array's device address (one runtime query with
 *    that device current, result kept); make that first call before starting any stream capture.
 *  - All calls share the one array, which keeps whatever the previous call left. Each call
 *    overwrites every slot it later reads, so no clearing is needed, but two calls whose kernels
 *    may overlap on the GPU (different streams without an ordering between them) race on it:
 *    serialise them. Calls on one stream are safe. The arrival counters of the split merge sit in a
 *    second fixed array (4096 entries, one per sequence and kv head; with more than that a second
 *    kernel merges the splits instead); it is not reachable from the host, starts at zero when the
 *    library is loaded and every launch leaves it at zero again.
 * Errors: POP_E_INVALID (null pointer, bad head_dim or head counts), POP_E_NOSPACE (over the limit,
 * or block table too short), POP_E_CUDA. */
#define POP_STATIC_SCRATCH_FLOATS (4 * 1024 * 1024)
int pop_k_decode_attention_static(const void* q, int64_t ldq, const void* k_pool, const void* v_pool,
                                  const int32_t* block_table, int32_t max_pages_per_seq, int32_t page_size,
                                  void* out, int64_t ldo, int32_t batch, int32_t n_q, int32_t n_kv,
                                  int32_t head_dim, int32_t kv_len, int32_t window, void* stream);

/* ---------------------------------------------------------------------------------------------------
 * 8-bit paged cache: half the bytes of pop_kv_cache_t. One layer consists of
 *   k_codes, v_codes: uint8 [num_pages][n_kv][page_size][hd], OCP E4M3 codes (16-byte aligned);
 *   k_scales, v_scales: uint8 [num_pages][n_kv][page_size / 16], one E8M0 scale (a power of two, stored as its
 *     exponent + 127) for each block of 16 positions and kv head:  value = code * 2^(scale - 127);
 *   block_table, page_size, num_pages, max_pages_per_seq as in pop_kv_cache_t (page_size 16, 32, 64 or a multiple of
 *     128; a page serves K and V alike). Positions of one page and head are contiguous.
 * The scale of a block is the smallest power of two s >= 2^-64 with max |value| <= 448 s (NaN does not count; infinities
 * make it 2^120), a code is value / s rounded to nearest even, saturating at 448 (NaN stays NaN). hd is 64, 128 or 256.
 * Device-side checks in every call: a block-table entry outside [0, num_pages), a length above the stated maximum, a
 * rotation row outside the table are never turned into addresses; the status word is raised to POP_E_INVALID and what
 * depends on them is not written or reads as zeros; the other sequences, and calls made while the word holds POP_E_INVALID,
 * are not touched by it (behind POP_E_DEVICE_TIMEOUT pop_k_attention_e4m3 may leave rows as they are). Lengths (kv_len,
 * max_len) go up to 2^31 - 2^16. The codes behind a sequence's last position are left as they are. cu_rows is taken at its
 * word: the calls do not know how many rows in, q and out have.
 * Scale bytes are 63 to 247, as these calls write them. The V scales of the positions that a row sees may lie up to 2^100
 * apart (beside blocks of zeros: values up to 2^44); beyond that the small blocks' share of the softmax sum may be lost.
 *
 * pop_k_quant_cache_e4m3: the bf16 cache that a prefill left, for `layers` consecutive layers (src_layer_stride elements,
 *   code_layer_stride and scale_layer_stride bytes apart), positions 0 .. n-1 of every sequence, n = seq_lens[b] (device
 *   int32 [batch], each <= max_len) or max_len for all if seq_lens is NULL. The two caches have tables of their own. */
int pop_k_quant_cache_e4m3(const void* k_pool, const void* v_pool, int64_t src_layer_stride, const int32_t* src_table,
                           int32_t src_page_size, int32_t src_num_pages, int32_t src_max_pages_per_seq, void* k_codes,
                           void* v_codes, void* k_scales, void* v_scales, int64_t code_layer_stride,
                           int64_t scale_layer_stride, const int32_t* block_table, int32_t page_size,
                           int32_t num_pages, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t max_len,
                           int32_t layers, int32_t batch, int32_t n_kv, int32_t head_dim, void* stream);

/* pop_k_rope_cache for the 8-bit cache (paper Eq. 2-3; Eq. 14 with n_q = 0), with a position per sequence and rotations
 * over several axes. in: projections [q heads | k heads | v heads] * hd, fp32 or (in_bf16) bf16, row stride ld_in (a
 * multiple of 4; 16-byte aligned). Sequence b owns the packed rows cu_rows[b] .. cu_rows[b + 1] - 1 (device int32
 * [batch + 1], at most max_rows each), or rows b * max_rows .. if cu_rows is NULL; its first row goes to cache position
 * start[b] (device int32 [batch]) or pos0 for all if start is NULL. Per row: optional per-head RMSNorm of q and k
 * (q_gain / k_gain fp32 [hd] or NULL; eps), rotation of q and k, q to q_out (bf16, row stride ldq, a multiple of 4), k and
 * v to the cache.
 *   Rotation: pair (j, j + hd/2) turns by rope_table[p][j] = (cos, sin), float2 [table_rows][hd/2]. p is the cache position
 * if positions is NULL, else positions[axis * ld_pos + row] (device int32 [n_axes][ld_pos], row = packed row) with axis =
 * pair_axis[j] (device uint8 [hd/2], 4-byte aligned, values < n_axes; NULL: axis 0): time, height and width of image and
 * video tokens, in sections or interleaved as the model has it.
 *   Scales: a block whose 16 positions all come from this call, or whose earlier positions are all new, gets the scale of its
 * rows. A block that holds earlier positions (start not a multiple of 16) keeps the larger of its scale and the one the new
 * rows need, and its codes are brought to it. Positions at or behind `start` count as empty, whatever is there: a sequence
 * may be cut back and appended to again. Two sequences of one call may share pages only in front of both starts' blocks. */
int pop_k_rope_cache_e4m3(const void* in, int32_t in_bf16, int64_t ld_in, const int32_t* cu_rows, int32_t max_rows,
                          const int32_t* start, int32_t pos0, int32_t batch, void* q_out, int64_t ldq, void* k_codes,
                          void* v_codes, void* k_scales, void* v_scales, const int32_t* block_table, int32_t page_size,
                          int32_t num_pages, int32_t max_pages_per_seq, const float* q_gain, const float* k_gain,
                          float eps, const void* rope_table, int32_t table_rows, const int32_t* positions,
                          int64_t ld_pos, const void* pair_axis, int32_t n_axes, int32_t n_q, int32_t n_kv,
                          int32_t head_dim, void* stream);

/* Workspace of the two calls below: device memory, 16-byte aligned, contents irrelevant before and after. This size
 * covers every call; a smaller one is refused with POP_E_NOSPACE where the call needs more, NULL is taken where it needs
 * none. Calls that may overlap on the GPU (other streams, concurrently replayed graphs) need one each. */
#define POP_E4M3_WORKSPACE_BYTES (64 * 1024 * 1024)

/* pop_k_decode_attention over the 8-bit cache, with a length per sequence: one query per sequence at position
 * len - 1, len = seq_lens[b] (device int32 [batch], each <= kv_len) or kv_len for all if seq_lens is NULL, over the last
 * `window` positions (0: all). q bf16 [batch][ldq], out bf16 [batch][ldo] (strides multiples of 8, ldo >= n_q hd, 16-byte
 * aligned), any n_q that is a multiple of n_kv. A sequence of length 0 gets a row of zeros. batch <= 4096. Unequal lengths are
 * shared out over the whole GPU; results do not depend on scheduling. Blocks of 16 positions have 32-bit numbers, in the pool
 * (num_pages n_kv page_size / 16 < 2^31) and in the call (batch n_kv ceil(n_q / n_kv / 8) + 1 times the blocks of kv_len, or
 * of the window, < 2^31); a larger call is refused with POP_E_INVALID. */
int pop_k_decode_attention_e4m3(const void* q, int64_t ldq, const void* k_codes, const void* v_codes,
                                const void* k_scales, const void* v_scales, const int32_t* block_table,
                                int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq,
                                const int32_t* seq_lens, int32_t kv_len, void* workspace, size_t workspace_bytes,
                                void* out, int64_t ldo, int32_t batch, int32_t n_q, int32_t n_kv, int32_t head_dim,
                                int32_t window, void* stream);

/* pop_k_attention over the 8-bit cache: the last rows of each sequence are its queries (a whole prompt, a chunk of it,
 * a few drafted tokens). Sequence b has n = cu_rows[b + 1] - cu_rows[b] packed rows (device int32 [batch + 1], each n <=
 * max_rows), or max_rows rows each if cu_rows is NULL, and len cached positions (seq_lens / kv_len as above) which include
 * the rows' own: row i sits at position len - n + i and sees positions j <= its own, and j > its own - window if window > 0.
 * A row that sees nothing (a length below its sequence's rows) becomes zeros. Rows of no sequence are left as they are.
 * Pages in front of the window of every query are not read: their table entries may be anything (decode: the same). NaN
 * codes inside the part of a sequence that some row of the call sees may reach rows that do not see them. A row that sees a
 * position and has an infinite or NaN query element is NaN. Refused with POP_E_INVALID: num_pages n_kv page_size above
 * 2^31 - 16; max_rows above 131070 (hd 256: 65535) times floor(128 / min(128, n_q / n_kv)); where max_rows n_q / n_kv is 32 or
 * less, the decode call's limit on the blocks of the call with that product in place of n_q / n_kv. */
int pop_k_attention_e4m3(const void* q, int64_t ldq, const int32_t* cu_rows, int32_t max_rows, const void* k_codes,
                         const void* v_codes, const void* k_scales, const void* v_scales, const int32_t* block_table,
                         int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, const int32_t* seq_lens,
                         int32_t kv_len, void* workspace, size_t workspace_bytes, void* out, int64_t ldo,
                         int32_t batch, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t window, void* stream);

/* ---------------------------------------------------------------------------------------------------
 * A step that checks drafted tokens: several tokens of each sequence go through the full model at once (the decode stage of
 * paper Sec. 3.2 for more than one position), in the form of a tree whose rows each follow another row or the last cached
 * token. Projections of few rows with 4-bit weights, the append of the rows, their attention, and keeping of the path that was
 * accepted. Device-side checks as for the 8-bit cache: what the host cannot see (block-table entries, lengths, lists) is
 * never turned into an address where it is wrong; the status word is raised to POP_E_INVALID, and other sequences, and calls
 * made while the word holds POP_E_INVALID, are not touched by it.
 *
 * 4-bit weights W [N][K]: weight = (code - zero) * scale with codes 0 .. 15, and for every `group` (32, 64 or 128) consecutive
 * inputs of a row one scale (bf16) and one zero (uint8, 0 .. 15; zeros NULL: 8). They lie in tiles of 16 rows and 128 inputs:
 *   codes  uint8 [ceil(N / 16)][ceil(K / 128)][16][64]: the 64 bytes of a row are 16 32-bit words of 8 codes, word 4 t + j for
 *          inputs 32 j + 8 t .. + 7 of the 128; bits 4 p .. 4 p + 3 of a word are the code of its input 2 p (p < 4) or
 *          2 (p - 4) + 1;
 *   scales bf16, zeros uint8 [ceil(N / 16)][ceil(K / 128)][16][128 / group]: row r of the tile at index 2 (r % 8) + r / 8.
 * What lies behind row N or input K is read and has no effect, whatever it is. codes, scales and zeros 16-byte aligned.
 *
 * pop_k_gemv_w4: pop_k_gemv with such weights: out[b][n] = sum_k x[b][k] W[n][k], x bf16 [B][ldx] (16-byte aligned, ldx and K
 * multiples of 8), B up to 65535 (made for 1 to some dozens of rows). Modes as pop_k_gemv: 0 fp32 store, 2 fp32 +=, 3 gated -> bf16
 * (N a multiple of 256: 128 gate rows, then the 128 matching up rows; act 0 SiLU, 1 tanh-GELU). The products of
 * codes and activations are exact (of activations within 2^-28 of the largest of their 128 inputs; smaller ones are off by at
 * most 2^-36 of it); sums are fp32, in an order that depends on the sizes alone, in units of 2^-24 (results below 2^-101 lose
 * digits, as subnormals do). An activation row with an infinite or NaN input gives a row of NaN. Weights are read ahead, before
 * the kernel in front of the call on the stream has ended (as pop_k_gemv reads its own): whoever writes them on the GPU
 * synchronises before the first call that uses them. */
int pop_k_gemv_w4(const void* x, int64_t ldx, const void* codes, const void* scales, const void* zeros, int32_t group,
                  void* workspace, size_t workspace_bytes, void* out, int64_t ldo, int32_t B, int32_t N, int32_t K,
                  int32_t mode, int32_t act, int32_t n_valid, void* stream);
/* Bytes of device workspace (16-byte aligned, contents irrelevant before and after; one for each of calls that may overlap)
 * that the call needs for its activations; 0 for one or two rows and for small products, where workspace may be NULL. A smaller
 * one is POP_E_NOSPACE. */
size_t pop_k_gemv_w4_workspace_bytes(int32_t B, int32_t N, int32_t K, int32_t group);

/* pop_k_rope_cache for drafted rows. in: projections [q heads | k heads | v heads] * hd of `rows` packed rows, fp32 or
 * (in_bf16) bf16, row stride ld_in (a multiple of 4; 16-byte aligned). Sequence b owns rows cu_rows[b] .. cu_rows[b + 1] - 1
 * (device int32 [batch + 1], at most max_rows each), or rows b * max_rows .. if cu_rows is NULL; in front of them it has
 * start[b] cached positions (device int32 [batch]), or pos0 for all if start is NULL. Row i of the sequence goes to cache slot
 * start + i and has the rotary position start + depth[row] (device int32 [rows], row = packed row: 0 for rows that follow the
 * last cached token, one more than the row that it follows for the others; NULL: i, a chain). Per row: optional per-head
 * RMSNorm of q and k (q_gain / k_gain fp32 [hd] or NULL; eps), rotation of q and k by rope_table[position] (float2
 * [table_rows][hd/2], 16-byte aligned), q to q_out (bf16, row stride ldq, a multiple of 4; n_q may be 0), k and v to the
 * cache (one layer, pop_kv_cache_t's layout). A row whose position is outside the table is rotated by its row 0 (status word). */
int pop_k_rope_cache_tree(const void* in, int32_t in_bf16, int64_t ld_in, int32_t rows, const int32_t* cu_rows,
                          int32_t max_rows, const int32_t* start, int32_t pos0, const int32_t* depth, int32_t batch,
                          void* q_out, int64_t ldq, void* k_pool, void* v_pool, const int32_t* block_table,
                          int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, const float* q_gain,
                          const float* k_gain, float eps, const void* rope_table, int32_t table_rows, int32_t n_q,
                          int32_t n_kv, int32_t head_dim, void* stream);

/* Workspace of the call below: device memory, 16-byte aligned, contents irrelevant before and after. This size covers every
 * call. How much a call asks for depends on head_dim, batch and the GPU's SMs and not on lengths, so that a call that is taken
 * for one length is taken for all; a smaller one, or NULL, is refused with POP_E_NOSPACE (calls of a few short sequences ask
 * for it too, though they leave it as it is). Calls that may overlap on the GPU (other streams, concurrently replayed graphs)
 * need one each. */
#define POP_TREE_WORKSPACE_BYTES (64 * 1024 * 1024)

/* Attention of drafted rows over the paged cache (one layer) that has them already: packed rows, cu_rows, max_rows and start
 * as above (start[b] <= max_start; max_start for all if start is NULL). Row i sees the start positions in front of the draft,
 * and of the sequence's drafted slots those whose bit is set in its mask: mask device uint32 [rows][mask_words], slot j is bit
 * j % 32 of word j / 32 (mask_words * 32 >= max_rows; the row's own slot is a bit like the others; bits behind the sequence's
 * rows have no effect; NULL: slots 0 .. i, a chain). window > 0: only of positions within the last `window` of the row's, its
 * own included; a drafted slot's position is start + its depth (as above; NULL: a chain).
 * q bf16 [rows][ldq], out bf16 [rows][ldo] (strides multiples of 8, at least n_q hd; 16-byte aligned), n_q / n_kv <= 128,
 * batch <= 4096, hd 64, 128 or 256. A row that sees nothing becomes zeros; rows of no sequence are left as they are. Positions
 * behind a sequence's rows and in front of every row's window may hold anything, their block-table entries too where a whole
 * page does. An infinite or NaN value in a drafted slot, or in a position that is in front of some rows' windows, may reach rows
 * of the sequence that do not see it. Scores, maxima and sums are fp32; the softmax's weights enter the product with V as bf16
 * (the sum that divides takes them before that rounding), as in the library's other attention calls over bf16. Unequal
 * lengths are shared out over the whole GPU; results do not depend on scheduling. The key tiles of 64 positions of the call,
 * batch n_kv ceil(max_rows / rows per tile) ceil((max_start + max_rows) / 64), are at most 2^30 (POP_E_INVALID otherwise). */
int pop_k_tree_attention(const void* q, int64_t ldq, int32_t rows, const int32_t* cu_rows, int32_t max_rows,
                         const int32_t* start, int32_t max_start, const void* mask, int32_t mask_words,
                         const int32_t* depth, const void* k_pool, const void* v_pool, const int32_t* block_table,
                         int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, void* workspace,
                         size_t workspace_bytes, void* out, int64_t ldo, int32_t batch, int32_t n_q, int32_t n_kv,
                         int32_t head_dim, int32_t window, void* stream);

/* Keeps the accepted path of every sequence: the entries of drafted slots kept[b][0] < kept[b][1] < ... move to slots 0, 1,
 * ... of the draft (cache positions start + i), in `layers` consecutive layers (layer_stride elements apart, a page of one
 * layer at least) of K and V.
 * kept: device int32 [batch][ld_kept], the first n_kept[b] (device int32 [batch], at most max_kept; NULL: max_kept) of a
 * row; max_kept <= 1024. start / pos0 as above. The other entries stay as they are. A sequence whose list does not rise or
 * leaves its block table or the pool is left as it is (status word). */
int pop_k_cache_keep(void* k_pool, void* v_pool, int64_t layer_stride, int32_t layers, const int32_t* block_table,
                     int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, const int32_t* kept,
                     int64_t ld_kept, const int32_t* n_kept, int32_t max_kept, const int32_t* start, int32_t pos0,
                     int32_t batch, int32_t n_kv, int32_t head_dim, void* stream);

/* The four calls above (call 0 pop_k_gemv_w4, 1 pop_k_rope_cache_tree, 2 pop_k_tree_attention, 3 pop_k_cache_keep) with their
 * arguments as 64-bit words in their order: pointers, integers, and eps as the bits of a double. For callers whose foreign
 * function interface converts argument by argument, which for these calls can cost as much as the launch. */
int pop_k_packed(int32_t call, const int64_t* words);

/* Synchronise the stream, then read and clear the library's device status word. */
int pop_k_status(void* stream);

/* Self-test of the library's failure path (no counterpart in the paper). Every device-side wait of
 * the GEMM and attention kernels (on an mbarrier that a TMA copy or a tensor-core commit completes)
 * is bounded: when it runs out, the kernel raises the status word to POP_E_DEVICE_TIMEOUT, unwinds and
 * returns, and kernels launched while the word is raised return at once. This call launches one small
 * kernel that performs that very wait on a barrier nothing arrives at, for at most limit_cycles SM
 * cycles (1 .. 1 000 000, i.e. well under a millisecond; POP_E_INVALID otherwise), so the path can be
 * exercised without a fault, a trap or an endless loop: afterwards pop_k_status returns
 * POP_E_DEVICE_TIMEOUT once and POP_OK from then on. */
int pop_k_wait_selftest(int64_t limit_cycles, void* stream);

/* Per-kernel timing for benchmarks. pop_k_profile(1) makes every launch of this library record a
 * CUDA-event pair on its stream; pop_k_profile_summary waits for the recorded events of one kind
 * (0 projection GEMM, 1 prefill attention, 2 elementwise, 3 GEMV, 4 decode attention), returns
 * their summed duration in ms, their summed algorithmic work (flops for kinds 0-1, bytes
 * otherwise) and their count, and forgets them. Off by default; costs nothing when off. */
void pop_k_profile(int32_t enable);
int pop_k_profile_summary(int32_t kind, double* total_ms, double* total_work, int64_t* launches);

/* Kernel launches enqueued by this library since the last pop_k_reset_launch_count(). */
int64_t pop_k_launch_count(void);
void pop_k_reset_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* POP_KERNELS_H_ */
