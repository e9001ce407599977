/*
 * pipo_ops.h -- the decoder's individual GPU operations, exposed for unit
 * tests and profiling.  Each call enqueues one operation of the layer
 * computation (PIPO's "Computation" task, Section 3.1.2) on `stream`
 * (a hipStream_t, or NULL for the default stream) and returns without
 * waiting.  All tensor pointers are device pointers unless stated;
 * ownership stays with the caller.  Shapes outside a kernel's range return
 * PIPO_ERR_UNSUPPORTED before anything is launched.
 */
#ifndef PIPO_OPS_H
#define PIPO_OPS_H

#include "pipo.h"

#ifdef __cplusplus
extern "C" {
#endif

/* --- device memory helpers (so tests need no other GPU runtime) --- */
pipo_status pipo_dev_alloc(size_t bytes, void** out);
pipo_status pipo_dev_free(void* p);
pipo_status pipo_copy_h2d(void* dst_dev, const void* src_host, size_t bytes);
pipo_status pipo_copy_d2h(void* dst_host, const void* src_dev, size_t bytes);
pipo_status pipo_dev_synchronize(void);

/* GEMM epilogues: acc = X[m] . W[n] (fp32), then
 *   PIPO_EPI_F16:       out_f16[m][n] = acc + bias[n]
 *   PIPO_EPI_RELU_F16:  out_f16[m][n] = max(acc + bias[n], 0)
 *   PIPO_EPI_ADD_F32:   out_f32[m][n] += acc + bias[n]     (residual stream)
 *   PIPO_EPI_F32:       out_f32[m][n] = acc + bias[n]      (logits)
 * bias may be NULL (treated as 0).
 *   PIPO_EPI_SWIGLU:    the gated MLP's SwiGLU (LLaMA): W stacks the gate rows
 *                       [0, F) over the up rows [F, 2F) (N = 2F, even), bias
 *                       must be NULL, out_f16 has F columns (row stride F):
 *                       out_f16[m][i] = silu(g) * u in fp32, rounded once, with
 *                       g = fp16(acc of row i), u = fp16(acc of row F + i),
 *                       silu(g) = g / (1 + exp(-g)); the same values as
 *                       PIPO_EPI_F16 followed by pipo_op_swiglu.  Only for
 *                       M <= 16 (else PIPO_ERR_UNSUPPORTED). */
enum { PIPO_EPI_F16 = 0, PIPO_EPI_RELU_F16 = 1, PIPO_EPI_ADD_F32 = 2, PIPO_EPI_F32 = 3,
       PIPO_EPI_SWIGLU = 5 };

/*
 * Y = X . W^T with the chosen epilogue (the projections of a layer and the
 * output head).  X: [M][K] fp16 (row stride K); W: [N][K] fp16; out: [M][N]
 * (row stride N), fp16 or fp32 per epilogue ([M][N/2] fp16 for
 * PIPO_EPI_SWIGLU).  K must be a multiple of 128 and M below 2^31 (else
 * PIPO_ERR_UNSUPPORTED).
 * For M > 16 the K range may be split over workgroups whose fp32 partial
 * sums go to `workspace` (device, caller-owned, contents arbitrary) of
 * pipo_op_gemm_workspace_bytes(M, N, K, wfmt) bytes; a second kernel adds
 * them in a fixed order and applies the epilogue.  With less (or NULL)
 * workspace the GEMM takes the tiles that run best with the K ranges that
 * fit, or unsplit; the result is the same up to rounding.  Calls sharing a workspace must not
 * overlap in time.  Operands run fastest with X and the weights on 16-byte
 * boundaries and the (scale, min) pairs on 4-byte ones; any other address is
 * taken too.  For a given (M, N, K, wfmt, epilogue), alignment and
 * room in the workspace the summation order is fixed, so repeated calls give
 * the same bits.
 */
pipo_status pipo_op_gemm_f16(const uint16_t* X, const uint16_t* W, const uint16_t* bias,
                             void* out, int64_t M, int64_t N, int64_t K, int32_t epi,
                             void* workspace, int64_t workspace_bytes, void* stream);

/* Same with group-wise INT4 W (pipo_q4 layout, device pointers): the codes
 * are expanded to fp16 inside the GEMM (Section 3.4), never in HBM; every
 * code becomes code * scale + min rounded once to fp16. */
pipo_status pipo_op_gemm_w4(const uint16_t* X, const uint8_t* Wq, const uint16_t* Wsm,
                            const uint16_t* bias, void* out, int64_t M, int64_t N, int64_t K,
                            int32_t epi, void* workspace, int64_t workspace_bytes,
                            void* stream);

/* The same two GEMMs with W (or Wq, Wsm) in PIPO_LAYOUT_FRAGMENT order
 * (pipo.h; N % 16 == 0): the same products in the same summation order, so
 * with aligned operands and the same workspace the result equals the row-major
 * call bit for bit. */
pipo_status pipo_op_gemm_f16_frag(const uint16_t* X, const uint16_t* W, const uint16_t* bias,
                                  void* out, int64_t M, int64_t N, int64_t K, int32_t epi,
                                  void* workspace, int64_t workspace_bytes, void* stream);
pipo_status pipo_op_gemm_w4_frag(const uint16_t* X, const uint8_t* Wq, const uint16_t* Wsm,
                                 const uint16_t* bias, void* out, int64_t M, int64_t N,
                                 int64_t K, int32_t epi, void* workspace,
                                 int64_t workspace_bytes, void* stream);

/* Workspace bytes the GEMM of this shape uses to split K (0: never splits).
 * wfmt: PIPO_W_FP16 or PIPO_W_INT4_G64. */
int64_t pipo_op_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int32_t wfmt);

/* y[r][:] = LN(x[r*src_stride + src_offset][:]) * gamma + beta, r < rows;
 * x fp32 [.][d], y fp16 [rows][d], statistics in fp32. */
pipo_status pipo_op_layernorm(const float* x, const uint16_t* gamma, const uint16_t* beta,
                              uint16_t* y, int64_t rows, int64_t d, int64_t src_stride,
                              int64_t src_offset, float eps, void* stream);

/*
 * Decode attention for b sequences at position t (keys 0..t visible).
 * q: [b][d] fp16 (already scaled by head_dim^-1/2); kc, vc: KV cache
 * [>= t+1][b][d] fp16 (position-major: row p*b + i holds sequence i's key at
 * position p); o: [b][d] fp16.  head_dim 64 or 128, t + 1 <= 65536 (beyond:
 * PIPO_ERR_UNSUPPORTED).
 * When b * n_heads is small the keys are split over several workgroups and
 * a second kernel merges the splits in order; the partials need `workspace`
 * (device, caller-owned, contents arbitrary) of
 * pipo_op_attn_decode_workspace_bytes(b, n_heads, head_dim, t) bytes.  With
 * less (or NULL) the kernel runs unsplit; the result is the same up to
 * rounding.  Calls sharing a workspace must not overlap in time.  The
 * workspace size covers this call and pipo_op_attn_decode_kv4 alike.
 */
pipo_status pipo_op_attn_decode(const uint16_t* q, const uint16_t* kc, const uint16_t* vc,
                                uint16_t* o, int32_t b, int32_t n_heads, int32_t head_dim,
                                int32_t t, void* workspace, int64_t workspace_bytes,
                                void* stream);
int64_t pipo_op_attn_decode_workspace_bytes(int32_t b, int32_t n_heads, int32_t head_dim,
                                            int32_t t);

/*
 * pipo_op_attn_decode for callers that cannot allocate device memory (code
 * under HIP graph capture, serving loops, harnesses that forbid
 * hipMalloc): the same kernels, split choice and result bit for bit as
 * pipo_op_attn_decode with a sufficient workspace, but the split partials
 * go to one fixed 4 MiB array of the library on each device (held until
 * the process ends) instead of a caller workspace; nothing is allocated.
 * Every shape this kernel accepts needs at most about 0.8 MB of it; a
 * shape that would need more returns PIPO_ERR_UNSUPPORTED.  All calls on a
 * device share that array, so calls that overlap in time on one device
 * (on different streams, or from several threads) race and must be
 * serialised by the caller.  The array's contents are arbitrary between
 * calls (every partial is written before it is read).
 */
pipo_status pipo_op_attn_decode_noalloc(const uint16_t* q, const uint16_t* kc,
                                        const uint16_t* vc, uint16_t* o, int32_t b,
                                        int32_t n_heads, int32_t head_dim, int32_t t,
                                        void* stream);

/* The same over an INT4 KV cache (PIPO_KV_INT4_G64 rows of 9d/16 bytes,
 * position-major like the fp16 cache; d % 256 == 0): every key and value
 * is read as code * scale + min, in fp32.  Same workspace. */
pipo_status pipo_op_attn_decode_kv4(const uint16_t* q, const uint8_t* kc, const uint8_t* vc,
                                    uint16_t* o, int32_t b, int32_t n_heads, int32_t head_dim,
                                    int32_t t, void* workspace, int64_t workspace_bytes,
                                    void* stream);

/* INT4 KV cache rows (Section 2; the conversion is part of saving and
 * loading the cache, Section 3.1.2): quantize `rows` fp16 rows x [rows][d]
 * into out [rows][9d/16 bytes] with the PIPO_KV_INT4_G64 recipe (pipo.h),
 * or expand INT4 rows back to fp16 y [rows][d].  d % 256 == 0. */
pipo_status pipo_op_kv_quant(const uint16_t* x, uint8_t* out, int64_t rows, int64_t d,
                             void* stream);
pipo_status pipo_op_kv_dequant(const uint8_t* in, uint16_t* y, int64_t rows, int64_t d,
                               void* stream);

/*
 * Causal prefill attention over P positions of b sequences.
 * q: [b][P][d] fp16 (scaled); kc, vc: [>= P][b][d] position-major as
 * above; o: [b][P][d] fp16.  head_dim 64 or 128.  b * d * 64 (64 cached
 * positions of every sequence) must stay below 2^31 elements, else
 * PIPO_ERR_UNSUPPORTED.
 */
pipo_status pipo_op_attn_prefill(const uint16_t* q, const uint16_t* kc, const uint16_t* vc,
                                 uint16_t* o, int32_t b, int32_t P, int32_t n_heads,
                                 int32_t head_dim, void* stream);

/* --- LLaMA-family operations (PIPO_FAMILY_LLAMA in pipo.h) --- */

/* Grouped-query decode attention: q [b][n_heads * head_dim], cache rows of
 * n_kv_heads * head_dim (fp16, or PIPO_KV_INT4_G64 rows when kv_fmt says
 * so, then n_kv_heads * head_dim % 256 == 0); query head h reads key/value
 * head h / (n_heads / n_kv_heads), 1, 2, 4 or 8 query heads per key/value
 * head.  One workgroup serves all query heads of a key/value head, so each
 * cached row is read once.  Workspace as for pipo_op_attn_decode, sized by
 * pipo_op_attn_decode_gqa_workspace_bytes. */
pipo_status pipo_op_attn_decode_gqa(const uint16_t* q, const void* kc, const void* vc,
                                    uint16_t* o, int32_t b, int32_t n_heads, int32_t n_kv_heads,
                                    int32_t head_dim, int32_t t, int32_t kv_fmt, void* workspace,
                                    int64_t workspace_bytes, void* stream);
int64_t pipo_op_attn_decode_gqa_workspace_bytes(int32_t b, int32_t n_heads, int32_t n_kv_heads,
                                                int32_t head_dim, int32_t t);

/* Grouped-query causal prefill attention (layouts as pipo_op_attn_prefill,
 * cache rows of n_kv_heads * head_dim). */
pipo_status pipo_op_attn_prefill_gqa(const uint16_t* q, const uint16_t* kc, const uint16_t* vc,
                                     uint16_t* o, int32_t b, int32_t P, int32_t n_heads,
                                     int32_t n_kv_heads, int32_t head_dim, void* stream);

/* RMSNorm: y[r][:] = x[src] / sqrt(mean(x[src]^2) + eps) * gamma with
 * src = r*src_stride + src_offset; x fp32, y fp16, statistics in fp32. */
pipo_status pipo_op_rmsnorm(const float* x, const uint16_t* gamma, uint16_t* y, int64_t rows,
                            int64_t d, int64_t src_stride, int64_t src_offset, float eps,
                            void* stream);

/*
 * Rotary positions, in place (pipo.h, PIPO_FAMILY_LLAMA).  Row m (m < M)
 * is sequence m / rows_per_seq at position pos0 + m % rows_per_seq.
 * q: [M][n_heads * head_dim] fp16, each head rotated and then multiplied by
 * q_scale; k: rows (kpos0 + m % rows_per_seq) * batch + m / rows_per_seq of
 * [.][n_kv_heads * head_dim] fp16 (a position-major cache, or with kpos0 = 0
 * a staging buffer), rotated.  cos_sin: device fp32 [positions][head_dim/2]
 * [2] = (cos, sin) of p * w_i (pipo_rope_table).  head_dim 64 or 128.
 */
pipo_status pipo_op_rope(uint16_t* q, uint16_t* k, const float* cos_sin, int64_t M,
                         int64_t rows_per_seq, int64_t pos0, int64_t kpos0, int64_t batch,
                         int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float q_scale,
                         void* stream);

/* The rotary table of a LLaMA shape on the host: out[p][i][2] = (cos, sin)
 * of p * w_i (w_i as in pipo.h, with the 3.1 scaling when rope_factor >
 * 0), computed in double and stored as fp32, for p < n_pos and i <
 * head_dim / 2.  `out` holds n_pos * head_dim floats.  Errors: ARG. */
pipo_status pipo_rope_table(const pipo_shape* shape, int32_t n_pos, float* out);

/* --- batches of sequences of different lengths over a paged 4-bit KV cache ---
 *
 * Keys and values live in pages of `page_size` positions (16, 32, 64, 128 or
 * 256), each page holding all n_kv_heads heads (head_dim 64 or 128) of its
 * positions, 4 bits an element in groups of 64 with the recipe of
 * PIPO_KV_INT4_G64.  Sequence i of n_seq keeps the positions p * page_size ..
 * of its cache in page table[i * table_stride + p]; which pages are free is for
 * the caller (or pipo_op_kv_pages_resize and its neighbours) to say.  Every
 * layer has a pool of the same n_pages pages, the pools layer_bytes apart (a
 * multiple of 16, at least n_pages * pipo_kv_page_bytes), and one table serves
 * them all.  A page's bytes are in the order the kernels read fastest
 * (kvpages.h); they are written by pipo_op_kv_pages_append and may be moved
 * whole.  `pool` (16-byte aligned) and `table` are device pointers, the
 * struct itself is read on the host during the call.
 *
 * Positions, sequences, pages and lengths come from device memory, where the
 * host cannot check them.  No value of theirs makes a call read or write
 * outside the arrays it was given: what a wrong one does is said at each
 * call.
 */
typedef struct {
  void* pool;
  int64_t layer_bytes;
  const int32_t* table;
  int64_t table_stride;
  int32_t n_layers, n_pages, page_size, n_kv_heads, head_dim, n_seq;
} pipo_kv_pages;

/* Bytes of a page of one layer, page_size * n_kv_heads * 9 head_dim / 8; 0 for
 * a shape that is not supported (see above; 2^31 bytes or more). */
int64_t pipo_kv_page_bytes(int32_t page_size, int32_t n_kv_heads, int32_t head_dim);

/*
 * Per-head RMSNorm of q and k and their rotary positions in one pass, each row
 * at a position of its own: with y = x / sqrt(mean(x^2) + eps) * gamma over a
 * head's head_dim elements (q_gamma, k_gamma [head_dim] fp16; NULL: y = x),
 * q_out = rotate(y) * q_scale and k_out = rotate(y), the rotation being
 * pipo_op_rope's by row pos[m] of cos_sin [n_pos][head_dim/2][2]; in fp32,
 * rounded once.  Row m of q starts at q + m * ldq and holds n_heads heads (k:
 * ldk, n_kv_heads), so both may lie in the rows of a fused projection; q_out
 * may be q with ldqo = ldq (k_out likewise), other overlaps are not allowed.
 * A row whose position is negative or not below n_pos is left as it was
 * (padding).  head_dim 64 or 128 and M below 2^31, else PIPO_ERR_UNSUPPORTED.
 * Rows on 16 bytes run fastest.
 */
pipo_status pipo_op_qk_norm_rope(const uint16_t* q, int64_t ldq, const uint16_t* k, int64_t ldk,
                                 const uint16_t* q_gamma, const uint16_t* k_gamma,
                                 const float* cos_sin, int64_t n_pos, const int32_t* pos,
                                 uint16_t* q_out, int64_t ldqo, uint16_t* k_out, int64_t ldko,
                                 int64_t M, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                 float eps, float q_scale, void* stream);

/*
 * Rows of new keys and values into the pages of `layer`: row m of k and v
 * (fp16, n_kv_heads * head_dim elements at k + m * ldk and v + m * ldv) becomes
 * position pos[m] of sequence seq[m], quantized with the recipe of
 * PIPO_KV_INT4_G64; elements are first clamped to +-57344 and NaN counts as
 * 0, so that what the cache holds is finite.  A row is skipped where seq[m] is
 * not in [0, n_seq), pos[m] is negative or past the table's row, or the table's
 * entry is not a page.  No two rows of a call may name the same position of
 * the same page (one of them, or a mixture, stays).
 */
pipo_status pipo_op_kv_pages_append(const pipo_kv_pages* cache, int32_t layer, const int32_t* seq,
                                    const int32_t* pos, const uint16_t* k, int64_t ldk,
                                    const uint16_t* v, int64_t ldv, int64_t M, void* stream);

/* The reverse: position pos[m] of sequence seq[m] to row m of k and v, code *
 * scale + min rounded once to fp16.  Rows that append would skip are left as
 * they were. */
pipo_status pipo_op_kv_pages_read(const pipo_kv_pages* cache, int32_t layer, const int32_t* seq,
                                  const int32_t* pos, uint16_t* k, int64_t ldk, uint16_t* v,
                                  int64_t ldv, int64_t M, void* stream);

/*
 * Causal attention of each sequence's newest rows over its pages.  Rows
 * q_start[i] .. q_start[i+1] - 1 of q (fp16, scaled, n_heads * head_dim
 * elements at q + m * ldq; o and ldo alike) are the last positions of sequence
 * i, whose keys 0 .. kv_len[i] - 1 (its own rows' included) are in the cache:
 * with n rows, row j sits at position kv_len[i] - n + j and sees the keys up to
 * that position.  q_start has n_seq + 1 entries that do not decrease.  Query
 * head h reads key/value head h / (n_heads / n_kv_heads), any whole ratio.
 * Every key and value is read as code * scale + min; softmax and sums in fp32,
 * the output rounded once to fp16.  Where a sequence may have more than 64 rows
 * times query heads of a key/value head, each weight times a value's scale is
 * rounded to fp16 as well, which adds up to as much as the output's own rounding.
 *
 * M: rows of q and o; max_q, max_len: bounds of a sequence's rows and keys that
 * the host knows (max_len at most table_stride * page_size).  A length above
 * max_len counts as max_len, a start outside [0, M] as the nearer end, and of a
 * sequence of more than max_q rows those past the max_q-th are left as they were.
 * Keys on an entry of the table that is not a page are not seen, a row that
 * sees no key becomes 0, rows outside q_start[0] .. q_start[n_seq] - 1 are left
 * as they were.
 *
 * Where there are few sequences their keys are split over workgroups, whose
 * partials go to `workspace` (device, caller-owned, contents arbitrary, 16-byte
 * aligned) of pipo_op_attn_pages_workspace_bytes bytes for a second kernel to
 * merge in order; with less (or NULL) they are not split: the same result up
 * to rounding.  Calls sharing a workspace must not overlap in time.  The
 * order of all sums is fixed by the arguments of the call.
 * n_heads and n_seq up to 65535, n_seq * n_kv_heads below 2^22, max_len up to
 * 2^30, min(M, max_q) * n_heads up to 2^29 - 2^22 and M * n_heads below 2^30,
 * else PIPO_ERR_UNSUPPORTED.
 */
pipo_status pipo_op_attn_pages(const pipo_kv_pages* cache, int32_t layer, const uint16_t* q,
                               int64_t ldq, const int32_t* q_start, const int32_t* kv_len,
                               uint16_t* o, int64_t ldo, int32_t n_heads, int64_t M, int32_t max_q,
                               int32_t max_len, void* workspace, int64_t workspace_bytes,
                               void* stream);
/* (pool and table of `cache` are not read; 0 for a call that would be refused
 * or never splits) */
int64_t pipo_op_attn_pages_workspace_bytes(const pipo_kv_pages* cache, int32_t n_heads, int64_t M,
                                           int32_t max_q, int32_t max_len);

/*
 * Page tables.  A sequence of len[i] tokens holds the first ceil(len[i] /
 * page_size) entries of its row (a negative length counts as 0), a page that
 * no row holds is free, and the same page may be in several rows (a shared
 * prefix).  The calls read a table [n_seq][table_stride] and lengths and write
 * the next ones, whose entries past a row's pages become -1.  resize and
 * compact may work in place (table_out = table, len_out = len); any other
 * overlap of an output with another array is PIPO_ERR_ARG.  Up to 2048
 * sequences, 2^20 pages and 2^31 - 1 table entries (else PIPO_ERR_UNSUPPORTED);
 * one workgroup does the work, so a captured decode loop can grow its
 * sequences without the host.
 *
 * resize: sequence i gets want[i] tokens (negative: it keeps its length).
 * Pages past ceil(want[i] / page_size) are given up, missing ones are the lowest
 * free pages (those given up in this call included), in order of the
 * sequences.  want[i] = 0 frees a sequence.  A sequence cut to end inside a page
 * that other rows hold too still shares it: what is appended to it there changes
 * theirs (forks alone never bring this about).  If there are too few pages, or a
 * row is too short, the table and lengths stay what they were and *missing
 * (device) is how many pages were lacking (2^31 - 1 for more than that), else 0.
 */
pipo_status pipo_op_kv_pages_resize(const int32_t* table, const int32_t* len, const int32_t* want,
                                    int32_t* table_out, int32_t* len_out, int64_t table_stride,
                                    int32_t n_seq, int32_t n_pages, int32_t page_size,
                                    int32_t* missing, void* stream);

/*
 * fork: sequence i < n_out of the output continues sequence parent[i] of the
 * input (outside [0, n_seq): it is empty).  Children share their parent's full
 * pages; a last page with room left stays with the parent's first child, and
 * each other child gets the lowest free page (free in the output, in order of
 * the children) and a pair (old page, new page) in `pairs` [n_out][2], for
 * pipo_op_kv_pages_copy.  *n_pairs and *missing are device counts; with
 * *missing > 0 pages lacking, *n_pairs is 0 and nothing else is written.
 */
pipo_status pipo_op_kv_pages_fork(const int32_t* table, const int32_t* len, int32_t n_seq,
                                  const int32_t* parent, int32_t* table_out, int32_t* len_out,
                                  int32_t n_out, int64_t table_stride, int32_t n_pages,
                                  int32_t page_size, int32_t* pairs, int32_t* n_pairs,
                                  int32_t* missing, void* stream);

/* compact: with U pages in use, those at U and above move, in order, to the
 * pages below U that are free; pairs [n_pages / 2][2] and *n_pairs say which
 * (old page, new page), for pipo_op_kv_pages_copy. */
pipo_status pipo_op_kv_pages_compact(const int32_t* table, const int32_t* len, int32_t* table_out,
                                     int64_t table_stride, int32_t n_seq, int32_t n_pages,
                                     int32_t page_size, int32_t* pairs, int32_t* n_pairs,
                                     void* stream);

/* Page pairs[i][0] onto page pairs[i][1] in every layer, for i below *n_pairs
 * (device; at most max_pairs count).  Pairs with an entry that is not a page
 * are skipped; a page that is written may be in no other pair. */
pipo_status pipo_op_kv_pages_copy(const pipo_kv_pages* cache, const int32_t* pairs,
                                  const int32_t* n_pairs, int32_t max_pairs, void* stream);

/* SwiGLU: h[m][i] = silu(gu[m][i]) * gu[m][F + i], silu(g) = g / (1 +
 * exp(-g)), in fp32; gu [M][2F], h [M][F] fp16, F % 8 == 0. */
pipo_status pipo_op_swiglu(const uint16_t* gu, uint16_t* h, int64_t M, int64_t F, void* stream);

/* Embedding: x[r][:] = tok_table[ids[r]] (+ pos_table[pos0 + r % rows_per_seq
 * + pos_offset] when pos_table is not NULL), fp32 x [rows][d]. */
pipo_status pipo_op_embed(const int32_t* ids, const uint16_t* tok_table, const uint16_t* pos_table,
                          float* x, int64_t rows, int64_t d, int64_t rows_per_seq, int64_t pos0,
                          int64_t pos_offset, void* stream);

/* next[r] = index of the largest logits[r][:] (ties: lowest index, NaNs
 * skipped; a row of NaNs gives 0).  rows <= 65535. */
pipo_status pipo_op_argmax(const float* logits, int32_t* next, int64_t rows, int64_t V,
                           void* stream);
/* The same with a row split over several workgroups whose candidates a
 * second kernel merges (same result); workspace (device, caller-owned,
 * contents arbitrary) of pipo_op_argmax_workspace_bytes(rows, V) bytes, or
 * less / NULL for the single-pass kernel. */
pipo_status pipo_op_argmax_ws(const float* logits, int32_t* next, int64_t rows, int64_t V,
                              void* workspace, int64_t workspace_bytes, void* stream);
int64_t pipo_op_argmax_workspace_bytes(int64_t rows, int64_t V);

/* Plain device-to-device copy kernel: reads and writes `bytes` once
 * (multiple of 16, 16-byte aligned pointers).  Not part of the decoder: it
 * gives a kernel of known HBM traffic for calibrating hardware counters. */
pipo_status pipo_op_copy(void* dst, const void* src, int64_t bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PIPO_OPS_H */
