/* libmcd: a paged KV cache of many utterances and the operators around it.
 *
 * mcd_outer (mcd_pipeline.h) decodes one utterance over a cache of its own.  A program that serves
 * many utterances of a Sec. 1 / Fig. 1 model (arXiv 2609.37007) has its layers' cache and attention
 * from these operators, their products from mcd_tc.h, and the row norms, residual sums and sampled tokens between them
 * from mcd_rows.h; activations are its own:
 *
 *   mcd_rope_append       the rows of the QKV product: per-head RMSNorm, rotary positions, K and V
 *                         into the cache's pages
 *   mcd_paged_attention   attention of every utterance's new rows over its pages: a single row, a
 *                         few drafted rows, a drafted tree (Fig. 2) or a whole prompt
 *   mcd_paged_attention_window   the same with a sliding window and a few first positions that stay visible, so that
 *                         an utterance of any length needs a bounded number of pages
 *   mcd_pages_fork        reorder, duplicate, extend and release utterances by reference counts
 *   mcd_pages_compact     move the kept tokens of every utterance together (accepted tree nodes,
 *                         positions kept when others are dropped)
 *
 * A cache is a pool of pages; a page holds page_size consecutive positions of one utterance in all
 * layers and KV heads.  An utterance (below: a sequence) is a row of a page table: entry c names
 * the page of positions c * page_size .., -1 past its last page.  Nothing here owns memory: pools,
 * tables, lengths and reference counts are the caller's.
 *
 * Conventions are those of mcd.h: a status is returned, nothing aborts across the ABI.  Every call
 * is asynchronous on `stream` (a cudaStream_t of the current device, or NULL for the default
 * stream), allocates nothing and can be captured into a graph.  Limits: 65,535 sequences, 1,024 KV heads,
 * fewer than 2^27 rows of a call (MCD_ERR_UNSUPPORTED beyond).  `err` (device int32, zeroed by the
 * caller) receives the first MCD_ERR_* of what only the device can check: lengths, page numbers and
 * parents that do not fit their bounds (MCD_ERR_INVALID_ARG), no free page left (MCD_ERR_OOM), a wait that
 * gave up (MCD_ERR_TIMEOUT).  No memory outside the given bounds is touched then.  Two calls that
 * may run at the same time need workspaces of their own.
 */
#ifndef MCD_CACHE_H
#define MCD_CACHE_H

#include "mcd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element (layer l, page p, KV head h, place t, dimension d) of k or v is at
 * l * layer_stride + p * page_stride + h * head_stride + t * token_stride + d (in elements; the
 * same strides for both, so any order of heads and places in a page will do).  Pointers are 16-byte
 * aligned and strides multiples of 16 bytes, at least head_dim (MCD_ERR_UNSUPPORTED otherwise); no
 * two elements share a place. */
typedef struct {
  void* k;
  void* v;
  int64_t layer_stride, page_stride, head_stride, token_stride;
  int32_t n_layers, n_pages, n_kv_heads;
  int32_t page_size;    /* 16, 32, 64 or 128                       */
  int32_t head_dim;     /* 64 or 128                                */
  int32_t dtype;        /* MCD_WEIGHT_F32 or MCD_WEIGHT_BF16        */
} mcd_paged_kv;

/* The new rows of one call.  Sequence s has cached[s] positions in the cache and brings rows
 * row_start[s] .. row_start[s + 1] - 1 (none is allowed) of the packed row buffers; row i of them
 * has position (slot) cached[s] + i, whose page is in the table before the call.  Rows from
 * row_start[n_seqs] on belong to nobody: they are not written, and what they hold touches nothing.
 * A sequence that does not fit the bounds below is skipped (MCD_ERR_INVALID_ARG in err; where row_start is
 * not ascending, others may be too); so is, by mcd_rope_append, a row whose page number is outside the
 * pool, while mcd_paged_attention gives the rows that read such a page unspecified values.
 * Any bounds that hold give the same rows (but for the rounding of sums taken in other parts); the launch
 * goes by them, so that tight ones are faster.  One bf16 row over 630 keys: 7.6 us, with a max_tokens of
 * 32,768 20 (as many parts as that would want).  128 single rows: 50.5 us, with a max_rows of 128 64 in bf16
 * (both kernels are launched) and 445 for 205 in fp32 (a CTA for every tile that there could be). */
typedef struct {
  const int32_t* table;      /* dev [n_seqs][table_stride]                              */
  const int32_t* cached;     /* dev [n_seqs]                                            */
  const int32_t* row_start;  /* dev [n_seqs + 1], ascending, within 0..n_rows           */
  int32_t n_seqs;
  int32_t table_stride;      /* entries per row of the table                            */
  int32_t n_rows;            /* rows of the packed buffers                              */
  int32_t max_rows;          /* bound on the rows of one sequence                       */
  int32_t max_tokens;        /* bound on cached[s] + rows, <= table_stride * page_size  */
} mcd_chunks;

/* Rotary positions: pair j (of rot_dim / 2) of a head is turned by position * inv_freq[j] radians
 * and multiplied by `scale`.  Pairs are (j, j + rot_dim / 2), or (2 j, 2 j + 1) when interleaved;
 * dimensions from rot_dim on stay as they are.  rot_dim is a multiple of 16 up to head_dim, or 0:
 * no rotation. */
typedef struct {
  const double* inv_freq;    /* dev [rot_dim / 2]                                       */
  float scale;               /* 1, or the factor that mcd_rope_freqs gives               */
  int32_t rot_dim;
  int32_t interleaved;
} mcd_rope;

/* Frequencies (host, double [rot_dim / 2]) of inv_freq: w_j = base^(-2 j / rot_dim), stretched for
 * contexts `factor` times as long as the model was trained on:
 *   MCD_ROPE_PLAIN     w_j (factor is 1)
 *   MCD_ROPE_LINEAR    w_j / factor
 *   MCD_ROPE_BASE      w_j of the base base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is
 *                      stretched by factor, the fastest not at all
 *   MCD_ROPE_BY_PARTS  per pair (YaRN, Peng et al. 2023): with r = train_tokens * w_j / (2 pi) turns
 *                      over the trained context, w_j where r >= beta_fast, w_j / factor where
 *                      r <= beta_slow, between them mixed in proportion to the pair's number:
 *                      g = clamp((j - lo) / (hi - lo), 0, 1), w_j (1 - g) + (w_j / factor) g,
 *                      lo / hi the (real) pair numbers where r = beta_fast / beta_slow
 * scale (host, optional) receives the factor for mcd_rope.scale: 0.1 ln(factor) + 1 by parts, else
 * 1.  rot_dim even (above 2 with MCD_ROPE_BASE), base > 1, factor >= 1; by parts train_tokens >= 1 and
 * beta_fast > beta_slow > 0: MCD_ERR_INVALID_ARG otherwise. */
enum { MCD_ROPE_PLAIN = 0, MCD_ROPE_LINEAR = 1, MCD_ROPE_BASE = 2, MCD_ROPE_BY_PARTS = 3 };
mcd_status mcd_rope_freqs(int32_t kind, int32_t rot_dim, double base, double factor, int32_t train_tokens,
                          double beta_fast, double beta_slow, double* inv_freq, float* scale);

/* Rows of a QKV product into the cache: for every new row, its n_q_heads query heads and the
 * cache's n_kv_heads key heads are normalised (x * gain / sqrt(mean x^2 + eps), per head, gains
 * q_norm / k_norm: dev float [head_dim], NULL for none), rotated and rounded once to the cache's type:
 * queries to q_out, keys to the row's slot of `layer`; value heads go there as they are.
 *   qkv        dev [n_rows][qkv_stride], qkv_dtype MCD_WEIGHT_F32 or, for a bf16 cache, also
 *              MCD_WEIGHT_BF16: query, key and value heads one after another
 *   q_out      dev [n_rows][q_stride] in the cache's type
 *   positions  dev int32 [n_rows], optional: the rows' positions for the rotation (a drafted tree's
 *              rows: their depths'); NULL: their slots
 * Row strides in elements, rows and gains 16-byte aligned, n_q_heads at most 4,096 (MCD_ERR_UNSUPPORTED
 * otherwise); q_out may not overlap qkv.  No two sequences of one
 * call may write to the same place of a page. */
mcd_status mcd_rope_append(const mcd_paged_kv* kv, int32_t layer, const mcd_chunks* chunks, int32_t n_q_heads,
                           const void* qkv, int64_t qkv_stride, int32_t qkv_dtype, void* q_out, int64_t q_stride,
                           const mcd_rope* rope, const int32_t* positions, const float* q_norm, const float* k_norm,
                           float eps, int32_t* err, void* stream);

/* Attention of the new rows (after mcd_rope_append) over `layer`: out row = softmax over the
 * visible positions of scale * q . k, times v.  Row i of a sequence sees every cached position and
 * of the sequence's new rows 0..i, or, with a mask, the rows j whose bit is set: bit j % 32 of word
 * j / 32 of its mask row (a drafted tree: its ancestors and itself).  A row that sees nothing gets
 * zeros.  What a row does not see does not touch it, whatever it holds (infinities and NaN
 * included).  What it sees counts as the formula has it: a score of -inf has weight 0; a score of +inf or
 * NaN, no score above -inf, or a value that is not finite (0 times it too) makes the row's result not finite.
 *   q, out     dev [n_rows][stride] in the cache's type, n_q_heads heads one after another, query
 *              head h reading KV head h / (n_q_heads / n_kv_heads); row strides in elements, rows
 *              16-byte aligned; out may not overlap q
 *   scale      > 0, finite
 *   mask       dev uint32 [n_rows][mask_words], mask_words >= ceil(max_rows / 32); NULL: causal
 *   workspace  dev, 16-byte aligned, at least mcd_paged_attention_workspace bytes (a function of the
 *              sizes alone; may be 0: then NULL will do); needs no initial value
 * n_q_heads is a multiple of n_kv_heads, at most 16 times as many.  Scores, softmax statistics and
 * sums are fp32; bf16 models multiply bf16 queries, keys, values and probabilities on the tensor cores: a
 * sequence with up to 16 query vectors per KV head (its rows times the heads of a group) has probabilities
 * of two bf16 terms, off by 2^-16, one with more of one term, off by 2^-8; so has every sequence of a call
 * whose n_rows has room for max_rows of each, if those are more than 16 vectors. */
mcd_status mcd_paged_attention(const mcd_paged_kv* kv, int32_t layer, const mcd_chunks* chunks, int32_t n_q_heads,
                               const void* q, int64_t q_stride, void* out, int64_t out_stride, float scale,
                               const uint32_t* mask, int32_t mask_words, void* workspace, int64_t workspace_bytes,
                               int32_t* err, void* stream);
int64_t mcd_paged_attention_workspace(const mcd_paged_kv* kv, const mcd_chunks* chunks, int32_t n_q_heads);

/* mcd_paged_attention for utterances that remember their last `window` positions and their first n_sinks ones: of what
 * a row at position p sees there (cached positions and, without a mask, new rows), it keeps the positions j with
 * p - j < window or j < n_sinks.  p is the row's slot; with a mask it is cached[s] + the number of new rows that it sees - 1
 * (a drafted tree: the depth's position; a row that sees no new row: cached[s]), and which new rows it sees the mask alone says:
 * those of a tree that is deeper than the window see ancestors from before it, as rows fed one by one would not (a row of as many
 * bits as the window is long, or fewer, sees what they would).
 * Positions from n_sinks to cached[s] - window are seen by no row: entries of the table whose pages hold nothing else are not
 * looked at and may be -1, the pages given back.  (mcd_pages_fork and mcd_pages_compact want every page of a sequence in its
 * row of the table.)
 *   window     >= 1 (one of max_tokens or more hides nothing), n_sinks >= 0: MCD_ERR_INVALID_ARG otherwise
 * All else as there, the workspace at least mcd_paged_attention_window_workspace bytes. */
mcd_status mcd_paged_attention_window(const mcd_paged_kv* kv, int32_t layer, const mcd_chunks* chunks, int32_t n_q_heads,
                                      const void* q, int64_t q_stride, void* out, int64_t out_stride, float scale,
                                      int32_t window, int32_t n_sinks, const uint32_t* mask, int32_t mask_words,
                                      void* workspace, int64_t workspace_bytes, int32_t* err, void* stream);
int64_t mcd_paged_attention_window_workspace(const mcd_paged_kv* kv, const mcd_chunks* chunks, int32_t n_q_heads,
                                             int32_t window, int32_t n_sinks);

/* n_dst new sequences from n_src old ones.  Sequence d continues parent[d] (-1: starts empty):
 *   len_out[d]    = the parent's length
 *   table_out[d]  has pages for len_out[d] + reserve[d] tokens, then -1.  Pages that the parent has filled
 *                 are shared.  The part-filled page becomes a fresh one with a copy of its tokens
 *                 (k and v, every layer), pages behind it fresh ones; but with `release` the
 *                 parent's first child (lowest d) takes over those that nobody else holds.
 *   ref_out       = ref_in, one more for every entry of table_out, with `release` one less for
 *                 every entry of table_in: the old sequences end.  A page is free while its count
 *                 is 0: ref_in has 1 at least for every page that a table names.
 * Fresh pages are the free pages of ref_in in ascending order, handed out in the order of d, then of
 * position; what this call releases is free for the next.  With parent = 0, 1, 2, .. and `release` the call
 * only makes room for `reserve` more tokens.  table_in [n_src][src_cols] holds pages for len_in[s]
 * tokens at least; `reserve` (dev int32 [n_dst]) may be NULL: none.  Outputs may not overlap
 * inputs.  When free pages run out (MCD_ERR_OOM in err) or a length, page or parent does not fit
 * (MCD_ERR_INVALID_ARG), ref_out is ref_in, and tables, lengths and pages stay as they were.
 * n_src, n_dst <= 4096 (MCD_ERR_UNSUPPORTED).  workspace: dev, 16-byte aligned, at least
 * mcd_pages_fork_workspace(n_src, n_dst, dst_cols) bytes; needs no initial value. */
mcd_status mcd_pages_fork(const mcd_paged_kv* kv, const int32_t* ref_in, int32_t* ref_out, int32_t n_src,
                          const int32_t* table_in, int32_t src_cols, const int32_t* len_in, int32_t n_dst,
                          const int32_t* parent, const int32_t* reserve, int32_t* table_out, int32_t dst_cols,
                          int32_t* len_out, int32_t release, void* workspace, int64_t workspace_bytes, int32_t* err,
                          void* stream);
int64_t mcd_pages_fork_workspace(int32_t n_src, int32_t n_dst, int32_t dst_cols);

/* For every sequence s and i < n_keep[s], all layers: the token at position start[s] + keep[s][i] of table_in
 * moves to position start[s] + i of table_out; len_out[s] (optional) = start[s] + n_keep[s].  len_out is an
 * array of its own: it may not overlap start, n_keep, keep or a table (MCD_ERR_INVALID_ARG).
 * table_out may be table_in (in place): then keep is strictly ascending in each row.  Otherwise
 * keep may have any order and name a position twice, and no page that the call writes is one that
 * it reads.  Pages that a sequence writes are its own (mcd_pages_fork leaves part-filled pages so).
 * keep: dev int32 [n_seqs][max_keep], entries >= 0.  Both tables have table_cols entries a row.  A sequence
 * whose numbers do not fit (MCD_ERR_INVALID_ARG in err) keeps its len_out, and in place its tokens; in
 * another table some of its tokens may have moved.  At most 32,767 layers and table_cols * page_size below 2^31
 * (MCD_ERR_UNSUPPORTED otherwise). */
mcd_status mcd_pages_compact(const mcd_paged_kv* kv, int32_t n_seqs, const int32_t* table_in, const int32_t* table_out,
                             int32_t table_cols, const int32_t* start, const int32_t* keep, int32_t max_keep,
                             const int32_t* n_keep, int32_t* len_out, int32_t* err, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MCD_CACHE_H */
