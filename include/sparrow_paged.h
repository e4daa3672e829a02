/*
 * sparrow_paged.h — C ABI of the paged-cache operators (libsparrow_paged.so): what a target model's forward pass
 * needs around its projections when the K/V cache of its requests lives on pages.
 *
 *   sparrow_page_update   block tables and slot maps from request lengths, on the GPU
 *   sparrow_mrope_table   cos/sin rows of positions with several axes (sparrow_draft_qkv_append reads them)
 *   sparrow_mrope_append  the same rotation of a chunk's q and k; K and V appended to the paged cache
 *   sparrow_chunk_attn    attention of the new tokens of a batch over the paged cache
 *
 * The common rules of sparrow.h hold (ownership, asynchrony, errors, types, alignment, grouping of heads), with two
 * differences: lengths, offsets and tables are device arrays that the kernels read when they run, so that a captured
 * call replays with other lengths; and the text of the last error is sparrow_paged_last_error()'s.
 *
 * Device arrays are not trusted: a length is clamped to what the block table of its request can hold, a page id to the
 * cache's pages, a row to the call's rows.  Contents that break a precondition give undefined results, never an access
 * outside the buffers as described by the arguments.
 */
#ifndef SPARROW_PAGED_H
#define SPARROW_PAGED_H

#include "sparrow.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (SPARROW_ERR_UNSUPPORTED beyond them). */
#define SPARROW_MAX_PAGED_BATCH 256           /* sequences per call */
#define SPARROW_MAX_PAGED_TOKENS (1 << 22)    /* tokens that one block table can hold: table_width * page_size */

typedef struct {
  int32_t dtype;        /* sparrow_dtype of q, k, v, the caches and out */
  int32_t n_q_heads;    /* Hq */
  int32_t n_kv_heads;   /* Hkv, divides Hq */
  int32_t head_dim;     /* d: 64 or 128 */
  float scale;          /* softmax scale; 0 selects 1/sqrt(head_dim); up to 2.3e38; read by sparrow_chunk_attn only */
  int32_t page_size;    /* tokens per page: a power of two from 16 to 4096 */
  int32_t n_pages;      /* pages of the cache; n_pages * page_size < 2^31 */
  /* Element (page p, token t of it, head c, 0) of a cache, K and V alike: p*kv_stride_page + t*kv_stride_token +
   * c*kv_stride_head, all multiples of 16 bytes; the d elements of a head's row are contiguous.  page_size *
   * kv_stride_token elements are less than 2^31 bytes. */
  int64_t kv_stride_page;
  int64_t kv_stride_token;
  int64_t kv_stride_head;
  /* Elements between the rows of q (of k and v in sparrow_mrope_append: kv_stride_row), multiples of 16 bytes; a row's
   * heads are contiguous.  Rows of a fused QKV product are Hq*d + 2*Hkv*d apart. */
  int64_t q_stride_row;
  int64_t kv_stride_row;
} sparrow_paged_desc;

/*
 * Block tables and slot maps.  A request of length n holds the first ceil(n / page_size) entries of its row of
 * block_table.  The call takes every request from old_len[b] to new_len[b] tokens: one that grows takes pages from the
 * stack of free pages, one that shrinks (draft tokens rejected, request finished: new_len 0) gives its surplus back.
 *   given back:  the k-th page, k counting over (b, entry) in ascending order, goes to free_pages[n_free + R - 1 - k]
 *   taken:       the k-th page is free_pages[n_free + R - 1 - k]
 * with R the pages given back in the call, before any is taken; n_free becomes n_free + R - (pages taken).  A call from
 * new_len to old_len therefore undoes one that only grew, stack included.  Entries behind a request's pages are left as they were.
 * The tokens that came are numbered through the batch: rows cu_new[b] .. cu_new[b+1]-1 are those of request b, and
 *   slots[cu_new[b] + i]     = block_table[b][(old_len[b] + i) / page_size] * page_size + (old_len[b] + i) % page_size
 *   positions[cu_new[b] + i] = old_len[b] + i + (pos_offset ? pos_offset[b] : 0)
 * Rows behind the last request get slot -1 and position 0.
 *
 *  old_len, new_len  dev int32 [B], in [0, table_width * page_size]
 *  block_table dev int32 [B, table_stride], in/out, table_width <= table_stride entries a row in use
 *  free_pages  dev int32 [capacity], in/out; n_free dev int32 [1], in/out: entries 0 .. n_free-1 are the stack
 *  n_rows      rows of slots and positions
 *  slots, positions  dev int32 out [n_rows]; positions may be NULL (both, where n_rows = 0)
 *  cu_new      dev int32 out [B+1]
 *  status      dev int32 out [1]: 0; p > 0: p pages are missing; -1: more new tokens than n_rows; -2: a length out of
 *              range; -3: n_free out of range, or more pages given back than capacity holds.  With a status other than 0
 *              nothing is taken or given back, cu_new is all 0 and every slot -1: what follows in the stream has no rows.
 *  The ids are copied as they are.  Two entries of the batch must not hold the same page.
 *  B = 0: nothing is enqueued, the outputs stay as they were (slots of a step before would be written to again: the binding clears them).
 */
int sparrow_page_update(const int32_t *old_len, const int32_t *new_len, int32_t B, int32_t page_size,
                        int32_t *block_table, int32_t table_width, int64_t table_stride, int32_t *free_pages,
                        int32_t capacity, int32_t *n_free, const int32_t *pos_offset, int32_t n_rows, int32_t *slots,
                        int32_t *positions, int32_t *cu_new, int32_t *status, void *hip_stream);

/*
 * Rotary tables of positions with several axes (time, height, width of a video's tokens; equal on text):
 *     cos[n][i], sin[n][i] = cos, sin of positions[freq_axis[i]][n] * inv_freq[i]        (i < d/2)
 * The angle is worked out and reduced in 64 bits, so that far positions cost nothing.
 *  positions  dev int32: axis a, token n at positions[a * axis_stride + n]; axis_stride 0 serves one axis as all
 *  n_axes     1 to 4
 *  inv_freq   host double [d/2], finite;  freq_axis  host int32 [d/2], in [0, n_axes)
 *  cos, sin   dev float out [N, d/2]
 *  d          64 or 128
 */
int sparrow_mrope_table(const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                        const int32_t *freq_axis, int32_t d, int32_t N, float *cos, float *sin, void *hip_stream);

/*
 * Rotation of a chunk's q and k rows by those angles (rotate-half, as sparrow_draft_qkv_append) and the append to the cache:
 *     q_out[n, h] = rot(q[n, h]);  k_cache[slots[n], c] = rot(k[n, c]);  v_cache[slots[n], c] = v[n, c]
 *  q          dev, row n at n*q_stride_row;  k, v dev, row n at n*kv_stride_row
 *  slots      dev int32 [N] (page * page_size + token of it, as sparrow_page_update writes them), all distinct; a row whose
 *             slot lies outside the cache (-1) is skipped: its row of q_out is left as it was too
 *  q_out      dev out [N, Hq, d] contiguous; may be q itself where q's rows are contiguous
 *  N < 2^24
 */
int sparrow_mrope_append(const sparrow_paged_desc *desc, const void *q, const void *k, const void *v,
                         const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                         const int32_t *freq_axis, const int32_t *slots, int32_t N, void *q_out, void *k_cache,
                         void *v_cache, void *hip_stream);

/*
 * Attention of the new tokens of a batch over its paged cache, which holds their K and V already: request b has
 * kv_len[b] tokens in the cache, the last cu_new[b+1] - cu_new[b] of them new.  New token i sits at position
 * p = kv_len[b] - n_new + i and sees the keys 0 .. p:
 *     out[row, h] = softmax(scale * q[row, h] . K[0..p]^T) V[0..p];  lse natural-log sum-exp of the scaled scores
 * A token at a position below 0 (n_new > kv_len: a padded request) sees nothing: out 0, lse -inf.
 *
 *  q            dev, row r at r*q_stride_row, [n_rows, Hq, d]
 *  block_table  dev int32 [B, table_stride], table_width entries a row in use; entry j holds tokens j*page_size ..
 *  cu_new       dev int32 [B+1] ascending from 0; rows from cu_new[B] on are left as they were in out and lse
 *  kv_len       dev int32 [B]
 *  max_new      no request has more new tokens than this (later rows of one that has are not computed)
 *  out          dev [n_rows, Hq, d];  lse dev float [n_rows, Hq] or NULL
 *  workspace    dev, 256-byte aligned, at least sparrow_chunk_attn_workspace() bytes; calls that may run at the same time
 *               need one each
 *  Limits: B <= SPARROW_MAX_PAGED_BATCH, table_width * page_size and n_rows <= SPARROW_MAX_PAGED_TOKENS, n_rows * Hq < 2^31.
 *  Scores, weights' sums and partial results are fp32; in bf16 a weight is rounded once, for its product with V (row sums take it unrounded), and
 *  the output once.
 *  Values and keys that a row does not see do not reach it, infinities and NaN included.
 *  Scores may be as large as fp32 holds them, unscaled and scaled: among scores whose distances pass what fp32 resolves, the largest takes all.
 *  B = 0, n_rows = 0 or max_new = 0: nothing is enqueued.  The workspace of sizes that the call refuses is 0 bytes.
 */
size_t sparrow_chunk_attn_workspace(const sparrow_paged_desc *desc, int32_t B, int32_t n_rows, int32_t max_new);
int sparrow_chunk_attn(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                       const int32_t *block_table, int32_t table_width, int64_t table_stride, const int32_t *cu_new,
                       const int32_t *kv_len, int32_t B, int32_t n_rows, int32_t max_new, void *out, float *lse,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/* Thread-local description of the last error of this library on this thread; "" if none. */
const char *sparrow_paged_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SPARROW_PAGED_H */
