/*
 * sparrow_serve.h — C ABI of the operators for many requests about one long video (libsparrow_serve.so): a paged K/V cache of 8 bits
 * per element, and attention of a batch whose requests share a long prefix.
 *
 *   sparrow_mrope_append8  as sparrow_mrope_append; K and V are quantised as they are written
 *   sparrow_page_gather    tokens of a paged cache (8 bits, or the model's type) into contiguous rows, as sparrow_verify_attn reads them
 *   sparrow_chunk_attn8    as sparrow_chunk_attn, over an 8-bit cache
 *   sparrow_prefix_attn    as sparrow_chunk_attn, with a prefix that several requests share read once for all of them
 *
 * The rules of sparrow_paged.h hold, its descriptor is used; the text of the last error is sparrow_serve_last_error()'s.
 *
 * An 8-bit cache holds e4m3 numbers (OCP: 448 is the largest, no infinities, NaN 0x7f and 0xff) and, for each (token, KV head), one
 * power of two for the row of K and one for that of V:
 *     element = code * 2^(byte - 127),   byte at exponents[((page * Hkv + head) * page_size + token of the page) * 2 + (0: K, 1: V)]
 * It is written with the smallest power, 2^-100 at least, for which no finite element of the row passes 448; a code is the e4m3 number nearest
 * to the element, ties to even.  An infinite or NaN element (also one of K that its rotation takes beyond fp32) becomes NaN.  So bytes from 27 to 247 are
 * written, and a held element is a bf16 number that is read back without a rounding, or 2^128, which elements from 248 * 2^120 (3.3e38) on round to
 * and which is read back as infinite.
 * The strides of such a cache count bytes.  Contents are not trusted: a byte above 254 or below 1 is taken as the nearest of these, by the attention
 * one of V below 9 as 9.  Of powers that are not written, elements below 2^-133 are no bf16 numbers, and those from 2^128 on are infinite when read back.
 */
#ifndef SPARROW_SERVE_H
#define SPARROW_SERVE_H

#include "sparrow_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits (SPARROW_ERR_UNSUPPORTED beyond them). */
#define SPARROW_MAX_PREFIX_GROUPS 64          /* groups of one call */

/*
 * sparrow_mrope_append into an 8-bit cache.  desc->dtype is the type of q, k, v and q_out; k is rotated in 64 bits and rounded once.
 *  exponents  dev uint8 [n_pages, Hkv, page_size, 2]
 */
int sparrow_mrope_append8(const sparrow_paged_desc *desc, const void *q, const void *k, const void *v,
                          const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                          const int32_t *freq_axis, const int32_t *slots, int32_t N, void *q_out, void *k_cache,
                          void *v_cache, uint8_t *exponents, void *hip_stream);

/*
 * Tokens of the requests of a batch, read from their pages into contiguous rows: with r = cu_rows[b] + i < cu_rows[b+1]
 *     k_out[r, c] = K of token first[b] + i of request b, head c;  v_out alike
 * desc->dtype is the type of k_out and v_out; n_q_heads, scale and the row strides are not read.
 *  exponents   dev uint8 of an 8-bit cache; NULL: the cache is of desc->dtype
 *  first       dev int32 [B] or NULL (0 for all)
 *  cu_rows     dev int32 [B+1] ascending from 0; rows from cu_rows[B] on, and rows of a token that the table cannot hold, are left as they were
 *  k_out, v_out  dev, element (row r, head c, 0) at r*out_stride_row + c*out_stride_head, multiples of 16 bytes; both layouts of
 *              sparrow_attn_desc can be written
 */
int sparrow_page_gather(const sparrow_paged_desc *desc, const void *k_cache, const void *v_cache, const uint8_t *exponents,
                        const int32_t *block_table, int32_t table_width, int64_t table_stride, const int32_t *first,
                        const int32_t *cu_rows, int32_t B, int32_t n_rows, void *k_out, void *v_out,
                        int64_t out_stride_row, int64_t out_stride_head, void *hip_stream);

/*
 * sparrow_chunk_attn over an 8-bit cache: its arguments, and exponents behind the caches.  The workspace is
 * sparrow_prefix_attn_workspace()'s for n_groups = 0.
 * The output is finite where the sum of the elements that a row sees, each times its weight about the largest score (1 at most), is a number of fp32.
 */
int sparrow_chunk_attn8(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                        const uint8_t *exponents, const int32_t *block_table, int32_t table_width, int64_t table_stride,
                        const int32_t *cu_new, const int32_t *kv_len, int32_t B, int32_t n_rows, int32_t max_new,
                        void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * sparrow_chunk_attn for requests that share prefixes: requests group_start[g] .. group_start[g+1]-1 of the batch begin with the same
 * prefix_len[g] tokens, and each group's prefix is read once for the new tokens of all its requests.  out and lse are what
 * sparrow_chunk_attn gives for the same tables.
 * Where the tables of the batch hold little (B * table_width * page_size tokens of 200 MiB of K and V of all heads at most, 32 MiB for fp32; over 8 bits
 * from 80 and 16 MiB on, by the query rows of a request), a plan for groups costs more than it saves, and every request reads its own: n_groups changes nothing
 * then.
 *
 *  exponents    dev uint8 of an 8-bit cache; NULL: the cache is of desc->dtype (the weights then reach 2^8, as in sparrow_chunk_attn: elements of V above
 *               2^119 can pass fp32 in a product or a sum, the output is infinite or NaN then)
 *  block_table  every request's row holds its whole context.  The prefix is read through the row of the group's first request that has new
 *               tokens; the tokens behind it through each request's own.  Whole pages of a prefix are usually the same pages in all rows.
 *  group_start  dev int32 [n_groups+1] ascending, from 0 to B; requests outside all groups share nothing.  NULL where n_groups = 0
 *  prefix_len   dev int32 [n_groups].  What is shared is cut to the tokens that come before the new ones of every request of the group (0 where
 *               one has no such tokens): the result does not change, the keys behind the cut are read request by request
 * Limits: as sparrow_chunk_attn, n_groups <= SPARROW_MAX_PREFIX_GROUPS.
 * The workspace is asked for as for the widest tables, with the groups and without, whatever the call's tables hold; a piece's part of it is for a whole block
 * of rows (16, 64 or 256).  28 and 4 heads of 128, a group of 32 single tokens: 136 MB, of 256 209 MB; 32 heads of each, 256 requests: 1.2 GB.
 */
size_t sparrow_prefix_attn_workspace(const sparrow_paged_desc *desc, int32_t B, int32_t n_groups, int32_t n_rows, int32_t max_new);
int sparrow_prefix_attn(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                        const uint8_t *exponents, const int32_t *block_table, int32_t table_width, int64_t table_stride,
                        const int32_t *cu_new, const int32_t *kv_len, int32_t B, const int32_t *group_start,
                        const int32_t *prefix_len, int32_t n_groups, int32_t n_rows, int32_t max_new, void *out, float *lse,
                        void *workspace, size_t workspace_bytes, void *hip_stream);

/* Thread-local description of the last error of this library on this thread; "" if none. */
const char *sparrow_serve_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SPARROW_SERVE_H */
