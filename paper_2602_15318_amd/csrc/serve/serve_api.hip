// Host side of the C ABI declared in include/sparrow_serve.h: argument validation and launches.  No device allocation, no
// synchronisation, no device reads.
#include <algorithm>
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "serve.hpp"

namespace sparrow {
namespace {
thread_local char g_err[512] = "";

int fail(int code, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
int shift_of(int32_t power) { return 31 - __builtin_clz((unsigned)power); }
int64_t per_16_bytes(int32_t dtype) { return dtype == SPARROW_BF16 ? 8 : 4; }

int check_table(int32_t B, int32_t page_size, int32_t table_width, int64_t table_stride) {
  if (B > SPARROW_MAX_PAGED_BATCH) return fail(SPARROW_ERR_UNSUPPORTED, "B = %d exceeds %d sequences", B, SPARROW_MAX_PAGED_BATCH);
  if (table_width <= 0 || table_stride < table_width || table_stride > 1ll << 40)
    return fail(SPARROW_ERR_INVALID_ARG, "table_width %d (at least 1), table_stride %lld (table_width to 2^40)", table_width, (long long)table_stride);
  if ((int64_t)table_width * page_size > SPARROW_MAX_PAGED_TOKENS)
    return fail(SPARROW_ERR_UNSUPPORTED, "table_width %d of pages of %d: more than %d tokens", table_width, page_size, SPARROW_MAX_PAGED_TOKENS);
  return SPARROW_OK;
}

// A cache of `eight` bits or of desc->dtype.  Query heads and scale are the attention's.
int check_desc(const sparrow_paged_desc *d, bool eight, bool queries) {
  if (!d) return fail(SPARROW_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != SPARROW_F32 && d->dtype != SPARROW_BF16)
    return fail(SPARROW_ERR_UNSUPPORTED, "dtype %d is neither SPARROW_F32 nor SPARROW_BF16", d->dtype);
  if (d->n_kv_heads <= 0 || (queries && (d->n_q_heads <= 0 || d->n_q_heads % d->n_kv_heads != 0)))
    return fail(SPARROW_ERR_INVALID_ARG, "n_q_heads %d must be a positive multiple of n_kv_heads %d", d->n_q_heads, d->n_kv_heads);
  if (d->n_kv_heads > 1 << 15 || (queries && d->n_q_heads > 1 << 15))
    return fail(SPARROW_ERR_UNSUPPORTED, "%d query and %d KV heads (up to %d)", d->n_q_heads, d->n_kv_heads, 1 << 15);
  if (d->head_dim != 64 && d->head_dim != 128) return fail(SPARROW_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
  if (d->page_size < 16 || d->page_size > 4096 || (d->page_size & (d->page_size - 1)) != 0)
    return fail(SPARROW_ERR_UNSUPPORTED, "page_size %d (a power of two from 16 to 4096)", d->page_size);
  if (d->n_pages <= 0) return fail(SPARROW_ERR_INVALID_ARG, "n_pages %d must be positive", d->n_pages);
  if ((int64_t)d->n_pages * d->page_size >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "%d pages of %d tokens: slots pass 31 bits", d->n_pages, d->page_size);
  const int64_t per = eight ? 16 : per_16_bytes(d->dtype), es = 16 / per;
  const int64_t st[3] = {d->kv_stride_page, d->kv_stride_token, d->kv_stride_head};
  for (int64_t s : st)
    if (s < d->head_dim || s % per != 0 || s > 1ll << 40)
      return fail(SPARROW_ERR_INVALID_ARG, "kv strides (page %lld, token %lld, head %lld) must be multiples of 16 bytes from "
                  "head_dim to 2^40 elements", (long long)st[0], (long long)st[1], (long long)st[2]);
  if ((int64_t)d->page_size * d->kv_stride_token * es >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "page_size * kv_stride_token: tokens of a page more than 2^31 bytes apart");
  if (queries && (!(d->scale >= 0.f) || std::isinf(d->scale * kLog2e)))      // (scores are kept in base 2)
    return fail(SPARROW_ERR_INVALID_ARG, "scale must be >= 0 (0 = 1/sqrt(head_dim)), and finite in base 2: up to 2.3e38");
  return SPARROW_OK;
}

int check_rows(const char *what, int64_t stride, int64_t least, int32_t dtype) {
  if (stride < least || stride % per_16_bytes(dtype) != 0 || stride > 1ll << 36)
    return fail(SPARROW_ERR_INVALID_ARG, "%s %lld must be a multiple of 16 bytes from %lld to 2^36 elements", what, (long long)stride, (long long)least);
  return SPARROW_OK;
}

int frequencies(const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq, const int32_t *freq_axis,
                int32_t d, Frequencies *f) {
  if (!positions || !inv_freq || !freq_axis) return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among positions/inv_freq/freq_axis");
  if (!aligned(positions, 4)) return fail(SPARROW_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  if (n_axes < 1 || n_axes > 4) return fail(SPARROW_ERR_UNSUPPORTED, "n_axes %d (1 to 4)", n_axes);
  if (axis_stride < 0) return fail(SPARROW_ERR_INVALID_ARG, "axis_stride %lld is negative", (long long)axis_stride);
  *f = Frequencies{};
  for (int i = 0; i < d / 2; ++i) {
    if (!std::isfinite(inv_freq[i])) return fail(SPARROW_ERR_INVALID_ARG, "inv_freq[%d] is not finite", i);
    if (freq_axis[i] < 0 || freq_axis[i] >= n_axes)
      return fail(SPARROW_ERR_INVALID_ARG, "freq_axis[%d] = %d is not one of %d axes", i, freq_axis[i], n_axes);
    f->quarter[i] = inv_freq[i] * 0.63661977236758134308;  // 2 / pi
    f->axis[i] = (uint8_t)freq_axis[i];
  }
  return SPARROW_OK;
}

// sizes that the attention refuses have no workspace
bool attention_sizes(const sparrow_paged_desc *d, int32_t B, int32_t n_groups, int32_t n_rows, int32_t max_new) {
  return d && (d->dtype == SPARROW_F32 || d->dtype == SPARROW_BF16) && (d->head_dim == 64 || d->head_dim == 128) && d->n_q_heads > 0 &&
         d->n_q_heads <= 1 << 15 && d->n_kv_heads > 0 && d->n_q_heads % d->n_kv_heads == 0 && B > 0 && B <= SPARROW_MAX_PAGED_BATCH &&
         n_groups >= 0 && n_groups <= SPARROW_MAX_PREFIX_GROUPS && n_rows > 0 && n_rows <= SPARROW_MAX_PAGED_TOKENS &&
         (int64_t)n_rows * d->n_q_heads < 1ll << 31 && max_new > 0;
}

size_t workspace_of(const ServeShape &s, int32_t B, int32_t G) {
  return s.slots == 0 ? 0 : round_up((size_t)s.floats_o * 4, 256) + round_up((size_t)s.floats_ml * 4, 256) + round_up((size_t)B * 32, 256) +
                                (G == 0 ? 0 : 256 + round_up((size_t)s.slots * 48, 256));
}

int attention(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache, const uint8_t *exponents,
              const int32_t *block_table, int32_t table_width, int64_t table_stride, const int32_t *cu_new, const int32_t *kv_len,
              int32_t B, const int32_t *group_start, const int32_t *prefix_len, int32_t n_groups, int32_t n_rows, int32_t max_new,
              void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_desc(desc, exponents != nullptr, true)) return rc;
  if (B < 0 || n_rows < 0 || max_new < 0 || n_groups < 0)
    return fail(SPARROW_ERR_INVALID_ARG, "B = %d, n_groups = %d, n_rows = %d, max_new = %d", B, n_groups, n_rows, max_new);
  if (B == 0 || n_rows == 0 || max_new == 0) return SPARROW_OK;
  if (int rc = check_table(B, desc->page_size, table_width, table_stride)) return rc;
  if (int rc = check_rows("q_stride_row", desc->q_stride_row, (int64_t)desc->n_q_heads * desc->head_dim, desc->dtype)) return rc;
  if (n_groups > SPARROW_MAX_PREFIX_GROUPS)
    return fail(SPARROW_ERR_UNSUPPORTED, "n_groups = %d exceeds %d", n_groups, SPARROW_MAX_PREFIX_GROUPS);
  if (n_rows > SPARROW_MAX_PAGED_TOKENS)
    return fail(SPARROW_ERR_UNSUPPORTED, "n_rows = %d exceeds %d", n_rows, SPARROW_MAX_PAGED_TOKENS);
  if ((int64_t)n_rows * desc->n_q_heads >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "%d rows of %d heads (less than 2^31)", n_rows, desc->n_q_heads);
  if (!q || !k_cache || !v_cache || !block_table || !cu_new || !kv_len || !out || (n_groups > 0 && (!group_start || !prefix_len)))
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among q/k_cache/v_cache/block_table/cu_new/kv_len/group_start/prefix_len/out");
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) || !aligned(exponents, 16) ||
      !aligned(block_table, 4) || !aligned(cu_new, 4) || !aligned(kv_len, 4) || !aligned(lse, 4) || !aligned(group_start, 4) || !aligned(prefix_len, 4))
    return fail(SPARROW_ERR_INVALID_ARG, "q, the caches, the exponents and out must be 16-byte aligned, the other arrays 4-byte");
  const size_t need = sparrow_prefix_attn_workspace(desc, B, n_groups, n_rows, max_new);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(SPARROW_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
  if (need > 0 && !aligned(workspace, 256)) return fail(SPARROW_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  ServeArgs a;
  a.q = q; a.k = k_cache; a.v = v_cache; a.exponents = exponents;
  a.block_table = block_table; a.cu_new = cu_new; a.kv_len = kv_len; a.group_start = group_start; a.prefix_len = prefix_len;
  a.out = out; a.lse = lse;
  a.table_stride = table_stride; a.q_row = desc->q_stride_row;
  a.stride_page = desc->kv_stride_page; a.stride_token = desc->kv_stride_token; a.stride_head = desc->kv_stride_head;
  a.B = B; a.n_rows = n_rows; a.max_new = max_new; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads;
  a.g = desc->n_q_heads / desc->n_kv_heads;
  a.table_width = table_width; a.page_shift = shift_of(desc->page_size); a.n_pages = desc->n_pages;
  a.scale_log2 = (desc->scale > 0.f ? desc->scale : 1.0f / std::sqrt((float)desc->head_dim)) * kLog2e;
  a.inv_g = 1.0f / (float)a.g;
  const int64_t capacity = (int64_t)table_width * desc->page_size;
  a.G = serve_shares(desc->dtype, exponents != nullptr, desc->head_dim, a.Hkv, B, capacity, (int64_t)std::min(max_new, n_rows) * a.g) ? n_groups : 0;
  a.once = n_groups == 0 || a.G > 0;
  const ServeShape shape = serve_shape(desc->dtype, desc->head_dim, a.Hq, a.Hkv, B, a.G, n_rows, max_new, capacity);
  a.slots = shape.slots; a.round = shape.round; a.ways = shape.ways; a.block_shift = shift_of(shape.rows);
  a.part_o = (float *)workspace;
  a.part_ml = (float *)((unsigned char *)workspace + round_up((size_t)shape.floats_o * 4, 256));
  a.left = shape.slots == 0 ? nullptr : (ServeLeft *)((unsigned char *)a.part_ml + round_up((size_t)shape.floats_ml * 4, 256));
  a.n_pieces = a.G == 0 ? nullptr : (int32_t *)((unsigned char *)a.left + round_up((size_t)B * 32, 256));
  a.pieces = a.G == 0 ? nullptr : (ServePiece *)((unsigned char *)a.n_pieces + 256);
  const hipError_t e = launch_serve_attn(desc->dtype, desc->head_dim, shape, a, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "attention launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

}  // namespace
}  // namespace sparrow

using namespace sparrow;

extern "C" {

const char *sparrow_serve_last_error(void) { return g_err; }

int sparrow_mrope_append8(const sparrow_paged_desc *desc, const void *q, const void *k, const void *v,
                          const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                          const int32_t *freq_axis, const int32_t *slots, int32_t N, void *q_out, void *k_cache,
                          void *v_cache, uint8_t *exponents, void *hip_stream) {
  g_err[0] = 0;
  if (int rc = check_desc(desc, true, true)) return rc;
  if (N < 0) return fail(SPARROW_ERR_INVALID_ARG, "N = %d", N);
  if (N == 0) return SPARROW_OK;
  if (N >= 1 << 24) return fail(SPARROW_ERR_UNSUPPORTED, "N = %d (less than 2^24)", N);
  if (int rc = check_rows("q_stride_row", desc->q_stride_row, (int64_t)desc->n_q_heads * desc->head_dim, desc->dtype)) return rc;
  if (int rc = check_rows("kv_stride_row", desc->kv_stride_row, (int64_t)desc->n_kv_heads * desc->head_dim, desc->dtype)) return rc;
  if (!q || !k || !v || !slots || !q_out || !k_cache || !v_cache || !exponents)
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among q/k/v/slots/q_out/k_cache/v_cache/exponents");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) ||
      !aligned(exponents, 16) || !aligned(slots, 4))
    return fail(SPARROW_ERR_INVALID_ARG, "q, k, v, q_out, the caches and the exponents must be 16-byte aligned, slots 4-byte");
  if (q_out == q && desc->q_stride_row != (int64_t)desc->n_q_heads * desc->head_dim)
    return fail(SPARROW_ERR_INVALID_ARG, "q_out may be q only where q's rows are contiguous");
  Frequencies f;
  if (int rc = frequencies(positions, axis_stride, n_axes, inv_freq, freq_axis, desc->head_dim, &f)) return rc;
  Append8Args a;
  a.q = q; a.k = k; a.v = v; a.positions = positions; a.slots = slots;
  a.q_out = q_out; a.k_cache = (e4m3_t *)k_cache; a.v_cache = (e4m3_t *)v_cache; a.exponents = exponents;
  a.axis_stride = axis_stride; a.q_row = desc->q_stride_row; a.kv_row = desc->kv_stride_row;
  a.stride_page = desc->kv_stride_page; a.stride_token = desc->kv_stride_token; a.stride_head = desc->kv_stride_head;
  a.N = N; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads;
  a.page_shift = shift_of(desc->page_size); a.n_slots = desc->n_pages * desc->page_size;
  const hipError_t e = launch_mrope_append8(desc->dtype, a, f, desc->head_dim, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "mrope_append8 launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

int sparrow_page_gather(const sparrow_paged_desc *desc, const void *k_cache, const void *v_cache, const uint8_t *exponents,
                        const int32_t *block_table, int32_t table_width, int64_t table_stride, const int32_t *first,
                        const int32_t *cu_rows, int32_t B, int32_t n_rows, void *k_out, void *v_out,
                        int64_t out_stride_row, int64_t out_stride_head, void *hip_stream) {
  g_err[0] = 0;
  if (int rc = check_desc(desc, exponents != nullptr, false)) return rc;
  if (B < 0 || n_rows < 0) return fail(SPARROW_ERR_INVALID_ARG, "B = %d, n_rows = %d", B, n_rows);
  if (B == 0 || n_rows == 0) return SPARROW_OK;
  if (int rc = check_table(B, desc->page_size, table_width, table_stride)) return rc;
  if (n_rows >= 1 << 30) return fail(SPARROW_ERR_UNSUPPORTED, "n_rows = %d (less than 2^30)", n_rows);
  if (int rc = check_rows("out_stride_row", out_stride_row, desc->head_dim, desc->dtype)) return rc;
  if (int rc = check_rows("out_stride_head", out_stride_head, desc->head_dim, desc->dtype)) return rc;
  if (!k_cache || !v_cache || !block_table || !cu_rows || !k_out || !v_out)
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among k_cache/v_cache/block_table/cu_rows/k_out/v_out");
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(exponents, 16) || !aligned(k_out, 16) || !aligned(v_out, 16) ||
      !aligned(block_table, 4) || !aligned(first, 4) || !aligned(cu_rows, 4))
    return fail(SPARROW_ERR_INVALID_ARG, "the caches, the exponents, k_out and v_out must be 16-byte aligned, the other arrays 4-byte");
  GatherArgs a;
  a.k = k_cache; a.v = v_cache; a.exponents = exponents; a.block_table = block_table; a.first = first; a.cu_rows = cu_rows;
  a.k_out = k_out; a.v_out = v_out;
  a.table_stride = table_stride; a.stride_page = desc->kv_stride_page; a.stride_token = desc->kv_stride_token; a.stride_head = desc->kv_stride_head;
  a.out_row = out_stride_row; a.out_head = out_stride_head;
  a.B = B; a.n_rows = n_rows; a.Hkv = desc->n_kv_heads; a.table_width = table_width; a.page_shift = shift_of(desc->page_size); a.n_pages = desc->n_pages;
  const hipError_t e = launch_page_gather(desc->dtype, desc->head_dim, a, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "page_gather launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

size_t sparrow_prefix_attn_workspace(const sparrow_paged_desc *desc, int32_t B, int32_t n_groups, int32_t n_rows, int32_t max_new) {
  if (!attention_sizes(desc, B, n_groups, n_rows, max_new)) return 0;
  size_t most = 0;                         // with the groups and without: which it will be depends on the tables
  for (const int32_t G : {0, n_groups})
    most = std::max(most, workspace_of(serve_shape(desc->dtype, desc->head_dim, desc->n_q_heads, desc->n_kv_heads, B, G, n_rows, max_new,
                                                   SPARROW_MAX_PAGED_TOKENS), B, G));
  return most;
}

int sparrow_chunk_attn8(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                        const uint8_t *exponents, const int32_t *block_table, int32_t table_width, int64_t table_stride,
                        const int32_t *cu_new, const int32_t *kv_len, int32_t B, int32_t n_rows, int32_t max_new,
                        void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  g_err[0] = 0;
  if (!exponents) return fail(SPARROW_ERR_INVALID_ARG, "exponents is NULL");
  return attention(desc, q, k_cache, v_cache, exponents, block_table, table_width, table_stride, cu_new, kv_len, B, nullptr, nullptr, 0, n_rows,
                   max_new, out, lse, workspace, workspace_bytes, hip_stream);
}

int sparrow_prefix_attn(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                        const uint8_t *exponents, const int32_t *block_table, int32_t table_width, int64_t table_stride,
                        const int32_t *cu_new, const int32_t *kv_len, int32_t B, const int32_t *group_start,
                        const int32_t *prefix_len, int32_t n_groups, int32_t n_rows, int32_t max_new, void *out, float *lse,
                        void *workspace, size_t workspace_bytes, void *hip_stream) {
  g_err[0] = 0;
  return attention(desc, q, k_cache, v_cache, exponents, block_table, table_width, table_stride, cu_new, kv_len, B, group_start, prefix_len,
                   n_groups, n_rows, max_new, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
