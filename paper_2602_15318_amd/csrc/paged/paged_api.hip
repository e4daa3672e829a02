// Host side of the C ABI declared in include/sparrow_paged.h: argument validation and launches.  No device allocation, no
// synchronisation, no device reads.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "paged.hpp"

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

int shift_of(int32_t page_size) { return 31 - __builtin_clz((unsigned)page_size); }

int check_page_size(int32_t page_size) {
  if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)) != 0)
    return fail(SPARROW_ERR_UNSUPPORTED, "page_size %d (a power of two from 16 to 4096)", page_size);
  return SPARROW_OK;
}

int check_table(int32_t B, int32_t page_size, int32_t table_width, int64_t table_stride) {
  if (B > SPARROW_MAX_PAGED_BATCH) return fail(SPARROW_ERR_UNSUPPORTED, "B = %d exceeds %d sequences", B, SPARROW_MAX_PAGED_BATCH);
  if (table_width <= 0 || table_stride < table_width)
    return fail(SPARROW_ERR_INVALID_ARG, "table_width %d (at least 1), table_stride %lld (at least table_width)", table_width,
                (long long)table_stride);
  if ((int64_t)table_width * page_size > SPARROW_MAX_PAGED_TOKENS)
    return fail(SPARROW_ERR_UNSUPPORTED, "table_width %d of pages of %d: more than %d tokens", table_width, page_size,
                SPARROW_MAX_PAGED_TOKENS);
  return SPARROW_OK;
}

int check_desc(const sparrow_paged_desc *d) {
  if (!d) return fail(SPARROW_ERR_INVALID_ARG, "desc is NULL");
  if (d->dtype != SPARROW_F32 && d->dtype != SPARROW_BF16)
    return fail(SPARROW_ERR_UNSUPPORTED, "dtype %d is neither SPARROW_F32 nor SPARROW_BF16", d->dtype);
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->n_q_heads % d->n_kv_heads != 0)
    return fail(SPARROW_ERR_INVALID_ARG, "n_q_heads %d must be a positive multiple of n_kv_heads %d", d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads > 1 << 15) return fail(SPARROW_ERR_UNSUPPORTED, "n_q_heads %d exceeds %d", d->n_q_heads, 1 << 15);
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(SPARROW_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->head_dim);
  if (int rc = check_page_size(d->page_size)) return rc;
  if (d->n_pages <= 0) return fail(SPARROW_ERR_INVALID_ARG, "n_pages %d must be positive", d->n_pages);
  if ((int64_t)d->n_pages * d->page_size >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "%d pages of %d tokens: slots pass 31 bits", d->n_pages, d->page_size);
  const int64_t per = d->dtype == SPARROW_BF16 ? 8 : 4, es = 16 / per;
  const int64_t st[3] = {d->kv_stride_page, d->kv_stride_token, d->kv_stride_head};
  for (int64_t s : st)
    if (s < d->head_dim || s % per != 0 || s > 1ll << 40)
      return fail(SPARROW_ERR_INVALID_ARG, "kv strides (page %lld, token %lld, head %lld) must be multiples of 16 bytes from "
                  "head_dim to 2^40 elements", (long long)st[0], (long long)st[1], (long long)st[2]);
  if ((int64_t)d->page_size * d->kv_stride_token * es >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "page_size * kv_stride_token: tokens of a page more than 2^31 bytes apart");
  if (!(d->scale >= 0.f) || std::isinf(d->scale * kLog2e))      // (scores are kept in base 2)
    return fail(SPARROW_ERR_INVALID_ARG, "scale must be >= 0 (0 = 1/sqrt(head_dim)), and finite in base 2: up to 2.3e38");
  return SPARROW_OK;
}

int check_rows(const char *what, int64_t stride, int64_t heads, const sparrow_paged_desc *d) {
  const int64_t per = d->dtype == SPARROW_BF16 ? 8 : 4;
  if (stride < heads * d->head_dim || stride % per != 0 || stride > 1ll << 36)
    return fail(SPARROW_ERR_INVALID_ARG, "%s %lld must be a multiple of 16 bytes and hold %lld heads of %d", what, (long long)stride,
                (long long)heads, d->head_dim);
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

}  // namespace
}  // namespace sparrow

using namespace sparrow;

extern "C" {

const char *sparrow_paged_last_error(void) { return g_err; }

int sparrow_page_update(const int32_t *old_len, const int32_t *new_len, int32_t B, int32_t page_size,
                        int32_t *block_table, int32_t table_width, int64_t table_stride, int32_t *free_pages,
                        int32_t capacity, int32_t *n_free, const int32_t *pos_offset, int32_t n_rows, int32_t *slots,
                        int32_t *positions, int32_t *cu_new, int32_t *status, void *hip_stream) {
  g_err[0] = 0;
  if (B < 0 || n_rows < 0 || capacity < 0)
    return fail(SPARROW_ERR_INVALID_ARG, "B = %d, n_rows = %d, capacity = %d", B, n_rows, capacity);
  if (int rc = check_page_size(page_size)) return rc;
  if (B == 0) return SPARROW_OK;
  if (int rc = check_table(B, page_size, table_width, table_stride)) return rc;
  if (!old_len || !new_len || !block_table || !n_free || !cu_new || !status || (capacity > 0 && !free_pages) ||
      (n_rows > 0 && !slots))
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among old_len/new_len/block_table/free_pages/n_free/slots/cu_new/status");
  const void *all[] = {old_len, new_len, block_table, free_pages, n_free, pos_offset, slots, positions, cu_new, status};
  for (const void *p : all)
    if (!aligned(p, 4)) return fail(SPARROW_ERR_INVALID_ARG, "the arrays must be 4-byte aligned");
  PageUpdateArgs a;
  a.old_len = old_len; a.new_len = new_len; a.pos_offset = pos_offset;
  a.block_table = block_table; a.free_pages = free_pages; a.n_free = n_free;
  a.slots = slots; a.positions = positions; a.cu_new = cu_new; a.status = status;
  a.table_stride = table_stride;
  a.B = B; a.page_shift = shift_of(page_size); a.table_width = table_width; a.capacity = capacity; a.n_rows = n_rows;
  const hipError_t e = launch_page_update(a, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "page_update launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

int sparrow_mrope_table(const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                        const int32_t *freq_axis, int32_t d, int32_t N, float *cos, float *sin, void *hip_stream) {
  g_err[0] = 0;
  if (N < 0) return fail(SPARROW_ERR_INVALID_ARG, "N = %d", N);
  if (d != 64 && d != 128) return fail(SPARROW_ERR_UNSUPPORTED, "d = %d (supported: 64, 128)", d);
  if (N == 0) return SPARROW_OK;
  if (N >= 1 << 24) return fail(SPARROW_ERR_UNSUPPORTED, "N = %d (less than 2^24)", N);
  if (!cos || !sin || !aligned(cos, 16) || !aligned(sin, 16))
    return fail(SPARROW_ERR_INVALID_ARG, "cos and sin must be 16-byte aligned device arrays");
  Frequencies f;
  if (int rc = frequencies(positions, axis_stride, n_axes, inv_freq, freq_axis, d, &f)) return rc;
  RopeTableArgs a;
  a.positions = positions; a.axis_stride = axis_stride; a.cos = cos; a.sin = sin; a.N = N;
  const hipError_t e = launch_mrope_table(a, f, d, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "mrope_table launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

int sparrow_mrope_append(const sparrow_paged_desc *desc, const void *q, const void *k, const void *v,
                         const int32_t *positions, int64_t axis_stride, int32_t n_axes, const double *inv_freq,
                         const int32_t *freq_axis, const int32_t *slots, int32_t N, void *q_out, void *k_cache,
                         void *v_cache, void *hip_stream) {
  g_err[0] = 0;
  if (int rc = check_desc(desc)) return rc;
  if (N < 0) return fail(SPARROW_ERR_INVALID_ARG, "N = %d", N);
  if (N == 0) return SPARROW_OK;
  if (N >= 1 << 24) return fail(SPARROW_ERR_UNSUPPORTED, "N = %d (less than 2^24)", N);
  if (int rc = check_rows("q_stride_row", desc->q_stride_row, desc->n_q_heads, desc)) return rc;
  if (int rc = check_rows("kv_stride_row", desc->kv_stride_row, desc->n_kv_heads, desc)) return rc;
  if (!q || !k || !v || !slots || !q_out || !k_cache || !v_cache)
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among q/k/v/slots/q_out/k_cache/v_cache");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) ||
      !aligned(slots, 4))
    return fail(SPARROW_ERR_INVALID_ARG, "q, k, v, q_out and the caches must be 16-byte aligned, slots 4-byte");
  if (q_out == q && desc->q_stride_row != (int64_t)desc->n_q_heads * desc->head_dim)
    return fail(SPARROW_ERR_INVALID_ARG, "q_out may be q only where q's rows are contiguous");
  Frequencies f;
  if (int rc = frequencies(positions, axis_stride, n_axes, inv_freq, freq_axis, desc->head_dim, &f)) return rc;
  AppendArgs a;
  a.q = q; a.k = k; a.v = v; a.positions = positions; a.slots = slots;
  a.q_out = q_out; a.k_cache = k_cache; a.v_cache = v_cache;
  a.axis_stride = axis_stride; a.q_row = desc->q_stride_row; a.kv_row = desc->kv_stride_row;
  a.stride_page = desc->kv_stride_page; a.stride_token = desc->kv_stride_token; a.stride_head = desc->kv_stride_head;
  a.N = N; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads;
  a.page_shift = shift_of(desc->page_size); a.n_slots = desc->n_pages * desc->page_size;
  const hipError_t e = launch_mrope_append(desc->dtype, a, f, desc->head_dim, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "mrope_append launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

size_t sparrow_chunk_attn_workspace(const sparrow_paged_desc *desc, int32_t B, int32_t n_rows, int32_t max_new) {
  // (sizes that the call refuses would overflow what is worked out from them)
  if (!desc || (desc->dtype != SPARROW_F32 && desc->dtype != SPARROW_BF16) || (desc->head_dim != 64 && desc->head_dim != 128) ||
      desc->n_q_heads <= 0 || desc->n_q_heads > 1 << 15 || desc->n_kv_heads <= 0 || desc->n_q_heads % desc->n_kv_heads != 0 || B <= 0 ||
      B > SPARROW_MAX_PAGED_BATCH || n_rows <= 0 || n_rows > SPARROW_MAX_PAGED_TOKENS || (int64_t)n_rows * desc->n_q_heads >= 1ll << 31 ||
      max_new <= 0)
    return 0;
  const ChunkShape s = chunk_shape(desc->dtype, desc->head_dim, desc->n_q_heads, desc->n_kv_heads, B, n_rows, max_new, SPARROW_MAX_PAGED_TOKENS);
  return s.slots == 0 ? 0 : round_up((size_t)s.floats_o * 4, 256) + round_up((size_t)s.floats_ml * 4, 256) + round_up((size_t)B * 8, 256);
}

int sparrow_chunk_attn(const sparrow_paged_desc *desc, const void *q, const void *k_cache, const void *v_cache,
                       const int32_t *block_table, int32_t table_width, int64_t table_stride, const int32_t *cu_new,
                       const int32_t *kv_len, int32_t B, int32_t n_rows, int32_t max_new, void *out, float *lse,
                       void *workspace, size_t workspace_bytes, void *hip_stream) {
  g_err[0] = 0;
  if (int rc = check_desc(desc)) return rc;
  if (B < 0 || n_rows < 0 || max_new < 0)
    return fail(SPARROW_ERR_INVALID_ARG, "B = %d, n_rows = %d, max_new = %d", B, n_rows, max_new);
  if (B == 0 || n_rows == 0 || max_new == 0) return SPARROW_OK;
  if (int rc = check_table(B, desc->page_size, table_width, table_stride)) return rc;
  if (int rc = check_rows("q_stride_row", desc->q_stride_row, desc->n_q_heads, desc)) return rc;
  if (n_rows > SPARROW_MAX_PAGED_TOKENS)
    return fail(SPARROW_ERR_UNSUPPORTED, "n_rows = %d exceeds %d", n_rows, SPARROW_MAX_PAGED_TOKENS);
  if ((int64_t)n_rows * desc->n_q_heads >= 1ll << 31)
    return fail(SPARROW_ERR_UNSUPPORTED, "%d rows of %d heads (less than 2^31)", n_rows, desc->n_q_heads);
  if (!q || !k_cache || !v_cache || !block_table || !cu_new || !kv_len || !out)
    return fail(SPARROW_ERR_INVALID_ARG, "NULL pointer among q/k_cache/v_cache/block_table/cu_new/kv_len/out");
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16) || !aligned(block_table, 4) ||
      !aligned(cu_new, 4) || !aligned(kv_len, 4) || !aligned(lse, 4))
    return fail(SPARROW_ERR_INVALID_ARG, "q, the caches and out must be 16-byte aligned, the other arrays 4-byte");
  const size_t need = sparrow_chunk_attn_workspace(desc, B, n_rows, max_new);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(SPARROW_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
  if (need > 0 && !aligned(workspace, 256)) return fail(SPARROW_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  ChunkArgs a;
  a.q = q; a.k = k_cache; a.v = v_cache; a.block_table = block_table; a.cu_new = cu_new; a.kv_len = kv_len;
  a.out = out; a.lse = lse;
  a.table_stride = table_stride; a.q_row = desc->q_stride_row;
  a.stride_page = desc->kv_stride_page; a.stride_token = desc->kv_stride_token; a.stride_head = desc->kv_stride_head;
  a.B = B; a.n_rows = n_rows; a.max_new = max_new; a.Hq = desc->n_q_heads; a.Hkv = desc->n_kv_heads;
  a.g = desc->n_q_heads / desc->n_kv_heads; a.d = desc->head_dim;
  a.table_width = table_width; a.page_shift = shift_of(desc->page_size); a.n_pages = desc->n_pages;
  a.scale_log2 = (desc->scale > 0.f ? desc->scale : 1.0f / std::sqrt((float)desc->head_dim)) * kLog2e;
  a.inv_g = 1.0f / (float)a.g;
  const ChunkShape shape = chunk_shape(desc->dtype, desc->head_dim, a.Hq, a.Hkv, B, n_rows, max_new, (int64_t)table_width * desc->page_size);
  a.slots = shape.slots; a.round = shape.round; a.block_shift = shift_of(shape.rows);
  a.part_o = (float *)workspace;
  a.part_ml = (float *)((unsigned char *)workspace + round_up((size_t)shape.floats_o * 4, 256));
  a.plan = shape.slots == 0 ? nullptr : (int32_t *)((unsigned char *)a.part_ml + round_up((size_t)shape.floats_ml * 4, 256));
  const hipError_t e = launch_chunk_attn(desc->dtype, desc->head_dim, a, (hipStream_t)hip_stream);
  if (e != hipSuccess) return fail(SPARROW_ERR_DEVICE, "chunk_attn launch: %s", hipGetErrorString(e));
  return SPARROW_OK;
}

}  // extern "C"
