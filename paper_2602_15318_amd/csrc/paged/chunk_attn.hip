// Attention of new tokens over the paged cache, plain version: a wavefront takes one (row, query head), 64 keys a round.
#include <algorithm>

#include "paged.hpp"

namespace sparrow {

namespace {

template <typename T, int kD>
__global__ void __launch_bounds__(256) chunk_attn_plain_kernel(ChunkArgs a) {
  constexpr int kPer = Elem<T>::kPer16B;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int r = (int)(unit / a.Hq), h = (int)(unit % a.Hq), c = h / a.g;
  if (r >= a.n_rows) return;
  int b = -1;                                             // the request that owns row r
  for (int k = 0; k < a.B; ++k)
    if (r >= a.cu_new[k] && r < a.cu_new[k + 1]) { b = k; break; }
  if (b < 0 || r - a.cu_new[b] >= a.max_new) return;
  const int kv = max(a.kv_len[b], 0), L = min(kv, a.table_width << a.page_shift);
  const int pos = min(L - 1, kv - (min(a.cu_new[b + 1], a.n_rows) - a.cu_new[b]) + (r - a.cu_new[b]));
  const int32_t *table = a.block_table + b * a.table_stride;
  auto row_of = [&](int t) {
    const unsigned page = min((unsigned)table[t >> a.page_shift], (unsigned)(a.n_pages - 1));
    return (int64_t)page * a.stride_page + (int64_t)(t & ((1 << a.page_shift) - 1)) * a.stride_token + c * a.stride_head;
  };
  const T *q = (const T *)a.q + r * a.q_row + (int64_t)h * kD;
  float m = kNegBig, l = 0.f, o[kD / 64];
#pragma unroll
  for (int e = 0; e < kD / 64; ++e) o[e] = 0.f;
  for (int t0 = 0; t0 <= pos; t0 += 64) {
    float s = -INFINITY;
    if (t0 + lane <= pos) {
      const T *k = (const T *)a.k + row_of(t0 + lane);
      s = 0.f;
      for (int i = 0; i < kD; i += kPer) {
        float x[kPer], y[kPer];
        Elem<T>::unpack(*(const u32x4 *)(k + i), x);
        Elem<T>::unpack(*(const u32x4 *)(q + i), y);
#pragma unroll
        for (int e = 0; e < kPer; ++e) s = fmaf(x[e], y[e], s);
      }
      s *= a.scale_log2;
    }
    const float m_new = fmaxf(m, wave_max(s)), alpha = fast_exp2(m - m_new);
    const float p = fast_exp2(s - m_new);
    l = l * alpha + wave_sum(p);
    m = m_new;
#pragma unroll
    for (int e = 0; e < kD / 64; ++e) o[e] *= alpha;
    for (int j = 0; j < 64 && t0 + j <= pos; ++j) {
      const float pj = __shfl(p, j, 64);
      const T *v = (const T *)a.v + row_of(t0 + j);
#pragma unroll
      for (int e = 0; e < kD / 64; ++e) o[e] = fmaf(pj, Elem<T>::load(v + lane + 64 * e), o[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < kD / 64; ++e)
    Elem<T>::store((T *)a.out + ((int64_t)r * a.Hq + h) * kD + lane + 64 * e, pos < 0 ? 0.f : o[e] / l);
  if (a.lse && lane == 0) a.lse[(int64_t)r * a.Hq + h] = pos < 0 ? -INFINITY : (m + fast_log2(l)) * kLn2;
}

}  // namespace

hipError_t launch_chunk_few(int d, int rows, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_many(int d, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_combine(int dtype, int d, int rows, const ChunkArgs &a, hipStream_t st);

ChunkShape chunk_shape(int dtype, int d, int Hq, int Hkv, int B, int64_t n_rows, int max_new) {
  ChunkShape s{0, 0, 0, 0};
  const int64_t rows = std::min<int64_t>(max_new, n_rows) * (Hq / Hkv);
  if (dtype != SPARROW_BF16) return s;
  if (rows <= 64) {
    s.rows = rows <= 32 ? 32 : 64;
    s.slots = std::max(256 / Hkv, 2 * B);
  } else {
    s.rows = 256;
    const int64_t blocks = (n_rows * (Hq / Hkv) + 255) / 256;
    s.slots = blocks * Hkv <= 128 ? 256 / Hkv : 0;         // (cut only where every block gets two pieces and more)
  }
  const int64_t units = (int64_t)s.slots * Hkv * s.rows;
  s.floats_o = units * d;
  s.floats_ml = units * 2;
  return s;
}

hipError_t launch_chunk_attn(int dtype, int d, const ChunkArgs &a, hipStream_t st) {
  const ChunkShape s = chunk_shape(dtype, d, a.Hq, a.Hkv, a.B, a.n_rows, a.max_new);
  if (s.rows > 0) {
    hipError_t e;
    if (s.rows < 256) {
      e = launch_chunk_few(d, s.rows, a, st);
    } else {                                               // every request ends in a block of its own, not all of it filled
      const int64_t blocks = std::max<int64_t>(((int64_t)a.n_rows * a.g) / 256 + a.B, s.slots);
      e = launch_chunk_many(d, (int)blocks, a, st);
    }
    if (e != hipSuccess || s.slots == 0) return e;
    return launch_chunk_combine(dtype, d, s.rows, a, st);
  }
  const dim3 grid((unsigned)(((int64_t)a.n_rows * a.Hq + 3) / 4)), block(256);
  if (dtype == SPARROW_BF16) {
    if (d == 128) hipLaunchKernelGGL((chunk_attn_plain_kernel<bf16_t, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((chunk_attn_plain_kernel<bf16_t, 64>), grid, block, 0, st, a);
  } else {
    if (d == 128) hipLaunchKernelGGL((chunk_attn_plain_kernel<float, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((chunk_attn_plain_kernel<float, 64>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sparrow
