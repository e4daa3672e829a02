// Attention of new tokens over a paged cache of 8 bits or of the model's type: a wavefront per (row of the batch, query head), key by key.
#include <type_traits>

#include "../paged/chunk_plan.hpp"
#include "serve.hpp"

namespace sparrow {

namespace {

template <typename T, typename C, int kD>
__global__ void __launch_bounds__(64) serve_attn_plain_kernel(ServeArgs a) {
  constexpr int kPer = kD / 64;
  const int lane = threadIdx.x, h = blockIdx.x, r = blockIdx.y + 32768 * blockIdx.z, c = h / a.g;
  if (r >= a.n_rows) return;
  int b = -1, i = 0, past = 0;
  for (int k = 0; k < a.B && b < 0; ++k) {
    const int c0 = min(max(a.cu_new[k], 0), a.n_rows), c1 = min(max(a.cu_new[k + 1], 0), a.n_rows);
    if (r >= c0 && r < c1) {
      b = k;
      i = r - c0;
      past = max(a.kv_len[k], 0) - (c1 - c0);
    }
  }
  if (b < 0 || i >= a.max_new) return;
  const int64_t to = (int64_t)r * a.Hq + h;
  const int pos = min(past + i, min(max(a.kv_len[b], 0), a.table_width << a.page_shift) - 1);
  float q[kPer], o[kPer], m = kNothingSeen, l = 0.f;
  for (int e = 0; e < kPer; ++e) {
    q[e] = Elem<T>::load((const T *)a.q + r * a.q_row + (int64_t)h * kD + kPer * lane + e);
    o[e] = 0.f;
  }
  for (int t = 0; t <= pos; ++t) {
    const unsigned int page = min((unsigned int)a.block_table[b * a.table_stride + (t >> a.page_shift)], (unsigned int)(a.n_pages - 1));
    const int token = t & ((1 << a.page_shift) - 1);
    const int64_t at = page * a.stride_page + token * a.stride_token + c * a.stride_head + kPer * lane;
    float k[kPer], v[kPer], s = 0.f;
    for (int e = 0; e < kPer; ++e) {
      if constexpr (std::is_same<C, e4m3_t>::value) {
        const unsigned int bytes = ((const unsigned short *)a.exponents)[(((int64_t)page * a.Hkv + c) << a.page_shift) + token];
        k[e] = __builtin_amdgcn_cvt_f32_fp8(((const e4m3_t *)a.k)[at + e], 0) * power_of(bytes & 0xffu);
        v[e] = __builtin_amdgcn_cvt_f32_fp8(((const e4m3_t *)a.v)[at + e], 0) * power_of(bytes >> 8);
      } else {
        k[e] = Elem<C>::load((const C *)a.k + at + e);
        v[e] = Elem<C>::load((const C *)a.v + at + e);
      }
      s = fmaf(q[e], k[e], s);
    }
    s = wave_sum(s);
    const float m_new = fmaxf(m, s), alpha = factor(m, m_new, a.scale_log2), p = factor(s, m_new, a.scale_log2);
    m = m_new;
    l = fmaf(l, alpha, p);
    for (int e = 0; e < kPer; ++e) o[e] = fmaf(o[e], alpha, p * v[e]);
  }
  for (int e = 0; e < kPer; ++e) Elem<T>::store((T *)a.out + to * kD + kPer * lane + e, pos < 0 ? 0.f : o[e] / l);
  if (a.lse && lane == 0) a.lse[to] = pos < 0 ? -INFINITY : log_sum(m, a.scale_log2, l);
}

template <typename T, typename C> hipError_t launch(int d, const ServeArgs &a, hipStream_t st) {
  const dim3 grid(a.Hq, a.n_rows < 32768 ? a.n_rows : 32768, (a.n_rows + 32767) / 32768);
  if (d == 128) hipLaunchKernelGGL((serve_attn_plain_kernel<T, C, 128>), grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL((serve_attn_plain_kernel<T, C, 64>), grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_serve_attn(int dtype, int d, const ServeArgs &a, hipStream_t st) {
  if (dtype == SPARROW_F32) return a.exponents ? launch<float, e4m3_t>(d, a, st) : launch<float, float>(d, a, st);
  return a.exponents ? launch<bf16_t, e4m3_t>(d, a, st) : launch<bf16_t, bf16_t>(d, a, st);
}

}  // namespace sparrow
