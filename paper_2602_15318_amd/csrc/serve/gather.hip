// Tokens of a paged cache into contiguous rows, an 8-bit cache's as the bf16 or fp32 numbers that it holds.
#include <type_traits>

#include "serve.hpp"

namespace sparrow {

namespace {

constexpr int kThreads = 256;

// A workgroup takes kThreads / kParts rows of one KV head; a thread 16 bytes of the cache for K and for V.  The request of a row is looked
// up by halving cu_rows, in LDS.  Nothing is rounded: a code times its power is a bf16 number.
//
// Bound by memory: 26,112 tokens of four heads of 128, 8 bits to bf16, 16.6 us, 81 MB, 4.9 TB/s, a copy's rate.
template <typename T, typename C, int kD>
__global__ void __launch_bounds__(kThreads) page_gather_kernel(GatherArgs a) {
  constexpr int kPer = 16 / (int)sizeof(C), kParts = kD / kPer, kRows = kThreads / kParts;
  constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  __shared__ int cu[SPARROW_MAX_PAGED_BATCH + 1];
  for (int i = threadIdx.x; i <= a.B; i += kThreads) cu[i] = a.cu_rows[i];
  __syncthreads();
  const int part = threadIdx.x % kParts, c = blockIdx.y;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / kParts;
  if (r >= a.n_rows || r < cu[0] || r >= cu[a.B]) return;
  int b = 0, end = a.B;                                    // cu[b] <= r < cu[end]
  while (end - b > 1) {
    const int mid = (b + end) >> 1;
    if (cu[mid] <= r) b = mid;
    else end = mid;
  }
  const int64_t t = (int64_t)(a.first ? a.first[b] : 0) + (r - cu[b]);
  if (t < 0 || t >= (int64_t)a.table_width << a.page_shift) return;
  const int token = (int)t & ((1 << a.page_shift) - 1);
  const unsigned int page = min((unsigned int)a.block_table[b * a.table_stride + (t >> a.page_shift)], (unsigned int)(a.n_pages - 1));
  const int64_t from = page * a.stride_page + token * a.stride_token + c * a.stride_head + part * kPer;
  const int64_t to = r * a.out_row + c * a.out_head + part * kPer;
  const u32x4 k = *(const u32x4 *)((const C *)a.k + from), v = *(const u32x4 *)((const C *)a.v + from);
  T *const ko = (T *)a.k_out + to, *const vo = (T *)a.v_out + to;
  if constexpr (!k8) {
    *(u32x4 *)ko = k;
    *(u32x4 *)vo = v;
  } else {
    const unsigned int bytes = ((const unsigned short *)a.exponents)[(((int64_t)page * a.Hkv + c) << a.page_shift) + token];
    const auto write = [&](T *out, u32x4 codes, float power) __attribute__((always_inline)) {
      typedef __attribute__((ext_vector_type(2))) float f32x2;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int w = (int)codes[2 * half + i];
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
          x[4 * i] = lo[0] * power;
          x[4 * i + 1] = lo[1] * power;
          x[4 * i + 2] = hi[0] * power;
          x[4 * i + 3] = hi[1] * power;
        }
        if constexpr (sizeof(T) == 2) {
          *(u32x4 *)(out + 8 * half) = (u32x4){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        } else {
          *(f32x4 *)(out + 8 * half) = (f32x4){x[0], x[1], x[2], x[3]};
          *(f32x4 *)(out + 8 * half + 4) = (f32x4){x[4], x[5], x[6], x[7]};
        }
      }
    };
    write(ko, k, power_of(bytes & 0xffu));
    write(vo, v, power_of(bytes >> 8));
  }
}

template <typename T, typename C, int kD> hipError_t launch(const GatherArgs &a, hipStream_t st) {
  constexpr int kRows = kThreads / (kD / (16 / (int)sizeof(C)));
  hipLaunchKernelGGL((page_gather_kernel<T, C, kD>), dim3((a.n_rows + kRows - 1) / kRows, a.Hkv), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}
template <typename T> hipError_t launch(int d, const GatherArgs &a, hipStream_t st) {
  if (a.exponents) return d == 128 ? launch<T, e4m3_t, 128>(a, st) : launch<T, e4m3_t, 64>(a, st);
  return d == 128 ? launch<T, T, 128>(a, st) : launch<T, T, 64>(a, st);
}

}  // namespace

hipError_t launch_page_gather(int dtype, int d, const GatherArgs &a, hipStream_t st) {
  return dtype == SPARROW_F32 ? launch<float>(d, a, st) : launch<bf16_t>(d, a, st);
}

}  // namespace sparrow
