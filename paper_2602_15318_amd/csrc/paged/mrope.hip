// Rotary positions with several axes: table rows, and the rotation of a chunk's q and k with the append to the cache.
#include "paged.hpp"

namespace sparrow {

namespace {

struct CosSin { float c, s; };

// cos and sin of `pos` times a frequency given in quarter turns: x = pos * quarter in 64 bits (a position of 2^31 leaves 2^-22
// of a turn of its 53 bits' error), its nearest whole number of quarter turns taken off exactly; what is left, at most pi/4,
// goes through the Taylor series of sine and cosine, whose first missing terms are 2^-29 (x^11 / 11!) and 2^-33 (x^12 / 12!).
__device__ __forceinline__ CosSin cos_sin(int pos, double quarter) {
  const double x = (double)pos * quarter;
  const double n = __builtin_rint(x);
  const int k = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const float r = (float)((x - n) * 1.5707963267948966), r2 = r * r;
  float s = fmaf(r2, 2.7557319e-06f, -1.9841270e-04f);
  s = fmaf(r2, s, 8.3333333e-03f);
  s = fmaf(r2, s, -1.6666667e-01f);
  s = fmaf(r2 * s, r, r);
  float c = fmaf(r2, -2.7557319e-07f, 2.4801587e-05f);
  c = fmaf(r2, c, -1.3888889e-03f);
  c = fmaf(r2, c, 4.1666667e-02f);
  c = fmaf(r2, c, -0.5f);
  c = fmaf(r2, c, 1.0f);
  const float a = (k & 1) ? s : c, b = (k & 1) ? c : s;
  return {(k == 1 || k == 2) ? -a : a, (k & 2) ? -b : b};
}

// A thread takes one frequency of a token (four, for 16-byte stores: 26,112 tokens of heads of 128 5.9 -> 7.2 us).
template <int kD>
__global__ void __launch_bounds__(256) mrope_table_kernel(RopeTableArgs a, Frequencies f) {
  constexpr int kHalf = kD / 2;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int n = (int)(at / kHalf), i = (int)(at % kHalf);
  if (n >= a.N) return;
  const CosSin t = cos_sin(a.positions[f.axis[i] * a.axis_stride + n], f.quarter[i]);
  a.cos[at] = t.c;
  a.sin[at] = t.s;
}

// A workgroup takes a token: its angles once, then 16 bytes of both halves of a head per thread.  Bound by memory: 8,192 tokens of 28/4 heads of
// 128, bf16, 151 MB read and written, 31.6 us a call among others (4.8 TB/s, a large copy 5.05), 24.3 with the inputs in the Infinity Cache; in fp32 82
// behind other work on memory (bf16 44 there).
template <typename T, int kD>
__global__ void __launch_bounds__(256) mrope_append_kernel(AppendArgs a, Frequencies f) {
  constexpr int kHalf = kD / 2, kPer = Elem<T>::kPer16B, kParts = kHalf / kPer;
  __shared__ __attribute__((aligned(16))) float cs[2][kHalf];
  const int n = blockIdx.x, tid = threadIdx.x;
  const int slot = a.slots[n];
  if ((unsigned)slot >= (unsigned)a.n_slots) return;      // uniform
  if (tid < kHalf) {
    const CosSin t = cos_sin(a.positions[f.axis[tid] * a.axis_stride + n], f.quarter[tid]);
    cs[0][tid] = t.c;
    cs[1][tid] = t.s;
  }
  __syncthreads();
  const int64_t cache = (int64_t)(slot >> a.page_shift) * a.stride_page + (int64_t)(slot & ((1 << a.page_shift) - 1)) * a.stride_token;
  const int heads = a.Hq + 2 * a.Hkv;
  for (int x = tid; x < heads * kParts; x += 256) {
    const int h = x / kParts, i = x % kParts * kPer;
    const T *src;
    T *dst;
    if (h < a.Hq) {
      src = (const T *)a.q + n * a.q_row + (int64_t)h * kD;
      dst = (T *)a.q_out + ((int64_t)n * a.Hq + h) * kD;
    } else {
      const int c = h < a.Hq + a.Hkv ? h - a.Hq : h - a.Hq - a.Hkv;
      src = (const T *)(h < a.Hq + a.Hkv ? a.k : a.v) + n * a.kv_row + (int64_t)c * kD;
      dst = (T *)(h < a.Hq + a.Hkv ? a.k_cache : a.v_cache) + cache + c * a.stride_head;
    }
    u32x4 lo = *(const u32x4 *)(src + i), hi = *(const u32x4 *)(src + i + kHalf);
    if (h < a.Hq + a.Hkv) {
      float x0[kPer], x1[kPer];
      T y0[kPer], y1[kPer];
      Elem<T>::unpack(lo, x0);
      Elem<T>::unpack(hi, x1);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const float c = cs[0][i + e], s = cs[1][i + e];
        Elem<T>::store(&y0[e], x0[e] * c - x1[e] * s);
        Elem<T>::store(&y1[e], x1[e] * c + x0[e] * s);
      }
      __builtin_memcpy(&lo, y0, 16);
      __builtin_memcpy(&hi, y1, 16);
    }
    *(u32x4 *)(dst + i) = lo;
    *(u32x4 *)(dst + i + kHalf) = hi;
  }
}

}  // namespace

hipError_t launch_mrope_table(const RopeTableArgs &a, const Frequencies &f, int d, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.N * (d / 2) + 255) / 256));
  if (d == 128) hipLaunchKernelGGL(mrope_table_kernel<128>, grid, dim3(256), 0, st, a, f);
  else hipLaunchKernelGGL(mrope_table_kernel<64>, grid, dim3(256), 0, st, a, f);
  return hipGetLastError();
}

hipError_t launch_mrope_append(int dtype, const AppendArgs &a, const Frequencies &f, int d, hipStream_t st) {
  const dim3 grid(a.N), block(256);
  if (dtype == SPARROW_BF16) {
    if (d == 128) hipLaunchKernelGGL((mrope_append_kernel<bf16_t, 128>), grid, block, 0, st, a, f);
    else hipLaunchKernelGGL((mrope_append_kernel<bf16_t, 64>), grid, block, 0, st, a, f);
  } else {
    if (d == 128) hipLaunchKernelGGL((mrope_append_kernel<float, 128>), grid, block, 0, st, a, f);
    else hipLaunchKernelGGL((mrope_append_kernel<float, 64>), grid, block, 0, st, a, f);
  }
  return hipGetLastError();
}

}  // namespace sparrow
