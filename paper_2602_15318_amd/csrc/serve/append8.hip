// Rotation of a chunk's q and k rows, and the append of K and V to a paged cache of 8 bits per element.
#include "serve.hpp"

namespace sparrow {

namespace {

struct CosSin { double c, s; };

// cos and sin of `pos` times a frequency given in quarter turns, in 64 bits: the nearest whole number of quarter turns taken off, what is left, at
// most pi/4, through the Taylor series of sine and cosine, whose first missing terms are 2^-63 (x^19 / 19!) and 2^-59 (x^18 / 18!).
__device__ __forceinline__ CosSin cos_sin(int pos, double quarter) {
  const double x = (double)pos * quarter;
  const double n = __builtin_rint(x);
  const int k = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const double r = (x - n) * 1.5707963267948966, z = r * r;
  double s = 1.0 / 355687428096000.0, c = 1.0 / 20922789888000.0;
  s = fma(z, s, -1.0 / 1307674368000.0);
  s = fma(z, s, 1.0 / 6227020800.0);
  s = fma(z, s, -1.0 / 39916800.0);
  s = fma(z, s, 1.0 / 362880.0);
  s = fma(z, s, -1.0 / 5040.0);
  s = fma(z, s, 1.0 / 120.0);
  s = fma(z, s, -1.0 / 6.0);
  s = fma(z * s, r, r);
  c = fma(z, c, -1.0 / 87178291200.0);
  c = fma(z, c, 1.0 / 479001600.0);
  c = fma(z, c, -1.0 / 3628800.0);
  c = fma(z, c, 1.0 / 40320.0);
  c = fma(z, c, -1.0 / 720.0);
  c = fma(z, c, 1.0 / 24.0);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const double a = (k & 1) ? s : c, b = (k & 1) ? c : s;
  return {(k == 1 || k == 2) ? -a : a, (k & 2) ? -b : b};
}

// x in 32 bits, rounded to odd: what is rounded again to fewer bits from it comes out as from x itself.
__device__ __forceinline__ float to_odd(double x) {
  const float f = (float)x;
  const unsigned int u = __float_as_uint(f);
  if ((double)f == x || (u & 0x7f800000u) == 0x7f800000u) return f;      // exact; infinite; NaN
  return __uint_as_float((fabs((double)f) > fabs(x) ? u - 1u : u) | 1u);
}

// Over aligned groups of kN lanes
template <int kN> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = 1; o < kN; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// The power of two of a row whose largest finite size is `top`, as its byte: 448 is 0.875 * 2^9
__device__ __forceinline__ int byte_of(float top) {
  const unsigned int u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) > 0x600000u ? 7 : 8);
  return max(e, -100) + 127;
}

// A workgroup takes a token: its angles once, then a group of kParts lanes a head, 16 bytes of both halves each.  K is turned in 64 bits and rounded once,
// to the code: a key next to the border of two codes falls as the formula says; the power is that of what will be rounded.  q is turned in 32 bits by sines
// and cosines rounded from 64 and rounded once more to its type, off by some 2^-23 of the pair before that.
//
// Bound by memory: 8,192 tokens, 28 and 4 heads of 128 in bf16, 33.5 us, 143 MB, 4.3 TB/s (a copy: 4.9).  Eight tokens a workgroup 34.3 -> 36.9.  The call and
// its reading back, 43.8 us then: 50.9 with workgroups of 512, 44 to 47 with 64 and 128, 43.4 without the powers' stores, 42 with K in 32 bits: little but the
// bytes stands in the way.  13 tokens in fp32 3.4 us, a launch and its round trips.
template <typename T, int kD>
__global__ void __launch_bounds__(256) mrope_append8_kernel(Append8Args a, Frequencies f) {
  constexpr int kHalf = kD / 2, kPer = Elem<T>::kPer16B, kParts = kHalf / kPer;
  __shared__ double cs[2][kHalf];
  __shared__ float cs32[2][kHalf];
  const int n = blockIdx.x, tid = threadIdx.x;
  const int slot = a.slots[n];
  if ((unsigned)slot >= (unsigned)a.n_slots) return;      // uniform
  if (tid < kHalf) {
    const CosSin t = cos_sin(a.positions[f.axis[tid] * a.axis_stride + n], f.quarter[tid]);
    cs[0][tid] = t.c;
    cs[1][tid] = t.s;
    cs32[0][tid] = (float)t.c;
    cs32[1][tid] = (float)t.s;
  }
  __syncthreads();
  const int page = slot >> a.page_shift, token = slot & ((1 << a.page_shift) - 1);
  const int64_t cache = (int64_t)page * a.stride_page + (int64_t)token * a.stride_token;
  const int heads = a.Hq + 2 * a.Hkv;
  for (int x = tid; x < heads * kParts; x += 256) {       // (a group's lanes are all in or all out)
    const int h = x / kParts, part = x % kParts, i = part * kPer;
    const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
    const int c = is_v ? h - a.Hq - a.Hkv : h - a.Hq;
    const T *src = is_q ? (const T *)a.q + n * a.q_row + (int64_t)h * kD : (const T *)(is_v ? a.v : a.k) + n * a.kv_row + (int64_t)c * kD;
    u32x4 lo = *(const u32x4 *)(src + i), hi = *(const u32x4 *)(src + i + kHalf);
    float x0[kPer], x1[kPer];
    Elem<T>::unpack(lo, x0);
    Elem<T>::unpack(hi, x1);
    if (is_q) {
      T y0[kPer], y1[kPer];
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const float co = cs32[0][i + e], si = cs32[1][i + e];
        Elem<T>::store(&y0[e], x0[e] * co - x1[e] * si);
        Elem<T>::store(&y1[e], x1[e] * co + x0[e] * si);
      }
      __builtin_memcpy(&lo, y0, 16);
      __builtin_memcpy(&hi, y1, 16);
      T *dst = (T *)a.q_out + ((int64_t)n * a.Hq + h) * kD;
      *(u32x4 *)(dst + i) = lo;
      *(u32x4 *)(dst + i + kHalf) = hi;
      continue;
    }
    if (!is_v) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) {                     // in 64 bits: a key next to the border of two codes
        const double u = x0[e], w = x1[e], co = cs[0][i + e], si = cs[1][i + e];
        x0[e] = to_odd(u * co - w * si);
        x1[e] = to_odd(w * co + u * si);
      }
    }
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      if (!(fabsf(x0[e]) < INFINITY)) x0[e] = NAN;
      if (!(fabsf(x1[e]) < INFINITY)) x1[e] = NAN;
      top = fmaxf(top, fmaxf(fabsf(x0[e]), fabsf(x1[e])));       // (of a NaN and a number, the number)
    }
    const int byte = byte_of(group_max<kParts>(top));
    const float inv = __uint_as_float((unsigned int)(254 - byte) << 23);       // 2^(127 - byte), normal
    unsigned int w0[kPer / 4], w1[kPer / 4];
#pragma unroll
    for (int e = 0; e < kPer; e += 4) {
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(x0[e] * inv, x0[e + 1] * inv, 0, false);
      w0[e / 4] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(x0[e + 2] * inv, x0[e + 3] * inv, p, true);
      p = __builtin_amdgcn_cvt_pk_fp8_f32(x1[e] * inv, x1[e + 1] * inv, 0, false);
      w1[e / 4] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(x1[e + 2] * inv, x1[e + 3] * inv, p, true);
    }
    e4m3_t *dst = (is_v ? a.v_cache : a.k_cache) + cache + c * a.stride_head + i;
    __builtin_memcpy(__builtin_assume_aligned(dst, kPer), w0, kPer);
    __builtin_memcpy(__builtin_assume_aligned(dst + kHalf, kPer), w1, kPer);
    if (part == 0) a.exponents[((((int64_t)page * a.Hkv + c) << a.page_shift) + token) * 2 + (is_v ? 1 : 0)] = (uint8_t)byte;
  }
}

}  // namespace

hipError_t launch_mrope_append8(int dtype, const Append8Args &a, const Frequencies &f, int d, hipStream_t st) {
  const dim3 grid(a.N), block(256);
  if (dtype == SPARROW_BF16) {
    if (d == 128) hipLaunchKernelGGL((mrope_append8_kernel<bf16_t, 128>), grid, block, 0, st, a, f);
    else hipLaunchKernelGGL((mrope_append8_kernel<bf16_t, 64>), grid, block, 0, st, a, f);
  } else {
    if (d == 128) hipLaunchKernelGGL((mrope_append8_kernel<float, 128>), grid, block, 0, st, a, f);
    else hipLaunchKernelGGL((mrope_append8_kernel<float, 64>), grid, block, 0, st, a, f);
  }
  return hipGetLastError();
}

}  // namespace sparrow
