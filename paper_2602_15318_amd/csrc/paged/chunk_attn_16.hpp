// Building blocks of the chunk attention by tiles of 16 rows and 16 keys.
#pragma once
#include <type_traits>

#include "chunk_attn_mfma.hpp"

namespace sparrow {

typedef __attribute__((ext_vector_type(4))) short s16x4;

// Over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ f32x4 mul16(bf16x4 v, bf16x4 p, f32x4 o) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, v), __builtin_bit_cast(s16x4, p), o, 0, 0, 0);
}
__device__ __forceinline__ f32x4 infinities(f32x4 o, f32x4 up, f32x4 down) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] += (up[i] > 0.f ? INFINITY : 0.f) + (down[i] > 0.f ? -INFINITY : 0.f);
  return o;
}
// As add_masked (chunk_attn_mfma.hpp), of 16 keys.
template <int kN> __device__ __forceinline__ void add_masked16(const bf16x4 (&v)[kN], bf16x4 p, bf16x4 seen, f32x4 *o) {
  unsigned int any = 0u;
#pragma unroll
  for (int db = 0; db < kN; ++db) any |= not_finite(__builtin_bit_cast(u32x2, v[db])[0]) | not_finite(__builtin_bit_cast(u32x2, v[db])[1]);
  if (__builtin_amdgcn_ballot_w64(any != 0u) == 0ull) {
#pragma unroll
    for (int db = 0; db < kN; ++db) o[db] = mul16(v[db], p, o[db]);
    return;
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int db = 0; db < kN; ++db) {
    const u32x2 w = __builtin_bit_cast(u32x2, v[db]), fine = {w[0] & ~no_numbers(w[0]), w[1] & ~no_numbers(w[1])};
    const u32x2 up = {ones_of(w[0], false), ones_of(w[1], false)}, down = {ones_of(w[0], true), ones_of(w[1], true)};
    o[db] = infinities(mul16(__builtin_bit_cast(bf16x4, fine), p, o[db]), mul16(__builtin_bit_cast(bf16x4, up), seen, zero),
                       mul16(__builtin_bit_cast(bf16x4, down), seen, zero));
  }
}
// Of one k-step of the fp32 product, 4 keys.
template <int kN> __device__ __forceinline__ void add_masked4(const float (&v)[kN], float p, float seen, f32x4 *o) {
  bool any = false;
#pragma unroll
  for (int db = 0; db < kN; ++db) any |= (__float_as_uint(v[db]) & 0x7f800000u) == 0x7f800000u;
  if (__builtin_amdgcn_ballot_w64(any) == 0ull) {
#pragma unroll
    for (int db = 0; db < kN; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[db], p, o[db], 0, 0, 0);
    return;
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int db = 0; db < kN; ++db) {
    const bool no = (__float_as_uint(v[db]) & 0x7f800000u) == 0x7f800000u, nan = v[db] != v[db];
    o[db] = infinities(__builtin_amdgcn_mfma_f32_16x16x4f32(no ? 0.f : v[db], p, o[db], 0, 0, 0),
                       __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v[db] > 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0),
                       __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v[db] < 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0));
  }
}

}  // namespace sparrow
