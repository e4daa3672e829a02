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
// As add_masked (chunk_attn_mfma.hpp): a product of a tile in which some rows do not see some keys.
__device__ __forceinline__ f32x4 add_masked16(bf16x4 v, bf16x4 p, bf16x4 seen, f32x4 o) {
  u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 bad = {no_numbers(w[0]), no_numbers(w[1])};
  if (__builtin_amdgcn_ballot_w64((bad[0] | bad[1]) != 0u) == 0ull) return mul16(v, p, o);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const u32x2 up = {ones_of(w[0], false), ones_of(w[1], false)}, down = {ones_of(w[0], true), ones_of(w[1], true)};
  w &= ~bad;
  return infinities(mul16(__builtin_bit_cast(bf16x4, w), p, o), mul16(__builtin_bit_cast(bf16x4, up), seen, zero),
                    mul16(__builtin_bit_cast(bf16x4, down), seen, zero));
}
__device__ __forceinline__ f32x4 add_masked4(float v, float p, float seen, f32x4 o) {
  const bool no = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u, nan = v != v;
  if (__builtin_amdgcn_ballot_w64(no) == 0ull) return __builtin_amdgcn_mfma_f32_16x16x4f32(v, p, o, 0, 0, 0);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  return infinities(__builtin_amdgcn_mfma_f32_16x16x4f32(no ? 0.f : v, p, o, 0, 0, 0),
                    __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v > 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0),
                    __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v < 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0));
}

}  // namespace sparrow
