// What the two forms of the bf16 attention (attn_few.hpp, attn_many.hpp) share: where a tile's rows are, and rows of an 8-bit cache as bf16 numbers.
#pragma once
#include <type_traits>

#include "../paged/chunk_attn_16.hpp"
#include "serve_plan.hpp"

namespace sparrow {

// The pages of an item's KV head.  Rows that are asked for together lie on one page.
template <typename C> struct ServePages {
  const int32_t __attribute__((address_space(4))) *table;     // read through the scalar cache
  const unsigned char *k, *v;                                  // the head's first row
  const unsigned char *powers;                                 // the head's first token, K's byte below V's
  int64_t stride_page, powers_page;                            // bytes; tokens
  unsigned int stride_token;
  int shift, last;                                             // last page entry that the item holds
  unsigned int last_page;
  struct Place { int64_t at, token; };
  __device__ __forceinline__ Place place(int t) const {        // t uniform; tokens past the item's: some row of its last page
    const unsigned int page = min((unsigned int)table[min(t >> shift, last)], last_page);
    const int row = t & ((1 << shift) - 1);
    return {(int64_t)page * stride_page + (int64_t)row * stride_token, (int64_t)page * powers_page + row};
  }
  // The bytes of row `row` (and of its neighbour, four in all) of rows that begin at an even token
  __device__ __forceinline__ unsigned int powers_of(Place at, int row) const { return *(const unsigned int *)(powers + 2 * at.token + 2 * (row & ~1)); }
};
template <typename C> __device__ __forceinline__ ServePages<C> serve_pages(const ServeArgs &a, const ServeItem &it, int c) {
  ServePages<C> p;
  p.table = (const int32_t __attribute__((address_space(4))) *)(uintptr_t)(a.block_table + (int64_t)it.table * a.table_stride);
  p.k = (const unsigned char *)((const C *)a.k + (int64_t)c * a.stride_head);
  p.v = (const unsigned char *)((const C *)a.v + (int64_t)c * a.stride_head);
  p.powers = a.exponents + 2 * ((int64_t)c << a.page_shift);
  p.stride_page = (int64_t)sizeof(C) * a.stride_page;
  p.powers_page = (int64_t)a.Hkv << a.page_shift;
  p.stride_token = (unsigned int)(sizeof(C) * a.stride_token);
  p.shift = a.page_shift;
  p.last = max(it.to - 1, 0) >> a.page_shift;
  p.last_page = (unsigned int)(a.n_pages - 1);
  return p;
}

// K's, or V's, power of row `row` from the four bytes of it and its neighbour.  V's is kLowered (serve.hpp) below what stands there: finite times any weight.
__device__ __forceinline__ float power_in(unsigned int bytes, int row, bool is_v) {
  const unsigned int byte = (bytes >> (16 * (row & 1) + (is_v ? 8 : 0))) & 0xffu;
  return is_v ? __uint_as_float((min(max(byte, 9u), 254u) - 8u) << 23) : power_of(byte);
}
// Four codes times a power of two, exactly, as four bf16
__device__ __forceinline__ u32x2 four_of(unsigned int codes, float power) {
  return (u32x2){__builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, false)),
                 __builtin_bit_cast(unsigned int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, true))};
}

// 4 bytes per lane, each from an address of its own, to LDS: lane l's at dst + 4 l
__device__ __forceinline__ void global_to_lds_4(const void *at, unsigned int dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" ::"s"(dst), "v"(at) : "memory", "m0");
}

}  // namespace sparrow
