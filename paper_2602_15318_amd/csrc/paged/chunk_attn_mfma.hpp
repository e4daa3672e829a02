// Building blocks of the chunk attention on the matrix cores, bf16: tiles of pages in LDS, operands, softmax of a tile.
//
// With v_mfma_f32_32x32x16_bf16 (A: 32 x 16, lane = row + 32 * (k / 8), eight k each; B: 16 x 32, lane = column + 32 * (k / 8); D: 32 x
// 32, lane = column + 32 * h, element e in row 8 (e / 4) + 4 h + e % 4):
//   S^T = K Q^T    a lane holds, for its row of the batch (column lane % 32), the scores of keys 8 (e / 4) + 4 h + e % 4 of 32.
//   O^T += V^T P^T  the k index of a 16-key step is taken in the order in which the lanes hold the scores, so P^T is the scores' own
//                 registers and V^T two transposing reads (ds_read_b64_tr_b16) of four keys each.
#pragma once
#include "chunk_plan.hpp"

namespace sparrow {

typedef __attribute__((ext_vector_type(16))) float f32x16;

// 16 bytes per lane from base + off to LDS, lane l's at dst + 16 l (base and dst uniform).  Not counted by the compiler: wait_loads()
// waits.  The wait states are those between a scalar register written by the vector ALU, or M0, and its use here.
template <bool kNt> __device__ __forceinline__ void global_to_lds(const void *base, unsigned int off, unsigned int dst) {
  if constexpr (kNt)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(dst), "v"(off), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void global_to_lds_each(const void *at, unsigned int dst) {      // an address of its own per lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(at) : "memory", "m0");
}

// Rows of a tile: 2 kD bytes, the 16-byte chunks XOR-swizzled by the row so that what is read together falls on different banks: of K
// 16 bytes of each of 32 rows, of V, transposed, 64 bytes of each of four rows at a time.  What loads a tile writes LDS in lane order, so the
// lane picks the chunk that belongs there.  Both together, chunk of 2,048 tokens over 26,112: 692 -> 653 us.  (kFold: the chunk's lowest bit by the
// eight rows, without it rows 8 apart meet; few rows leave LDS idle, and its offsets cost registers there.)
template <int kD, bool kFold = true> struct Tile {
  static constexpr int kRow = 2 * kD, kChunks = kD / 8, kLoadRows = 64 / kChunks;    // rows that one load of a wavefront covers
  static __device__ __forceinline__ int swz_k(int row) {
    return (kD == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1) ^ (kFold ? (row >> 3) & 1 : 0);
  }
  static __device__ __forceinline__ int swz_v(int row) {
    return (kD == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2) | ((row >> 2) & 1) << 1;
  }
  static __device__ __forceinline__ int k(int row, int chunk) { return row * kRow + ((chunk ^ swz_k(row)) << 4); }
  static __device__ __forceinline__ int v(int row, int chunk) { return row * kRow + ((chunk ^ swz_v(row)) << 4); }
  // Of rows `row` + lane / kChunks: bytes from that row of the memory that lane fetches from
  static __device__ __forceinline__ unsigned int k_from(int lane, int row, unsigned int stride) {
    return (unsigned int)(lane / kChunks) * stride + 16u * ((lane % kChunks) ^ swz_k(row + lane / kChunks));
  }
  static __device__ __forceinline__ unsigned int v_from(int lane, int row, unsigned int stride) {
    return (unsigned int)(lane / kChunks) * stride + 16u * ((lane % kChunks) ^ swz_v(row + lane / kChunks));
  }
};

// The pages of a request's KV head: where the rows from a token on are.  Rows of one load lie on one page (16 tokens and more).
struct Pages {
  const int32_t __attribute__((address_space(4))) *table;     // read through the scalar cache
  const unsigned char *k, *v;                                  // the head's first row
  int64_t stride_page;                                         // bytes
  unsigned int stride_token;
  int shift, last;                                             // last page entry that the request holds
  unsigned int last_page;
  __device__ __forceinline__ int64_t offset(int t) const {     // t uniform; tokens past the request: some row of its last page
    const unsigned int page = min((unsigned int)table[min(t >> shift, last)], last_page);
    return (int64_t)page * stride_page + (int64_t)(t & ((1 << shift) - 1)) * stride_token;
  }
};
__device__ __forceinline__ Pages pages_of(const ChunkArgs &a, const Piece &pc, int c) {
  Pages p;
  p.table = (const int32_t __attribute__((address_space(4))) *)(uintptr_t)(a.block_table + (int64_t)pc.b * a.table_stride);
  p.k = (const unsigned char *)a.k + 2 * (int64_t)c * a.stride_head;
  p.v = (const unsigned char *)a.v + 2 * (int64_t)c * a.stride_head;
  p.stride_page = 2 * a.stride_page;
  p.stride_token = (unsigned int)(2 * a.stride_token);
  p.shift = a.page_shift;
  p.last = max(pc.rq.L - 1, 0) >> a.page_shift;
  p.last_page = (unsigned int)(a.n_pages - 1);
  return p;
}

// The wavefront's LDS reads and writes are done before the barrier; its loads to LDS are not waited for.
__device__ __forceinline__ void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ bf16x8 lds_b128(const unsigned char *p) { return *reinterpret_cast<const bf16x8 *>(p); }
__device__ __forceinline__ bf16x4 lds_tr(const unsigned char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)p);
}
// Offsets into a tile from which a lane's operands are one XOR (columns) and an immediate (rows) away: K of columns 16 ks .. by k_at ^ ks <<
// 5, V^T of the 32-wide d-block db by vt_at ^ db << 6.
template <int kD, bool kFold = true> __device__ __forceinline__ int k_at(int lane) { return Tile<kD, kFold>::k(lane & 31, lane >> 5); }
template <int kD> __device__ __forceinline__ int vt_at(int lane) {
  const int p = lane & 15;
  return Tile<kD>::v(4 * (lane >> 5) + (p >> 2), 2 * ((lane >> 4) & 1) + ((p >> 1) & 1)) + 8 * (p & 1);
}
// V^T operand of the 16-key step `s`, from the block's offset.  Lane: d 32 db + lane % 32, keys 16 s + 8 jj + 4 h + 0..3.
template <int kD> __device__ __forceinline__ bf16x8 read_vt(const unsigned char *at, int s) {
  const bf16x4 x = lds_tr(at + 16 * s * Tile<kD>::kRow), y = lds_tr(at + (16 * s + 8) * Tile<kD>::kRow);
  return (bf16x8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ float pair_max(float v) {            // over lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Two bf16 elements: the top bit of each half that is no number, and the whole halves.
__device__ __forceinline__ unsigned int not_finite(unsigned int w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ unsigned int no_numbers(unsigned int w) { return (not_finite(w) >> 15) * 0xffffu; }
// 1.0 in the halves that are infinite of that sign, or NaN
__device__ __forceinline__ unsigned int ones_of(unsigned int w, bool negative) {
  unsigned int r = 0u;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const unsigned int x = (w >> (16 * half)) & 0xffffu;
    const bool no = (x & 0x7f80u) == 0x7f80u, nan = (x & 0x7fu) != 0u;
    if (no && (nan || ((x & 0x8000u) != 0u) == negative)) r |= 0x3f80u << (16 * half);
  }
  return r;
}
// O^T += V^T P^T of a 16-key step of a tile in which some rows do not see some keys, all d-blocks.  0 * inf must not reach those rows, so what is
// no number leaves the operand; whether a row sees one such value or more is counted by products of ones, exactly, and adds the infinities
// then (a NaN counts as both).
template <int kN> __device__ __forceinline__ void add_masked(const bf16x8 (&v)[kN], bf16x8 p, bf16x8 seen, f32x16 *o) {
  unsigned int any = 0u;
#pragma unroll
  for (int db = 0; db < kN; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= not_finite(__builtin_bit_cast(u32x4, v[db])[i]);
  if (__builtin_amdgcn_ballot_w64(any != 0u) == 0ull) {
#pragma unroll
    for (int db = 0; db < kN; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db], p, o[db], 0, 0, 0);
    return;
  }
#pragma unroll
  for (int db = 0; db < kN; ++db) {
    u32x4 w = __builtin_bit_cast(u32x4, v[db]), up, down;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      up[i] = ones_of(w[i], false);
      down[i] = ones_of(w[i], true);
      w[i] &= ~no_numbers(w[i]);
    }
    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), p, o[db], 0, 0, 0);
    const f32x16 zero = {0.f};
    const f32x16 cu = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, up), seen, zero, 0, 0, 0);
    const f32x16 cd = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, down), seen, zero, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 16; ++e) o[db][e] += (cu[e] > 0.f ? INFINITY : 0.f) + (cd[e] > 0.f ? -INFINITY : 0.f);
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace sparrow
