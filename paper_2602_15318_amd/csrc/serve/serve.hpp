// Internal interface of the kernels behind include/sparrow_serve.h.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/sparrow_serve.h"
#include "../paged/paged.hpp"

namespace sparrow {

typedef unsigned char e4m3_t;   // raw bits

struct Append8Args {
  const void *q, *k, *v;
  const int32_t *positions, *slots;
  void *q_out;
  e4m3_t *k_cache, *v_cache;
  uint8_t *exponents;
  int64_t axis_stride, q_row, kv_row, stride_page, stride_token, stride_head;   // elements
  int32_t N, Hq, Hkv, page_shift, n_slots;
};
hipError_t launch_mrope_append8(int dtype, const Append8Args &a, const Frequencies &f, int d, hipStream_t st);

struct GatherArgs {
  const void *k, *v;
  const uint8_t *exponents;                               // NULL: caches of the outputs' type
  const int32_t *block_table, *first, *cu_rows;
  void *k_out, *v_out;
  int64_t table_stride, stride_page, stride_token, stride_head, out_row, out_head;    // elements
  int32_t B, n_rows, Hkv, table_width, page_shift, n_pages;
};
hipError_t launch_page_gather(int dtype, int d, const GatherArgs &a, hipStream_t st);

struct ServeLeft;
struct ServePiece;
struct ServeArgs {
  const void *q, *k, *v;
  const uint8_t *exponents;
  const int32_t *block_table, *cu_new, *kv_len, *group_start, *prefix_len;
  void *out;
  float *lse;
  int64_t table_stride, q_row, stride_page, stride_token, stride_head;          // elements
  int32_t B, G, n_rows, max_new, Hq, Hkv, g, table_width, page_shift, n_pages;
  int32_t block_shift;     // log2 of the rows of a block
  int32_t once;            // no page is another request's too, as far as is known
  int32_t slots, round;    // pieces per KV head at most (0: nothing is cut or shared, one piece a block); those that run at once
  int32_t ways;            // ways to cut that a plan without groups tries (serve_plan.hpp)
  float scale_log2, inv_g;
  float *part_o, *part_ml; // [piece * Hkv + KV head][row of the block]: unnormalised output [d]; reference score, sum
  ServeLeft *left;         // [B]; NULL where slots is 0
  ServePiece *pieces;      // with groups: [slots], n_pieces of them
  int32_t *n_pieces;
};
// How a call of these sizes is run: rows per block, wavefronts per workgroup (16 rows), pieces per KV head at most, those that run at once, ways to cut, workgroups per KV head, floats of part_o and part_ml.
struct ServeShape {
  int rows, waves, slots, round, ways, grid;
  int64_t floats_o, floats_ml;
};
// Whether prefixes are read once for their groups, by what the tables of the batch could hold: B of `capacity` tokens; rows: of a request, at most.
bool serve_shares(int dtype, bool eight, int d, int Hkv, int B, int64_t capacity, int64_t rows);
ServeShape serve_shape(int dtype, int d, int Hq, int Hkv, int B, int G, int64_t n_rows, int max_new, int64_t capacity);
hipError_t launch_serve_attn(int dtype, int d, const ServeShape &s, const ServeArgs &a, hipStream_t st);

// 2^(byte - 127) of a row of an 8-bit cache, normal and finite whatever the byte
__device__ __forceinline__ float power_of(unsigned int byte) { return __uint_as_float(min(max(byte, 1u), 254u) << 23); }

// Weights reach 2^8 (kSlack): beside an 8-bit cache the attention's outputs are kept, in partials too, times this, so that a weight times a power, or
// times an element, is finite where the element is.  What divides by the weights' sum puts it right, exactly.
constexpr float kLowered = 0x1p-8f;
__device__ __forceinline__ float lowered(const ServeArgs &a) { return a.exponents ? kLowered : 1.f; }

}  // namespace sparrow
