// Internal interface of the paged-cache kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/sparrow_paged.h"
#include "../common.hpp"

namespace sparrow {

struct PageUpdateArgs {
  const int32_t *old_len, *new_len, *pos_offset;
  int32_t *block_table, *free_pages, *n_free, *slots, *positions, *cu_new, *status;
  int64_t table_stride;
  int32_t B, page_shift, table_width, capacity, n_rows;
};
hipError_t launch_page_update(const PageUpdateArgs &a, hipStream_t st);

// Frequencies in quarter turns per position and the axis of each, by value with the launch.
struct Frequencies {
  double quarter[64];
  uint8_t axis[64];
};
struct RopeTableArgs {
  const int32_t *positions;
  int64_t axis_stride;
  float *cos, *sin;
  int32_t N;
};
hipError_t launch_mrope_table(const RopeTableArgs &a, const Frequencies &f, int d, hipStream_t st);

struct AppendArgs {
  const void *q, *k, *v;
  const int32_t *positions, *slots;
  void *q_out, *k_cache, *v_cache;
  int64_t axis_stride, q_row, kv_row, stride_page, stride_token, stride_head;   // elements
  int32_t N, Hq, Hkv, page_shift, n_slots;
};
hipError_t launch_mrope_append(int dtype, const AppendArgs &a, const Frequencies &f, int d, hipStream_t st);

struct ChunkArgs {
  const void *q, *k, *v;
  const int32_t *block_table, *cu_new, *kv_len;
  void *out;
  float *lse;
  int64_t table_stride, q_row, stride_page, stride_token, stride_head;          // elements
  int32_t B, n_rows, max_new, Hq, Hkv, g, d, table_width, page_shift, n_pages;
  int32_t block_shift;     // log2 of the rows of a block
  int32_t slots, round;    // pieces per KV head that the blocks of rows may be cut into (0: one piece each); those that run at once
  float scale_log2, inv_g;
  float *part_o, *part_ml; // [piece * Hkv + KV head][row of the block]: unnormalised output [d]; reference score, sum
  int32_t *plan;           // [B][2]: a request's first piece, pieces of each of its blocks; NULL where nothing is cut
};
// How a call of these sizes is run: rows per block, blocks per KV head at most, pieces, wavefronts per workgroup
// (blocks of 16 rows), floats of part_o and part_ml.
struct ChunkShape {
  int rows, blocks, slots, round, waves;
  int64_t floats_o, floats_ml;
};
ChunkShape chunk_shape(int dtype, int d, int Hq, int Hkv, int B, int64_t n_rows, int max_new, int64_t capacity);
hipError_t launch_chunk_attn(int dtype, int d, const ChunkArgs &a, hipStream_t st);

}  // namespace sparrow
