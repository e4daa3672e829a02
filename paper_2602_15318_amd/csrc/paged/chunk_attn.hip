// Which kernel runs a call of the chunk attention, and its launches.
#include <algorithm>

#include "paged.hpp"

namespace sparrow {

hipError_t launch_chunk_few16(int dtype, int d, int rows, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_few32(int d, int rows, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_many(int d, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_combine(int dtype, int d, int rows, const ChunkArgs &a, hipStream_t st);

ChunkShape chunk_shape(int dtype, int d, int Hq, int Hkv, int B, int64_t n_rows, int max_new) {
  ChunkShape s;
  const int64_t rows = std::min<int64_t>(max_new, n_rows) * (Hq / Hkv);        // of a request, at most
  const bool f32 = dtype == SPARROW_F32;
  s.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : f32 || rows <= 64 ? 64 : 256;
  // every request ends in a block of its own, not all of it filled
  s.blocks = rows <= s.rows ? B : (int)(n_rows * (Hq / Hkv) / s.rows) + B;
  if (rows <= s.rows) {
    s.slots = std::max((s.rows == 16 && !f32 ? 512 : 256) / Hkv, 2 * B);
  } else {
    const int64_t filled = (n_rows * (Hq / Hkv) + s.rows - 1) / s.rows;
    s.slots = filled * Hkv <= 128 ? 256 / Hkv : 0;         // (cut only where every block gets two pieces and more)
  }
  const int64_t units = (int64_t)s.slots * Hkv * s.rows;
  s.floats_o = units * d;
  s.floats_ml = units * 2;
  return s;
}

hipError_t launch_chunk_attn(int dtype, int d, const ChunkArgs &a, hipStream_t st) {
  const ChunkShape s = chunk_shape(dtype, d, a.Hq, a.Hkv, a.B, a.n_rows, a.max_new);
  const int blocks = std::max(s.blocks, s.slots);
  hipError_t e;
  if (dtype == SPARROW_F32 || s.rows == 16) e = launch_chunk_few16(dtype, d, s.rows, blocks, a, st);
  else if (s.rows < 256) e = launch_chunk_few32(d, s.rows, a, st);
  else e = launch_chunk_many(d, blocks, a, st);
  if (e != hipSuccess || s.slots == 0) return e;
  return launch_chunk_combine(dtype, d, s.rows, a, st);
}

}  // namespace sparrow
