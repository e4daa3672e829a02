// Which kernel runs a call of the chunk attention, and its launches.
#include <algorithm>

#include "paged.hpp"

namespace sparrow {

hipError_t launch_chunk_few16(int dtype, int d, int rows, int waves, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_few32(int d, int rows, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_f32(int d, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_many(int d, int blocks, const ChunkArgs &a, hipStream_t st);
hipError_t launch_chunk_combine(int dtype, int d, const ChunkArgs &a, hipStream_t st);

ChunkShape chunk_shape(int dtype, int d, int Hq, int Hkv, int B, int64_t n_rows, int max_new, int64_t capacity) {
  ChunkShape s;
  const int64_t rows = std::min<int64_t>(max_new, n_rows) * (Hq / Hkv);        // of a request, at most
  const bool f32 = dtype == SPARROW_F32;
  s.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : f32 || rows <= 64 ? 64 : 256;
  // every request ends in a block of its own, not all of it filled
  s.blocks = rows <= s.rows ? B : (int)(n_rows * (Hq / Hkv) / s.rows) + B;
  // Single tokens: the fewer (request, KV head) pairs, the fewer and larger the workgroups, and the fewer pieces there are to put together.  us with 8
  // / 4 / 2 wavefronts, 256 / 512 / 1,024 workgroups at once, 28/4 heads of 128: one request of 26,112 tokens 15.9 / 16.8 / 18.9, eight of up to 8,000
  // 19.6 / 20.4 / 22.1, 32 of up to 4,000 32.4 / 31.3 / 32.5, 96 of up to 3,000 68.4 / 70.5 / 65.7, 200 of up to 2,048 104 / 95 / 91.  Around the borders: 12 of
  // up to 3,000 15.1 / 15.7 / 15.9, 16 of them 16.5 / 16.6 / 17.8; from 160 pairs to 256 (40 to 64 requests of up to 1,000, 3,000 and 8,000) 4 and 2
  // are within 3 % of each other either way.
  s.waves = f32 ? 4 : B * Hkv <= 48 ? 8 : B * Hkv < 192 ? 4 : 2;
  // workgroups that run at once
  const int at_once = s.rows == 16 && !f32 ? 2048 / s.waves : f32 && s.rows == 64 ? (d == 128 ? 512 : 1024) : 256;
  if (rows <= s.rows) {
    s.round = std::max(at_once / Hkv, 2 * B);
    // Requests of up to 512 tokens (fp32: 128, a tile takes three times as long) in one piece each and without a second pass.  The host does not know
    // the lengths: it goes by what the tables hold, so that a program whose tables are wider does not come by this.  us: one token of 28/4
    // heads over 380 tokens 9.3 -> 6.9, over 500 9.4 -> 7.5, over 1,000 10.6 -> 10.1, four such 11.0 -> 14.0; fp32 over 120 10.5 -> 8.1, over 250 10.5 -> 11.5.
    s.slots = capacity <= (f32 ? 128 : 512) ? 0 : s.round;
  } else {
    // Cut where the blocks fill two thirds of the chip at most; two rounds of pieces if they end sooner.  us, cut / whole, 28/4 heads of 128, new
    // tokens over 2,000 | 8,192 | 26,112: 1,000 (44 % filled) 51 / 54 | 127 / 173 | 353 / 519, 1,300 (56 %) 72 / 54 | 172 / 174 | 465 / 534, 1,500 (64 %)
    // 75 / 55 | 183 / 184 | 509 / 570, 1,600 (69 %) - | 190 / 185 | 626 / 579, 1,750 (75 %) - | 219 / 194 | 635 / 603.  From half to two thirds it hangs
    // on the lengths, which the host does not know.  fp32: 800 over 4,000 (69 %) 478 / 474, 750 (65 %) 347 / 474.  One round of pieces alone: chunk of 777
    // beside 8 single tokens, 32/8 heads of 64, 70 -> 89.
    const int64_t filled = (n_rows * (Hq / Hkv) + s.rows - 1) / s.rows;
    s.round = std::max(at_once / Hkv, 1);
    s.slots = 3 * filled <= 2 * s.round ? 2 * s.round : 0;
  }
  const int64_t units = (int64_t)s.slots * Hkv * s.rows;
  s.floats_o = units * d;
  s.floats_ml = units * 2;
  return s;
}

hipError_t launch_chunk_attn(int dtype, int d, const ChunkArgs &a, hipStream_t st) {
  const ChunkShape s = chunk_shape(dtype, d, a.Hq, a.Hkv, a.B, a.n_rows, a.max_new, (int64_t)a.table_width << a.page_shift);
  const int blocks = std::max(s.blocks, s.slots);
  hipError_t e;
  if (s.rows == 16 || (dtype == SPARROW_F32 && s.rows == 32)) e = launch_chunk_few16(dtype, d, s.rows, s.waves, blocks, a, st);
  else if (dtype == SPARROW_F32) e = launch_chunk_f32(d, blocks, a, st);
  else if (s.rows < 256) e = launch_chunk_few32(d, s.rows, blocks, a, st);
  else e = launch_chunk_many(d, blocks, a, st);
  if (e != hipSuccess || s.slots == 0) return e;
  return launch_chunk_combine(dtype, d, a, st);
}

}  // namespace sparrow
