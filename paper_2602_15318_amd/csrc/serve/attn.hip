// Which kernel runs a call of the attention, and its launches.
#include <algorithm>

#include "serve.hpp"

namespace sparrow {

hipError_t launch_serve_plan(const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_bf16(int d, const ServeShape &s, const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_f32(int d, int pieces, const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_combine(int dtype, int d, const ServeArgs &a, hipStream_t st);

// The plan, blocks that are partly filled and a second pass over all rows cost 5 to 9 us, and what a group's requests read of one prefix comes out of the
// caches: below these sizes every request reads its own.  bf16, shared and not, us: 8 of 2,100 tokens (34 MB) 20.0 and 14.0; 4 of 8,500 (70 MB) 22.5 and
// 17.8; 8 of 8,300 (137 MB) 23.7 and 23.1; 16 of them 27.4 and 39.1; 8 of 26,300 (430 MB) 28.7 and 59.4.  fp32: 4 of 2,060 (34 MB) 21.3 and 20.7; 8
// (68 MB) 22.7 and 26.1.
bool serve_shares(int dtype, int64_t tokens, int64_t bytes) { return tokens > (dtype == SPARROW_F32 ? 1ll << 25 : 1ll << 27) / bytes; }

ServeShape serve_shape(int dtype, int d, int Hq, int Hkv, int B, int G, int64_t n_rows, int max_new, int64_t capacity) {
  ServeShape s;
  const bool f32 = dtype == SPARROW_F32;
  const int g = Hq / Hkv;
  const int64_t most = std::min<int64_t>(max_new, n_rows) * g;                 // rows of a request, at most
  const int64_t of_item = G > 0 ? n_rows * g : most;                           // of an item
  s.rows = of_item <= 16 ? 16 : f32 || of_item <= 64 ? 64 : 256;
  // every item ends in a block of its own, not all of it filled
  const int64_t blocks = (most <= s.rows ? 0 : n_rows * g / s.rows) + B + (G > 0 ? n_rows * g / s.rows + G : 0);
  // Single tokens: the fewer (request, KV head) pairs, the fewer and larger the workgroups, and the fewer pieces there are to put together.
  s.waves = B * Hkv <= 48 ? 8 : B * Hkv < 192 ? 4 : 2;
  const int at_once = f32 ? (d == 128 ? 512 : 1024) : G == 0 && s.rows == 16 ? 2048 / s.waves : 256;       // workgroups
  s.round = std::max(at_once / Hkv, 1);
  if (G > 0) {
    s.slots = (int)std::max<int64_t>(4 * s.round, blocks);
  } else if (most <= s.rows) {
    s.round = std::max(s.round, 2 * B);
    // Requests of up to 512 tokens (fp32: 128) in one piece each and without a second pass, by what the tables hold.
    s.slots = capacity <= (f32 ? 128 : 512) ? 0 : s.round;
  } else {
    // Cut where the blocks fill two thirds of the chip at most; two rounds of pieces if they end sooner.
    const int64_t filled = (n_rows * g + s.rows - 1) / s.rows;
    s.slots = 3 * filled <= 2 * s.round ? 2 * s.round : 0;
  }
  s.grid = (int)std::max<int64_t>(s.slots, G > 0 ? 0 : blocks);
  const int64_t units = (int64_t)s.slots * Hkv * s.rows;
  s.floats_o = units * d;
  s.floats_ml = units * 2;
  return s;
}

hipError_t launch_serve_attn(int dtype, int d, const ServeShape &s, const ServeArgs &a, hipStream_t st) {
  hipError_t e = a.G > 0 ? launch_serve_plan(a, st) : hipSuccess;
  if (e != hipSuccess) return e;
  e = dtype == SPARROW_F32 ? launch_serve_f32(d, s.grid, a, st) : launch_serve_bf16(d, s, a, st);
  if (e != hipSuccess || s.slots == 0) return e;
  return launch_serve_combine(dtype, d, a, st);
}

}  // namespace sparrow
