// Which kernel runs a call of the attention, and its launches.
#include <algorithm>

#include "serve.hpp"

namespace sparrow {

hipError_t launch_serve_plan(const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_bf16(int d, const ServeShape &s, const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_f32(int d, int pieces, const ServeArgs &a, hipStream_t st);
hipError_t launch_serve_combine(int dtype, int d, const ServeArgs &a, hipStream_t st);

// The plan, blocks that are partly filled and a second pass over all rows cost 5 to 9 us, and what a group's requests read of one prefix comes out of the
// caches: below these sizes every request reads its own.  bf16, shared and not, us: 8 of 2,100 tokens (34 MB) 19.0 and 13.1; 4 of 8,500 (70 MB) 22.6 and
// 17; 8 of 8,300 (137 MB) 23.5 and 19.2, with four query heads and one KV head 22.3 and 18.8; 3 chains of 26,300 (161 MB) 37.5 and 29.3; 12 chains of 8,300
// (206 MB) 40.1 and 35.0; 32 of 3,100 (206 MB) 28.5 and 22.2; 16 of 8,300 (275 MB) 26.6 and 26.5, with 8 KV heads of 64 22.7 and 30.7; 64 of 2,200 (288 MB)
// 32.1 and 27.3; 8 of 26,300 (430 MB) 28.9 and 36.2; 32 of them 41.6 and 97.  fp32: 4 of 2,060 (34 MB) 21.5 and 21.3; 8 (68 MB) 22.5 and 26.4.
// Over 8 bits the reads are cheaper and the keys not: what the rest costs goes by (token, KV head) rows.  Sharing begins at 1 Mi of them where requests have up
// to 16 rows and tables for more than 1,536 tokens (fp32: 16 MiB), at 640 Ki beyond 32 rows.  us shared and not; up to 16 rows, heads of 64: 28 and 4 heads, 8 of
// 25,500 (100 MiB, 0.8 Mi rows) 24.3 and 24.5, 64 of 3,100 27.1 and 24.8, 8 of 33,200 (130 MiB, 1.04 Mi) 26.8 and 30.5, 64 of 4,000 28.9 and 29.1; 32 and 8,
// 24 of 5,400 (130 MiB) 23.1 and 29.6, 128 of 900 31.2 and 22.4; heads of 128, 64 of 2,900 (190 MiB, 0.76 Mi) 32.5 and 29.1.  56 rows, heads of 128, 17,000
// tokens: 6 requests 46.7 and 39.6, 8 46.2 and 45.9, 10 (169 MiB, 676 Ki) 49.7 and 51.2, 11 49.7 and 59.2, 12 50.4 and 59.9; heads of 64, 32 of 5,000 (80 MiB)
// 37.8 and 38.5, of 6,300 39.8 and 45.0.  17 to 32 rows, 32 and 8 heads of 64, 12 of 13,500 (160 MiB) 45.5 and 47.3, of 128, 32 of 3,000 (204 MiB) 44.6 and 42.2:
// as bf16.  fp32, 28 and 4 heads of 128, 8 of 1,500 (12 MiB) 21.7 and 22.2, of 2,200 (18 MiB) 22.2 and 27.9; 6 of 2,900, 56 rows, 49.9 and 44.9.
bool serve_shares(int dtype, bool eight, int d, int Hkv, int B, int64_t capacity, int64_t rows) {
  const bool f32 = dtype == SPARROW_F32;
  const int64_t tokens = B * capacity, bytes = 2ll * Hkv * d * (eight ? 1 : f32 ? 4 : 2), kv_rows = tokens * Hkv;
  if (tokens > (f32 ? 32ll << 20 : 200ll << 20) / bytes) return true;
  if (!eight) return false;
  if (f32) return rows <= 16 && tokens > (16ll << 20) / bytes;
  return rows > 32 ? kv_rows > 640 << 10 : rows <= 16 && capacity > 1536 && kv_rows > 1 << 20;
}

ServeShape serve_shape(int dtype, int d, int Hq, int Hkv, int B, int G, int64_t n_rows, int max_new, int64_t capacity) {
  ServeShape s;
  const bool f32 = dtype == SPARROW_F32;
  const int g = Hq / Hkv;
  const int64_t most = std::min<int64_t>(max_new, n_rows) * g;                 // rows of a request, at most
  const int64_t of_item = G > 0 ? n_rows * g : most;                           // of an item
  s.rows = of_item <= 16 ? 16 : f32 || of_item <= 64 ? 64 : 256;
  // every item ends in a block of its own, not all of it filled
  const int64_t blocks = (most <= s.rows ? 0 : n_rows * g / s.rows) + B + (G > 0 ? n_rows * g / s.rows + G : 0);
  // Single tokens: the fewer (request, KV head) pairs, the fewer and larger the workgroups, and the fewer pieces there are to put together.  8 bits, heads of
  // 128, contexts of up to 8,000, us by workgroups of 8, 4 and 2: 32 pairs 18.2, 19.3, 19.0; 52 pairs 23.7, 23.0, 23.5; 160 pairs 58, 45.6, 46.1; 192 pairs
  // 61, 55.0, 54.0; 256 pairs 68, 67.5, 65.5.
  s.waves = B * Hkv <= 48 ? 8 : B * Hkv < 192 ? 4 : 2;
  const int at_once = f32 ? (d == 128 ? 512 : 1024) : G == 0 && s.rows == 16 ? 2048 / s.waves : 256;       // workgroups
  s.round = std::max(at_once / Hkv, 1);
  s.ways = 1;
  if (G > 0) {
    // Two rounds of pieces beside the blocks, one of which every request has: the plan tries to cut some 0.5 to 2.4 rounds off.  us where the blocks were counted
    // among the four rounds, and now, single tokens over a shared 26,112, heads of 128, bf16: 28 and 4 heads, 224 requests 152 and 128, 240 517 and 134,
    // 256 516 and 139; 32 and 8, 112 92 and 92, 124 512 and 95, 256 517 and 172; 32 of each, 32 404 and 117.  (Half a round: 256 over 8 bits 143 -> 151.)
    s.slots = (int)std::max<int64_t>(4 * s.round, blocks + 2 * s.round);
  } else if (most <= s.rows) {
    s.round = std::max(s.round, 2 * B);                    // (256 of up to 3,000 tokens 99.5 us, of B + 1 pieces 110, of 4 B 104)
    // Requests of up to 512 tokens (fp32: 128), 1,024 where they fill half of the chip, in one piece each and without a second pass, by what the tables
    // hold.  8 bits, four KV heads of 128, us in one piece and cut: 8 of 500 tokens 9.8 and 12.3, of 1,000 12.5 and 11.5; 40 of 500 11.0 and 15.0, of 1,000
    // 15.5 and 18.4, of 1,500 20.5 and 21.8; 128 of 1,000 30.8 and 33.6.
    s.slots = capacity <= (f32 ? 128 : B * Hkv < 128 ? 512 : 1024) ? 0 : s.round;
  } else {
    // Cut where the blocks fill two thirds of the chip at most; two rounds of pieces if they end sooner.  8 bits over 26,112 tokens, four KV heads of 128, us
    // cut and not: 1,000 new tokens 357 and 644, 1,500 511 and 645, 1,700 694 and 645.  Nothing is cut off two tiles: 100 over 100 21.7 and 19.3, with heads
    // of 64 18.3 and 11.4; 75 over 300 23.3 and 23.9, 17.9 and 18.9.
    // A round of pieces at least beside the blocks, one of which every request has.  us where those took the place of the chunk's pieces, and now, a chunk of
    // 512 over 26,112 beside single tokens over up to 4,000, 8 bits, heads of 128: 28 and 4 heads, 63 of them 203 and 207, 95 322 and 233, 109 614 and 233,
    // 255 614 and 300; 32 and 8, 32 243 and 244, 47 322 and 260, 63 612 and 270, 255 615 and 430; beside 119 chains of 3, bf16, 514 and 310.
    const int64_t filled = (n_rows * g + s.rows - 1) / s.rows;
    s.ways = 3;
    s.slots = capacity > 128 && 3 * filled <= 2 * s.round ? (int)std::max<int64_t>(2 * s.round, blocks + s.round) : 0;
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
