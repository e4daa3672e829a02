// Which piece of the batch a workgroup of the attention takes.  As in the chunk attention (../paged/chunk_plan.hpp) lengths live on the device.
//
// An item is a run of the batch's rows and the keys that they share: the prefix of a group with the rows of all its requests, or what a
// request has behind its prefix (everything, where it shares none) with its own rows.  An item's rows (new token, query head of the group of
// heads) are cut into blocks, a block's keys into pieces of T tokens at most.  A prefix that is used is a whole number of 64 tokens, so that all
// tiles of keys begin on such a border and never cross a page within 16 tokens; what is left of it is read request by request.
//
// Without groups every workgroup works the same plan out itself, and that of a request's first piece leaves the second pass what it needs.  With
// groups the plan is more work, and there are several rounds of workgroups: a small kernel of its own (plan.hip) writes every piece down.
#pragma once
#include "../paged/chunk_plan.hpp"
#include "serve.hpp"

namespace sparrow {

struct ServeItem { int row0, n, past, from, to, table; };  // first row of the batch; rows (tokens); position of the first, past every key where all see
                                                           // all; keys; row of the block table
struct ServePiece {
  ServeItem it;
  int block, t0, t1;
  int direct;            // the rows' only piece: the output itself
  int unused[2];
};
static_assert(sizeof(ServePiece) == 48, "read 16 bytes at a time");
// What the second pass reads of a request: its first piece and pieces per block; those of its group's prefix (no pieces: it shares none), the
// group's first row and blocks
struct ServeLeft { int first, n_splits, group_first, group_splits, group_row0, group_blocks, unused[2]; };
static_assert(sizeof(ServeLeft) == 32, "read 16 bytes at a time");

__device__ __forceinline__ int serve_blocks(const ServeArgs &a, int n) {
  return (int)(((int64_t)n * a.g + (1 << a.block_shift) - 1) >> a.block_shift);
}
// Piece `split` of n_splits of an item's keys
__device__ __forceinline__ void cut(ServePiece *q, int split, int n_splits) {
  const int each = (quotient(q->it.to - q->it.from + n_splits - 1, n_splits, __builtin_amdgcn_rcpf((float)n_splits)) + kGrain - 1) / kGrain * kGrain;
  q->t0 = min(q->it.to, q->it.from + split * each);
  q->t1 = min(q->it.to, q->t0 + each);
}

// Without groups; piece number `idx` of a KV head, false: there are not that many.  Blocks count down: the last, whose rows see most, come first.  T is the
// smallest for which the heavy pieces, those of more than 16 rows where there are such, are not more than N, of a.ways ways that which should end first: one
// round of pieces, two, or one beside the blocks (where those alone take half a round: short requests fill the places, the time is the mean work and
// then the longest piece); a piece's beginning and end take about `extra` grains.  Light ones end soon and fit in between: with all of them counted, batches of a chunk and single
// tokens took 82 us instead of 74 (777 + 8 tokens, heads of 64) and 123 instead of 104 (512 + 16, heads of 128).
__device__ __forceinline__ bool serve_find_piece(const ServeArgs &a, int idx, ServePiece *out) {
  const int lane = threadIdx.x & 63, most = a.table_width << a.page_shift;
  ServeItem rq[kMaxPerLane];                               // lane l's requests l, l + 64, ...
  int n_blocks[kMaxPerLane], blocks = 0, heavy = 0;        // heavy: of more than 16 rows (blocks of 16: all)
  float weight = 0.f, heavy_weight = 0.f;
  const auto is_heavy = [&](const ServeItem &r) { return a.block_shift == 4 || r.n * a.g > 16; };
  const auto splits_of = [](const ServeItem &r, int T) { return quotient(max(r.to - 1, 0), T, __builtin_amdgcn_rcpf((float)T)) + 1; };
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    const int b = 64 * k + lane;
    rq[k] = {0, 0, 0, 0, 0, b};
    n_blocks[k] = 0;
    if (64 * k < a.B) {
      if (b < a.B) {
        const int c0 = min(max(a.cu_new[b], 0), a.n_rows), c1 = min(max(a.cu_new[b + 1], 0), a.n_rows), kv = max(a.kv_len[b], 0);
        rq[k].row0 = c0;
        rq[k].n = min(max(c1 - c0, 0), a.max_new);
        rq[k].past = kv - max(c1 - c0, 0);
        rq[k].to = min(kv, most);
        n_blocks[k] = serve_blocks(a, rq[k].n);
      }
      blocks += min(n_blocks[k], a.slots);                 // (offsets that overlap may promise any number)
      weight += (float)n_blocks[k] * (float)rq[k].to;
      if (is_heavy(rq[k])) {
        heavy += min(n_blocks[k], a.slots);
        heavy_weight += (float)n_blocks[k] * (float)rq[k].to;
      }
    }
  }
  const int U = lane_value(wave_scan(blocks), 63), H = lane_value(wave_scan(heavy), 63), extra = a.block_shift == 8 ? 2 : 4;
  const float W = wave_sum_valu(weight), V = wave_sum_valu(heavy_weight);
  int T = 1 << 29, best = 1 << 30;
  // (the mean work here, by a reciprocal: with a division in the loop a chain of 8 over 3,000 in fp32 took 30.0 us instead of 29.6, without a third way 29.3)
  const int ways = 2 * H > a.round ? a.ways : min(a.ways, 2), mean = (int)(V * __builtin_amdgcn_rcpf((float)(kGrain * a.round)));
  for (int way = 1; way <= ways && U < a.slots; ++way) {
    const int N = way < 3 ? way * a.round : H + a.round;
    if (N <= H) continue;
    const auto grains = [&](float t) { return (min((int)(t * (1.f + 0x1p-14f)), 1 << 28) + kGrain) / kGrain; };
    int hi = max(grains(V / (float)(N - H)), grains(W / (float)(a.slots - U)));           // always fits
    if (N < 8 * H) {
      int lo = max(grains(V / (float)N) - 1, 0);           // (too small, or not tried)
      for (int step = 0; step < 6 && hi - lo > 1; ++step) {
        const int mid = (lo + hi) >> 1;
        int sum = 0, of_heavy = 0;                         // (of them: 0 where all are)
#pragma unroll
        for (int k = 0; k < kMaxPerLane; ++k)
          if (64 * k < a.B) {
            const int pieces = min(n_blocks[k], a.slots) * splits_of(rq[k], mid * kGrain);
            sum += pieces;
            if (H < U) of_heavy += is_heavy(rq[k]) ? pieces : 0;
          }
        if (lane_value(wave_scan(sum), 63) <= (H < U ? a.slots : N) && (H == U || lane_value(wave_scan(of_heavy), 63) <= N)) hi = mid;
        else lo = mid;
      }
    }
    const int cost = way < 3 ? way * (hi + extra) : hi + extra + mean;
    if (cost < best) {
      best = cost;
      T = hi * kGrain;
    }
  }
  int before = 0, b = -1;
  ServePiece q;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k)
    if (b < 0 && 64 * k < a.B) {
      const int splits = splits_of(rq[k], T), end = before + wave_scan(n_blocks[k] * splits);
      before = lane_value(end, 63);
      const unsigned long long m = __builtin_amdgcn_ballot_w64(end > idx);
      if (m != 0ull) {
        const int l = __builtin_ctzll(m);
        b = 64 * k + l;
        q.it = {lane_value(rq[k].row0, l), lane_value(rq[k].n, l), lane_value(rq[k].past, l), 0, lane_value(rq[k].to, l), b};
        const int nb = lane_value(n_blocks[k], l), ns = lane_value(splits, l), first = lane_value(end, l) - nb * ns;
        const int split = quotient(idx - first, nb);
        q.block = nb - 1 - (idx - first - split * nb);
        q.direct = ns == 1;
        if (q.block < 0 || q.block >= nb || split < 0 || split >= ns) return false;       // (sums of such offsets that wrapped)
        cut(&q, split, ns);
        if (a.left && idx == first && blockIdx.x == 0 && threadIdx.x == 0) a.left[b] = {first, ns, 0, 0, 0, 0, {0, 0}};
      }
    }
  if (b < 0) return false;
  q.t0 = __builtin_amdgcn_readfirstlane(q.t0);
  q.t1 = __builtin_amdgcn_readfirstlane(q.t1);
  *out = q;
  return true;
}

// The piece of this workgroup: with groups as written down.
__device__ __forceinline__ bool serve_piece(const ServeArgs &a, int idx, ServePiece *out) {
  if (a.G == 0) return serve_find_piece(a, idx, out);
  typedef const int __attribute__((address_space(4))) *Ints;        // through the scalar cache
  if (idx >= *(Ints)(uintptr_t)a.n_pieces) return false;
  const Ints from = (Ints)(uintptr_t)(a.pieces + idx);
  ServePiece q;
  q.it = {from[0], from[1], from[2], from[3], from[4], from[5]};
  q.block = from[6];
  q.t0 = from[7];
  q.t1 = from[8];
  q.direct = from[9];
  *out = q;
  return q.it.n > 0;
}

}  // namespace sparrow
