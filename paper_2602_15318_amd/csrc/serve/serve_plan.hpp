// Which piece of the batch a workgroup of the attention takes.  As in the chunk attention (../paged/chunk_plan.hpp) lengths live on the device and
// every workgroup works the same plan out itself; the second pass reads what the workgroup of a request's first piece has left of it.
//
// An item is a run of the batch's rows and the keys that they share: the prefix of a group with the rows of all its requests, or what a
// request has behind its prefix (everything, where it shares none) with its own rows.  An item's rows (new token, query head of the group of
// heads) are cut into blocks, a block's keys into pieces of T tokens at most.  A prefix that is used is a whole number of 64 tokens, so that all
// tiles of keys begin on such a border and never cross a page within 16 tokens; what is left of it is read request by request.
#pragma once
#include "../paged/chunk_plan.hpp"
#include "serve.hpp"

namespace sparrow {

struct ServeItem {
  int row0, n, past;     // first row of the batch; rows (tokens); position of the first, past every key where all see all
  int from, to;          // keys
  int table;             // row of the block table
};
struct ServePiece {
  ServeItem it;
  int block, n_blocks, n_splits, t0, t1;
  bool direct;           // the rows' only piece: the output itself
};
// Lane l's requests l, l + 64, ... and its group l
struct ServePlan {
  ServeItem rq[kMaxPerLane], group;
  int n_blocks[kMaxPerLane], n_splits[kMaxPerLane], end[kMaxPerLane], of[kMaxPerLane];      // of: the request's group, -1: shares nothing
  int group_blocks, group_splits, group_end;
};

__device__ __forceinline__ int serve_blocks(const ServeArgs &a, int n) {
  return (int)(((int64_t)n * a.g + (1 << a.block_shift) - 1) >> a.block_shift);
}
__device__ __forceinline__ int serve_splits(int len, int T) { return quotient(max(len - 1, 0), T, __builtin_amdgcn_rcpf((float)T)) + 1; }

__device__ __forceinline__ ServePlan serve_plan(const ServeArgs &a, int lane) {
  ServePlan p;
  const int most = a.table_width << a.page_shift;
  p.group = {0, 0, most, 0, 0, 0};
  p.group_blocks = p.group_splits = p.group_end = 0;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    p.rq[k] = {0, 0, 0, 0, 0, 64 * k + lane};
    p.of[k] = -1;
    if (64 * k < a.B && 64 * k + lane < a.B) {
      const int b = 64 * k + lane;
      const int c0 = min(max(a.cu_new[b], 0), a.n_rows), c1 = min(max(a.cu_new[b + 1], 0), a.n_rows), kv = max(a.kv_len[b], 0);
      p.rq[k].row0 = c0;
      p.rq[k].n = max(c1 - c0, 0);                         // (of all; those computed below)
      p.rq[k].past = kv - p.rq[k].n;
      p.rq[k].to = min(kv, most);
    }
  }
  for (int g = 0; g < a.G; ++g) {                          // uniform
    const int s0 = min(max(a.group_start[g], 0), a.B), s1 = min(max(a.group_start[g + 1], 0), a.B);
    int least = min(max(a.prefix_len[g], 0), most), first = -1, with_rows = 0;
#pragma unroll
    for (int k = 0; k < kMaxPerLane; ++k)
      if (64 * k < a.B) {
        const int b = 64 * k + lane;
        const bool in = b >= s0 && b < s1 && p.rq[k].n > 0;
        const unsigned long long m = __builtin_amdgcn_ballot_w64(in);
        if (m != 0ull && first < 0) first = 64 * k + __builtin_ctzll(m);
        with_rows += __builtin_popcountll(m);
        least = in ? min(least, p.rq[k].past) : least;
      }
    const int P = max(__builtin_amdgcn_readfirstlane(wave_min_valu(least)), 0) & -64;
    if (P == 0 || with_rows < 2) continue;
    const int c0 = min(max(a.cu_new[s0], 0), a.n_rows), c1 = min(max(a.cu_new[s1], 0), a.n_rows);
    if (lane == g) {
      p.group = {c0, max(c1 - c0, 0), most, 0, P, first};
      p.group_blocks = serve_blocks(a, p.group.n);
    }
#pragma unroll
    for (int k = 0; k < kMaxPerLane; ++k)
      if (64 * k + lane >= s0 && 64 * k + lane < s1) {
        p.rq[k].from = min(P, p.rq[k].to);
        p.of[k] = g;
      }
  }
  int blocks = min(p.group_blocks, a.slots);               // (offsets that overlap may promise any number)
  float weight = (float)p.group_blocks * (float)p.group.to;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    p.rq[k].n = min(p.rq[k].n, a.max_new);
    p.n_blocks[k] = serve_blocks(a, p.rq[k].n);
    blocks += min(p.n_blocks[k], a.slots);
    weight += (float)p.n_blocks[k] * (float)(p.rq[k].to - p.rq[k].from);
  }
  // T: the smallest for which the pieces are not more than N, whole multiples of kGrain; of one to three rounds of pieces that which should
  // end first.  A piece's beginning and end take about `extra` grains.  With groups the pieces of a call differ much in length and the chip takes them
  // in turn: the mean work of a compute unit and the longest piece.
  const int U = lane_value(wave_scan(blocks), 63);
  const float W = wave_sum_valu(weight);
  const int extra = a.block_shift == 8 ? 2 : 4;
  int T = 1 << 29;
  float best = 3.4e38f;
  for (int round = 1; round * a.round <= a.slots; ++round) {
    const int N = round * a.round;
    if (N <= U) continue;
    const auto grains = [&](float t) { return (min((int)(t * (1.f + 0x1p-14f)), 1 << 28) + kGrain) / kGrain; };
    int hi = grains(W / (float)(N - U));
    int lo = max(grains(W / (float)N) - 1, 0);
    for (int step = 0; step < 6 && hi - lo > 1; ++step) {
      const int mid = (lo + hi) >> 1;
      int sum = min(p.group_blocks, a.slots) * serve_splits(p.group.to, mid * kGrain);
#pragma unroll
      for (int k = 0; k < kMaxPerLane; ++k)
        if (64 * k < a.B) sum += min(p.n_blocks[k], a.slots) * serve_splits(p.rq[k].to - p.rq[k].from, mid * kGrain);
      if (lane_value(wave_scan(sum), 63) <= N) hi = mid;
      else lo = mid;
    }
    const float cost = a.G == 0 ? (float)(round * (hi + extra)) : (W * (1.f / kGrain) + (float)(extra * N)) / (float)a.round + (float)hi;
    if (cost < best) {
      best = cost;
      T = hi * kGrain;
    }
  }
  p.group_splits = serve_splits(p.group.to, T);
  p.group_end = wave_scan(p.group_blocks * p.group_splits);
  int before = lane_value(p.group_end, 63);
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    p.n_splits[k] = 1;
    p.end[k] = before;
    if (64 * k < a.B) {
      p.n_splits[k] = serve_splits(p.rq[k].to - p.rq[k].from, T);
      p.end[k] = before + wave_scan(p.n_blocks[k] * p.n_splits[k]);
      before = lane_value(p.end[k], 63);
    }
  }
  return p;
}

__device__ __forceinline__ ServeItem lane_item(const ServeItem &i, int l) {
  return {lane_value(i.row0, l), lane_value(i.n, l), lane_value(i.past, l), lane_value(i.from, l), lane_value(i.to, l), lane_value(i.table, l)};
}

// What the second pass reads of a request: its first piece and pieces per block; those of its group's prefix (no pieces: it shares none), the
// group's first row and blocks
struct ServeLeft { int first, n_splits, group_first, group_splits, group_row0, group_blocks, unused[2]; };
static_assert(sizeof(ServeLeft) == 32, "read 16 bytes at a time");

// Piece number `idx` of a KV head; false: there are not that many.  Prefixes come first, a request's or group's blocks count down: the last, whose rows
// see most, come first.
__device__ __forceinline__ bool serve_find_piece(const ServeArgs &a, int idx, int lane, ServePiece *out) {
  const ServePlan p = serve_plan(a, lane);
  ServePiece q;
  int end = -1, group = -1, b = -1;
  unsigned long long m = __builtin_amdgcn_ballot_w64(p.group_end > idx);
  if (m != 0ull) {
    const int l = __builtin_ctzll(m);
    q.it = lane_item(p.group, l);
    q.n_blocks = lane_value(p.group_blocks, l);
    q.n_splits = lane_value(p.group_splits, l);
    q.direct = false;
    end = lane_value(p.group_end, l);
  } else {
#pragma unroll
    for (int k = 0; k < kMaxPerLane; ++k)
      if (b < 0 && 64 * k < a.B) {
        m = __builtin_amdgcn_ballot_w64(p.end[k] > idx);
        if (m != 0ull) {
          const int l = __builtin_ctzll(m);
          b = 64 * k + l;
          q.it = lane_item(p.rq[k], l);
          q.n_blocks = lane_value(p.n_blocks[k], l);
          q.n_splits = lane_value(p.n_splits[k], l);
          group = lane_value(p.of[k], l);
          q.direct = q.n_splits == 1 && group < 0;
          end = lane_value(p.end[k], l);
        }
      }
    if (b < 0) return false;
  }
  const int first = end - q.n_blocks * q.n_splits;
  const int split = quotient(idx - first, q.n_blocks);
  q.block = q.n_blocks - 1 - (idx - first - split * q.n_blocks);
  if (q.block < 0 || q.block >= q.n_blocks || split < 0 || split >= q.n_splits) return false;       // (sums of such offsets that wrapped)
  const int each = (quotient(q.it.to - q.it.from + q.n_splits - 1, q.n_splits) + kGrain - 1) / kGrain * kGrain;
  q.t0 = min(q.it.to, q.it.from + split * each);
  q.t1 = min(q.it.to, q.t0 + each);
  if (a.left && b >= 0 && idx == first && blockIdx.x == 0 && threadIdx.x == 0) {
    ServeLeft left = {first, q.n_splits, 0, 0, 0, 0, {0, 0}};
    if (group >= 0) {
      left.group_splits = lane_value(p.group_splits, group);
      left.group_blocks = lane_value(p.group_blocks, group);
      left.group_first = lane_value(p.group_end, group) - left.group_blocks * left.group_splits;
      left.group_row0 = lane_value(p.group.row0, group);
    }
    a.left[b] = left;
  }
  *out = q;
  return true;
}

}  // namespace sparrow
