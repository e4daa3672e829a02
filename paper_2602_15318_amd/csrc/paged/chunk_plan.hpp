// Which piece of the batch a workgroup of the chunk attention takes.  Lengths live on the device, so the workgroups of the first pass work the
// plan out themselves, each the same one: a wavefront holds a request per lane (and register, above 64 requests).  The second pass, another
// kernel, must not depend on its floating-point operations coming out the same there: the workgroup of a request's first piece leaves
// the request's part of the plan in the workspace.
//
// A row is a (new token, query head of the group) pair; the rows of a request and KV head are cut into blocks, a
// block's keys into pieces of T tokens at most, T as small as it may be for the sum over the blocks of ceil(length / T) to be at
// most N, the pieces per KV head that the chip holds at once, or twice that if two rounds of shorter pieces end sooner.  Blocks are not cut
// at all where N is not above their number U.
#pragma once
#include "paged.hpp"

namespace sparrow {

template <int kCtrl, int kRows> __device__ __forceinline__ int dpp_from(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xF, false);
}
// Inclusive sum over the lanes of a wavefront, on the vector ALU
__device__ __forceinline__ int wave_scan(int v) {
  v += dpp_from<0x111, 0xF>(v);          // row_shr 1, 2, 4, 8: within each row of 16 lanes
  v += dpp_from<0x112, 0xF>(v);
  v += dpp_from<0x114, 0xF>(v);
  v += dpp_from<0x118, 0xF>(v);
  v += dpp_from<0x142, 0xA>(v);          // row_bcast 15, 31: the rows before
  v += dpp_from<0x143, 0xC>(v);
  return v;
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Weights of a row are 2^((score - m) * scale): about m, the largest score so far or one up to kSlack less, unscaled.  The difference comes first:
// about a scaled and rounded point the largest weight would be 2 to what the rounding took off, infinite or 0 once half a step
// of the point passes 128.  A row that has seen nothing stands at the lowest finite score.
constexpr float kNothingSeen = -3.402823466e38f;
constexpr float kSlack = 8.0f;            // log2 units
// What weights about `from` are multiplied by to stand about `to`
__device__ __forceinline__ float factor(float from, float to, float scale_log2) { return fast_exp2((from - to) * scale_log2); }
// m * scale, finite
__device__ __forceinline__ float scaled(float m, float scale_log2) { return fminf(fmaxf(m * scale_log2, kNothingSeen), -kNothingSeen); }
// Natural logarithm of a sum of weights l about m, the scaled m to twice fp32's bits
__device__ __forceinline__ float log_sum(float m, float scale_log2, float l) {
  const float r = scaled(m, scale_log2);
  return (r + (fmaf(m, scale_log2, -r) + fast_log2(l))) * kLn2;
}

struct Request {
  int row0, n_all, n, L, past;     // first row; new tokens; those computed; tokens in the cache; position of the first new one
};
__device__ __forceinline__ Request request_of(const ChunkArgs &a, int b) {
  Request r;
  const int c0 = min(max(a.cu_new[b], 0), a.n_rows), c1 = min(max(a.cu_new[b + 1], 0), a.n_rows), kv = max(a.kv_len[b], 0);
  r.row0 = c0;
  r.n_all = max(c1 - c0, 0);
  r.n = min(r.n_all, a.max_new);
  r.L = min(kv, a.table_width << a.page_shift);
  r.past = kv - r.n_all;
  return r;
}

// floor(x / y) for 0 <= x < 2^31, y >= 1 and a quotient below 2^22
__device__ __forceinline__ int quotient(int x, int y, float inv_y) {
  int q = (int)((float)x * inv_y);
  const int r = x - q * y;
  return r < 0 ? q - 1 : r >= y ? q + 1 : q;
}
__device__ __forceinline__ int quotient(int x, int y) {
  return __builtin_amdgcn_readfirstlane(quotient(x, y, __builtin_amdgcn_rcpf((float)y)));
}

// Blocks of the rows of n new tokens
__device__ __forceinline__ int blocks_of(const ChunkArgs &a, int n) {
  return (int)(((int64_t)n * a.g + (1 << a.block_shift) - 1) >> a.block_shift);
}

struct Piece {
  Request rq;
  int b, block, n_blocks, split, n_splits, first, t0, t1;    // first: number of the request's first piece
};
constexpr int kMaxPerLane = SPARROW_MAX_PAGED_BATCH / 64;
constexpr int kGrain = 64;                                    // pieces are whole multiples of this many tokens

struct Plan {
  int T, n_blocks[kMaxPerLane], n_splits[kMaxPerLane], end[kMaxPerLane];
  Request rq[kMaxPerLane];
};
// Pieces of a request's blocks.  In blocks of 256 rows and heads of 128, a request whose rows leave half of the wavefronts idle gets pieces of
// twice the length: a tile of its takes half as long (chunk of 512 beside 16 single tokens, contexts of up to 8,192 tokens: 130 -> 110
// us; with heads of 64 the softmax of one wavefront sets the pace either way, 82 -> 97).
__device__ __forceinline__ int splits_of(const ChunkArgs &a, const Request &r, int T) {
  if (a.block_shift == 8 && a.d == 128 && r.n <= 128 / a.g) T *= 2;
  return quotient(max(r.L - 1, 0), T, __builtin_amdgcn_rcpf((float)T)) + 1;
}
// Lane l's requests l, l + 64, ...
__device__ __forceinline__ Plan make_plan(const ChunkArgs &a, int lane) {
  Plan p;
  int blocks = 0;
  float weight = 0.f;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    p.n_blocks[k] = 0;
    p.rq[k] = {0, 0, 0, 0, 0};
    if (64 * k < a.B) {
      if (64 * k + lane < a.B) {
        p.rq[k] = request_of(a, 64 * k + lane);
        p.n_blocks[k] = blocks_of(a, p.rq[k].n);
      }
      blocks += min(p.n_blocks[k], a.slots);               // (offsets that overlap may promise any number)
      weight += (float)p.n_blocks[k] * (float)p.rq[k].L;
    }
  }
  const int U = lane_value(wave_scan(blocks), 63);
  const float W = wave_sum_valu(weight);
  p.T = 1 << 29;
  int best = 1 << 30;
  for (int round = 1; round * a.round <= a.slots; ++round) {
    const int N = round * a.round;
    if (N <= U) continue;
    // T1 = W / (N - U) always fits; the smallest that does lies between W / N and it, and is looked for where they differ by much (N
    // below 8 U.  Never: chunk of 512 beside 16 single tokens 107 -> 126 us, of 300 beside 4 51 -> 59, twelve chains 33.6 -> 32.9; always: eight single
    // tokens 19.6 -> 19.9, chunk of 256 over 8,192 53.3 -> 52.4).
    // (the factor: the sum is off by 2^-16 at most)
    const auto grains = [&](float t) { return (min((int)(t * (1.f + 0x1p-14f)), 1 << 28) + kGrain) / kGrain; };
    int hi = grains(W / (float)(N - U));
    if (N < 8 * U) {
      int lo = max(grains(W / (float)N) - 1, 0);             // (lo: too small, or not tried)
      for (int step = 0; step < 6 && hi - lo > 1; ++step) {
        const int mid = (lo + hi) >> 1;
        int sum = 0;
#pragma unroll
        for (int k = 0; k < kMaxPerLane; ++k)
          if (64 * k < a.B) sum += min(p.n_blocks[k], a.slots) * splits_of(a, p.rq[k], mid * kGrain);
        if (lane_value(wave_scan(sum), 63) <= N) hi = mid;
        else lo = mid;
      }
    }
    const int cost = round * (hi + (a.block_shift == 8 ? 2 : 4));    // (so many grains a piece's beginning and end take: 0 to 4
                                                                     // make no difference, 8 one round of an fp32 chunk, 214 -> 259 us)
    if (cost < best) {
      best = cost;
      p.T = hi * kGrain;
    }
  }
  int before = 0;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k) {
    p.n_splits[k] = 1;
    p.end[k] = before;
    if (64 * k < a.B) {
      p.n_splits[k] = splits_of(a, p.rq[k], p.T);
      p.end[k] = before + wave_scan(p.n_blocks[k] * p.n_splits[k]);
      before = lane_value(p.end[k], 63);
    }
  }
  return p;
}

// Piece number `idx` of a KV head; false: there are not that many.  Blocks count down: the last, whose rows see most, come first.
__device__ __forceinline__ bool find_piece(const ChunkArgs &a, int idx, int lane, Piece *out) {
  const Plan p = make_plan(a, lane);
  Piece q;
  q.b = -1;
  int end = 0;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k)
    if (q.b < 0 && 64 * k < a.B) {
      const unsigned long long m = __builtin_amdgcn_ballot_w64(p.end[k] > idx);
      if (m != 0ull) {
        const int l = __builtin_ctzll(m);
        q.b = 64 * k + l;
        q.n_blocks = lane_value(p.n_blocks[k], l);
        q.n_splits = lane_value(p.n_splits[k], l);
        end = lane_value(p.end[k], l);
        q.rq = {lane_value(p.rq[k].row0, l), lane_value(p.rq[k].n_all, l), lane_value(p.rq[k].n, l), lane_value(p.rq[k].L, l),
                lane_value(p.rq[k].past, l)};
      }
    }
  if (q.b < 0) return false;
  q.first = end - q.n_blocks * q.n_splits;
  q.split = quotient(idx - q.first, q.n_blocks);
  q.block = q.n_blocks - 1 - (idx - q.first - q.split * q.n_blocks);
  if (q.block < 0 || q.block >= q.n_blocks || q.split < 0 || q.split >= q.n_splits) return false;    // (sums of such offsets that wrapped)
  const int each = (quotient(q.rq.L + q.n_splits - 1, q.n_splits) + kGrain - 1) / kGrain * kGrain;
  q.t0 = min(q.rq.L, q.split * each);
  q.t1 = min(q.rq.L, q.t0 + each);
  if (a.plan && idx == q.first && blockIdx.x == 0 && threadIdx.x == 0) {
    a.plan[2 * q.b] = q.first;
    a.plan[2 * q.b + 1] = q.n_splits;
  }
  *out = q;
  return true;
}

}  // namespace sparrow
