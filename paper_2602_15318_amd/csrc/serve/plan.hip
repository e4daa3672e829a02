// The plan of a batch in groups (serve_plan.hpp), worked out once: every piece of a KV head, and what the second pass needs.  One workgroup; a thread takes
// a request, then a wavefront ways of cutting, then a thread pieces.  Measured 6 us a call of 32 requests; by every workgroup of the attention itself, which
// takes one compute unit each, it cost some 4 us a round of them.
#include "serve_plan.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kMaxItems = SPARROW_MAX_PREFIX_GROUPS + SPARROW_MAX_PAGED_BATCH, kWays = 8;

struct Plan {                     // in LDS: groups first, then requests
  int row0[kMaxItems], n[kMaxItems];   // first row of the batch; rows (tokens)
  int past[kMaxItems];                 // position of the first, past every key where all see all
  int from[kMaxItems], to[kMaxItems];  // keys
  int of[kMaxItems];                   // a request's group (-1: shares nothing); the request through whose table a prefix is read
  int blocks[kMaxItems], splits[kMaxItems], end[kMaxItems];      // pieces of a block; pieces of all items up to this one
  int cu[SPARROW_MAX_PAGED_BATCH + 1], start[SPARROW_MAX_PREFIX_GROUPS + 1];
  int least[SPARROW_MAX_PREFIX_GROUPS], first[SPARROW_MAX_PREFIX_GROUPS], with_rows[SPARROW_MAX_PREFIX_GROUPS];
  float cost[kWays];
  int T[kWays];
};
// T: of kWays ways to cut the longest item that which should end first, among those whose pieces the workspace holds.  In grains of 64 tokens of an item of
// more than 64 rows (kTail: of others), each piece with its beginning and end (kMany: its partial output is up to 128 KB; kFew): the mean work of a
// workgroup's place and some of the longest piece, or the rounds of pieces of more than half of that, whichever is more; and the second pass, which reads what
// all leave (kCombine).  Fitted to nine batches at seven lengths each: that which it takes is 3.5 % behind the best of the seven at most.
__device__ __forceinline__ int best_piece(const ServeArgs &a, Plan *p, int items) {
  constexpr float kMany = 10.f, kFew = 3.f, kTail = 0.5f, kRest = 0.15f, kCombine = 0.006f;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float weight = 0.f, longest = 0.f;
  int blocks = 0;
  for (int i = lane; i < items; i += 64) {
    const float len = (float)(p->to[i] - p->from[i]);
    blocks += min(p->blocks[i], a.slots);                  // (offsets that overlap may promise any number)
    weight += (float)p->blocks[i] * len;
    longest = fmaxf(longest, p->blocks[i] > 0 ? len : 0.f);
  }
  const float W = wave_sum_valu(weight) * (1.f / kGrain), inv_round = 1.f / (float)a.round;
  const int L = max(((int)wave_max_valu(longest) + kGrain - 1) / kGrain, 1), U = lane_value(wave_scan(blocks), 63);
  int s = max(min((int)(0.5f * (float)a.round / fmaxf(W / (float)L, 1.f)), L), 1);
  for (int way = 0; way < w; ++way) s += max(s / 4, 1);
  if (w < kWays) {
    const int T = quotient(L + s - 1, s) * kGrain;
    const float inv_t = __builtin_amdgcn_rcpf((float)T);
    const auto pieces_of = [&](int i) { return quotient(max(p->to[i] - p->from[i] - 1, 0), T, inv_t) + 1; };
    const auto end_of = [&](int i) { return p->n[i] * a.g > 64 ? kMany : kFew; };
    const auto time_of = [&](int i, int splits) {
      return end_of(i) + (p->n[i] * a.g > 64 ? 1.f : kTail) * (1.f / kGrain) * (float)(p->to[i] - p->from[i]) * __builtin_amdgcn_rcpf((float)splits);
    };
    float ends = 0.f, sum = 0.f, most = 0.f, big = 0.f;
    int count = 0;
    for (int i = lane; i < items; i += 64) {
      const int splits = pieces_of(i), pieces = min(p->blocks[i], a.slots) * splits;
      const float time = time_of(i, splits);
      count += pieces;
      ends += (float)pieces * end_of(i);
      sum += (float)pieces * time;
      most = fmaxf(most, pieces > 0 ? time : 0.f);
    }
    most = wave_max_valu(most);
    for (int i = lane; i < items; i += 64) {
      const int splits = pieces_of(i);
      big += 2.f * time_of(i, splits) > most ? (float)(min(p->blocks[i], a.slots) * splits) : 0.f;
    }
    const int N = lane_value(wave_scan(count), 63);
    const float rounds = __builtin_ceilf(wave_sum_valu(big) * inv_round);
    const float cost = fmaxf(wave_sum_valu(sum) * inv_round + kRest * most, rounds * most) + kCombine * (float)a.Hkv * wave_sum_valu(ends);
    if (lane == 0) {
      p->cost[w] = N > a.slots && N > U ? 3.4e38f : cost;              // (uncut blocks always fit, and half a round more: the first way)
      p->T[w] = T;
    }
  }
  __syncthreads();
  const float mine = p->cost[lane % kWays], best = -wave_max_valu(-mine);
  const int T = p->T[lane % kWays];
  return best < 3.4e38f ? lane_value(T, __builtin_ctzll(__builtin_amdgcn_ballot_w64(mine == best))) : 1 << 29;
}

__global__ void __launch_bounds__(kThreads) serve_plan_kernel(ServeArgs a) {
  static_assert(kThreads >= SPARROW_MAX_PAGED_BATCH && kWaves >= kWays, "a thread a request, a wavefront a way");
  __shared__ Plan plan;
  Plan *const p = &plan;
  const int tid = threadIdx.x, lane = tid & 63, most = a.table_width << a.page_shift, items = a.G + a.B;
  int c0 = 0, c1 = 0, kv = 0, g = -1;
  if (tid < a.B) {
    c0 = min(max(a.cu_new[tid], 0), a.n_rows);
    c1 = min(max(a.cu_new[tid + 1], 0), a.n_rows);
    kv = max(a.kv_len[tid], 0);
  }
  const int n = max(c1 - c0, 0), past = kv - n;
  int from = 0;
  if (tid <= a.G) p->start[tid] = min(max(a.group_start[tid], 0), a.B);
  if (tid < a.G) {
    p->least[tid] = min(max(a.prefix_len[tid], 0), most);
    p->first[tid] = a.B;
    p->with_rows[tid] = 0;
  }
  if (tid < a.B) p->cu[tid] = c0;
  if (tid == a.B - 1) p->cu[a.B] = c1;
  __syncthreads();
  if (tid < a.B) {
    for (int i = 0; i < a.G; ++i)
      if (tid >= p->start[i] && tid < p->start[i + 1]) g = i;
    if (g >= 0 && n > 0) {
      atomicMin(&p->least[g], past);
      atomicMin(&p->first[g], tid);
      atomicAdd(&p->with_rows[g], 1);
    }
  }
  __syncthreads();
  // what requests without rows, or a single one, have in common is not used
  const auto shared = [&](int i) { return p->with_rows[i] > 1 ? max(p->least[i], 0) & -64 : 0; };
  if (g >= 0) {
    from = min(shared(g), min(kv, most));
    if (from == 0) g = -1;
  }
  if (tid < a.G) {
    const int r0 = p->cu[p->start[tid]], r1 = p->cu[p->start[tid + 1]], P = shared(tid);
    p->row0[tid] = r0;
    p->n[tid] = P > 0 ? max(r1 - r0, 0) : 0;
    p->past[tid] = most;
    p->from[tid] = 0;
    p->to[tid] = P;
    p->of[tid] = p->first[tid];
    p->blocks[tid] = serve_blocks(a, p->n[tid]);
  }
  if (tid < a.B) {
    const int i = a.G + tid;
    p->row0[i] = c0;
    p->n[i] = min(n, a.max_new);
    p->past[i] = past;
    p->from[i] = from;
    p->to[i] = min(kv, most);
    p->of[i] = g;
    p->blocks[i] = serve_blocks(a, p->n[i]);
  }
  __syncthreads();
  const int T = best_piece(a, p, items);
  const float inv_t = __builtin_amdgcn_rcpf((float)T);
  // every wavefront the same, so that none has to wait
  int total = 0;
  for (int i0 = 0; i0 < items; i0 += 64) {
    const int i = i0 + lane, splits = i < items ? quotient(max(p->to[i] - p->from[i] - 1, 0), T, inv_t) + 1 : 0;
    const int end = total + wave_scan(i < items ? p->blocks[i] * splits : 0);
    if (i < items) {
      p->splits[i] = splits;
      p->end[i] = end;
    }
    total = lane_value(end, 63);
  }
  __syncthreads();
  if (tid == 0) *a.n_pieces = min(total, a.slots);
  for (int idx = tid; idx < min(total, a.slots); idx += kThreads) {
    int i = 0, last = items - 1;                           // the first item that ends behind the piece
    while (i < last) {
      const int mid = (i + last) >> 1;
      if (p->end[mid] > idx) last = mid;
      else i = mid + 1;
    }
    const int nb = max(p->blocks[i], 1), ns = p->splits[i], local = idx - (p->end[i] - p->blocks[i] * ns);
    const int split = quotient(local, nb, __builtin_amdgcn_rcpf((float)nb)), of = p->of[i];
    ServePiece q{};
    q.it = {p->row0[i], p->n[i], p->past[i], p->from[i], p->to[i], i < a.G ? min(max(of, 0), a.B - 1) : i - a.G};
    q.block = nb - 1 - (local - split * nb);
    q.direct = i >= a.G && of < 0 && ns == 1;
    // (sums of overlapping offsets that wrapped: a piece without rows)
    if (local < 0 || q.block < 0 || q.block >= nb || split < 0 || split >= ns) q.it.n = 0;
    cut(&q, split, ns);
    a.pieces[idx] = q;
  }
  if (tid < a.B) {
    const int i = a.G + tid;
    ServeLeft left = {p->end[i] - p->blocks[i] * p->splits[i], p->splits[i], 0, 0, 0, 0, {0, 0}};
    if (g >= 0) {
      left.group_splits = p->splits[g];
      left.group_blocks = p->blocks[g];
      left.group_first = p->end[g] - p->blocks[g] * p->splits[g];
      left.group_row0 = p->row0[g];
    }
    a.left[tid] = left;
  }
}

}  // namespace

hipError_t launch_serve_plan(const ServeArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(serve_plan_kernel, dim3(1), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace sparrow
