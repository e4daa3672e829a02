// Block tables and slot maps from request lengths.  One workgroup: what each request gives back and takes is a prefix
// sum over the batch, then the lanes of the workgroup, shared out evenly among the requests, move page ids and write
// the rows.  A call of a decoding step moves a few kilobytes and lasts as long as its round trips to memory (2.8 us for 48 requests of
// eight new tokens).  A request's rows are its own lanes' work, 16 of 48 requests: 31 prompts of up to 1,500 tokens take 11 us, 47 single tokens
// beside a chunk of 8,192 rows 65, 255 of them beside it 259.  More rows than 32,768 are a second launch's, over the whole chip.
#include "paged.hpp"

namespace sparrow {

namespace {

constexpr int kThreads = 1024;
constexpr int kMaxB = SPARROW_MAX_PAGED_BATCH;
constexpr int kOneLaunch = 32768;
static_assert(kMaxB == 256, "four wavefronts scan the batch");

// Inclusive sum over the lanes of a wavefront
__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

template <bool kRows> __global__ void __launch_bounds__(kThreads) page_update_kernel(PageUpdateArgs a) {
  __shared__ int part[3][4], bad_part[4];
  __shared__ int s_old[kMaxB], s_new[kMaxB], s_give[kMaxB], s_take[kMaxB], s_row[kMaxB];   // offsets: exclusive sums
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int ps1 = (1 << a.page_shift) - 1;
  int give = 0, take = 0, add = 0, bad = 0, o = 0, n = 0;
  if (tid < kMaxB) {
    if (tid < a.B) {
      o = a.old_len[tid];
      n = a.new_len[tid];
      const int most = a.table_width << a.page_shift;
      bad = o < 0 || o > most || n < 0 || n > most;
      if (bad) o = n = 0;
      const int held = (o + ps1) >> a.page_shift, need = (n + ps1) >> a.page_shift;
      give = max(held - need, 0);
      take = max(need - held, 0);
      add = max(n - o, 0);
    }
    const int sg = wave_scan(give, lane), st = wave_scan(take, lane), sa = wave_scan(add, lane);
    const bool any = __any(bad);
    if (lane == 63) { part[0][w] = sg; part[1][w] = st; part[2][w] = sa; bad_part[w] = any; }
    s_old[tid] = o; s_new[tid] = n;
    s_give[tid] = sg - give; s_take[tid] = st - take; s_row[tid] = sa - add;
  }
  __syncthreads();
  int tot[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) tot[k] = part[k][0] + part[k][1] + part[k][2] + part[k][3];
  if (tid < kMaxB)
    for (int k = 0; k < w; ++k) { s_give[tid] += part[0][k]; s_take[tid] += part[1][k]; s_row[tid] += part[2][k]; }
  const int R = tot[0], A = tot[1], N = tot[2];
  const int nf = *a.n_free;
  int status = 0;
  if (bad_part[0] | bad_part[1] | bad_part[2] | bad_part[3]) status = -2;
  else if (nf < 0 || nf > a.capacity || R > a.capacity - nf) status = -3;
  else if (N > a.n_rows) status = -1;
  else if (A > nf + R) status = A - nf - R;
  __syncthreads();                                         // (also: everybody has read n_free)
  if (tid <= a.B) a.cu_new[tid] = status != 0 || tid == 0 ? 0 : tid == a.B ? N : s_row[tid];
  if (tid == 0) {
    *a.status = status;
    if (status == 0) *a.n_free = nf + R - A;
  }
  if (kRows)
    for (int r = (status == 0 ? N : 0) + tid; r < a.n_rows; r += kThreads) {
      a.slots[r] = -1;
      if (a.positions) a.positions[r] = 0;
    }
  if (status != 0) return;
  // lanes per request: the workgroup's over the batch, rounded up to a power of two
  const int lg = 32 - __clz(max(a.B - 1, 0) | 0), each = kThreads >> (a.B > 1 ? lg : 0);
  const int b = tid / each, i0 = tid % each;
  const int top = nf + R - 1;
  int held = 0, need = 0;
  int32_t *row = a.block_table + (int64_t)b * a.table_stride;
  if (b < a.B) {
    o = s_old[b]; n = s_new[b];
    held = (o + ps1) >> a.page_shift;
    need = (n + ps1) >> a.page_shift;
    for (int j = need + i0; j < held; j += each) a.free_pages[top - s_give[b] - (j - need)] = row[j];
  }
  __syncthreads();
  if (b < a.B)
    for (int j = held + i0; j < need; j += each) row[j] = a.free_pages[top - s_take[b] - (j - held)];
  if constexpr (!kRows) return;
  __syncthreads();
  if (b < a.B) {
    const int off = a.pos_offset ? a.pos_offset[b] : 0;
    for (int i = i0; i < n - o; i += each) {
      const int t = o + i;
      a.slots[s_row[b] + i] = (row[t >> a.page_shift] << a.page_shift) + (t & ps1);
      if (a.positions) a.positions[s_row[b] + i] = t + off;
    }
  }
}

// The rows alone, after the tables are made: a thread per row, its request by bisection of cu_new.
__global__ void __launch_bounds__(256) page_rows_kernel(PageUpdateArgs a) {
  __shared__ int cu[kMaxB + 1], old[kMaxB], off[kMaxB];
  for (int b = threadIdx.x; b <= a.B; b += 256) {
    cu[b] = a.cu_new[b];
    if (b < a.B) {
      old[b] = a.old_len[b];
      off[b] = a.pos_offset ? a.pos_offset[b] : 0;
    }
  }
  __syncthreads();
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r >= a.n_rows) return;
  int slot = -1, pos = 0;
  if (r < cu[a.B]) {                                       // (0 where the update was not done)
    int lo = 0, hi = a.B;                                  // cu[lo] <= r < cu[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= r) lo = mid;
      else hi = mid;
    }
    const int t = old[lo] + r - cu[lo];
    slot = (a.block_table[lo * a.table_stride + (t >> a.page_shift)] << a.page_shift) + (t & ((1 << a.page_shift) - 1));
    pos = t + off[lo];
  }
  a.slots[r] = slot;
  if (a.positions) a.positions[r] = pos;
}

}  // namespace

hipError_t launch_page_update(const PageUpdateArgs &a, hipStream_t st) {
  // A call takes the host longer than one workgroup takes for 29,000 rows (two calls and a copy 16.6 us, 18.1 with the second launch).
  if (a.n_rows <= kOneLaunch) {
    hipLaunchKernelGGL(page_update_kernel<true>, dim3(1), dim3(kThreads), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(page_update_kernel<false>, dim3(1), dim3(kThreads), 0, st, a);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL(page_rows_kernel, dim3((a.n_rows + 255) / 256), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sparrow
