// Second pass of the chunk attention: the pieces of a block's keys put together.  kSpread wavefronts (16, 4, or 1: the more rows, the
// fewer) share the pieces of one (row of the batch, query head), all loads of a wavefront on their way at once.
#include "chunk_plan.hpp"

namespace sparrow {

namespace {

constexpr int kAtOnce = 8;

template <typename T, int kD, int kBM, int kSpread>
__global__ void __launch_bounds__(64 * (kSpread == 1 ? 4 : kSpread)) chunk_combine_kernel(ChunkArgs a) {
  constexpr int kWaves = kSpread == 1 ? 4 : kSpread;
  constexpr int kPer = kD / 64;                            // floats of a lane
  __shared__ float sum_o[kWaves][kD], sum_l[kWaves], tops[kWaves];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.y + 32768 * blockIdx.z;
  if (r >= a.n_rows) return;
  const Plan p = make_plan<kBM>(a, lane);
  int b = -1, n_blocks = 0, n_splits = 0, first = 0;
  Request q{};
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k)
    if (b < 0 && 64 * k < a.B) {
      const unsigned long long m = __builtin_amdgcn_ballot_w64(r >= p.rq[k].row0 && r - p.rq[k].row0 < p.rq[k].n);
      if (m != 0ull) {
        const int l = __builtin_ctzll(m);
        b = 64 * k + l;
        n_blocks = lane_value(p.n_blocks[k], l);
        n_splits = lane_value(p.n_splits[k], l);
        first = lane_value(p.end[k], l) - n_blocks * n_splits;
        q = {lane_value(p.rq[k].row0, l), lane_value(p.rq[k].n_all, l), lane_value(p.rq[k].n, l), lane_value(p.rq[k].L, l),
             lane_value(p.rq[k].past, l)};
      }
    }
  if (b < 0 || n_splits == 1) return;                      // (in one piece: written already)
  const int i = r - q.row0;
  const int part = kSpread > 1 ? w : 0;                    // which of the row's pieces
  for (int h = kSpread > 1 ? (int)blockIdx.x : w; h < a.Hq; h += kSpread > 1 ? (int)gridDim.x : kWaves) {
    const int c = quotient(h, a.g), rho = i * a.g + h - c * a.g, block = rho / kBM;
    const int piece0 = first + n_blocks - 1 - block;
    if (piece0 < 0 || piece0 + (n_splits - 1) * n_blocks >= a.slots) return;     // (offsets that overlap promise any number of pieces)
    const auto at = [&](int s) { return ((int64_t)(piece0 + s * n_blocks) * a.Hkv + c) * kBM + rho % kBM; };
    float top = kNegBig, l = 0.f, o[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) o[e] = 0.f;
    for (int s0 = part; s0 < n_splits; s0 += kSpread * kAtOnce) {
      float m[kAtOnce], ls[kAtOnce], x[kAtOnce][kPer];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t k = at(min(s0 + kSpread * u, n_splits - 1));
        m[u] = a.part_ml[2 * k];
        ls[u] = a.part_ml[2 * k + 1];
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[u][e] = a.part_o[k * kD + kPer * lane + e];
      }
      float t = top;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (s0 + kSpread * u >= n_splits) m[u] = kNegBig, ls[u] = 0.f;
        t = fmaxf(t, m[u]);
      }
      const float f0 = fast_exp2(top - t);
      l *= f0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] *= f0;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (s0 + kSpread * u >= n_splits) continue;
        const float f = fast_exp2(m[u] - t);
        l = fmaf(ls[u], f, l);
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = fmaf(x[u][e], f, o[e]);
      }
      top = t;
    }
    if constexpr (kSpread > 1) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) sum_o[w][kPer * lane + e] = o[e];
      if (lane == 0) { sum_l[w] = l; tops[w] = top; }
      __syncthreads();
      if (w != 0) return;
      float t = tops[0], ls = 0.f;
#pragma unroll
      for (int k = 1; k < kWaves; ++k) t = fmaxf(t, tops[k]);
#pragma unroll
      for (int e = 0; e < kPer; ++e) o[e] = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float f = fast_exp2(tops[k] - t);
        ls = fmaf(sum_l[k], f, ls);
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = fmaf(sum_o[k][kPer * lane + e], f, o[e]);
      }
      l = ls;
      top = t;
    }
    const bool none = q.past + i < 0;
    const int64_t to = (int64_t)r * a.Hq + h;
#pragma unroll
    for (int e = 0; e < kPer; ++e) Elem<T>::store((T *)a.out + to * kD + kPer * lane + e, none ? 0.f : o[e] / l);
    if (a.lse && lane == 0) a.lse[to] = none ? -INFINITY : (top + fast_log2(l)) * kLn2;
    if (kSpread > 1) return;
  }
}

template <typename T, int kD, int kBM> hipError_t launch(const ChunkArgs &a, hipStream_t st) {
  const int y = a.n_rows < 32768 ? a.n_rows : 32768, z = (a.n_rows + 32767) / 32768;
  // as many wavefronts a (row, head) as the chip holds
  const int64_t rows = (int64_t)a.n_rows * a.Hq;
  if (rows <= 512) hipLaunchKernelGGL((chunk_combine_kernel<T, kD, kBM, 16>), dim3(a.Hq, y, z), dim3(1024), 0, st, a);
  else if (rows <= 2048) hipLaunchKernelGGL((chunk_combine_kernel<T, kD, kBM, 4>), dim3(a.Hq, y, z), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((chunk_combine_kernel<T, kD, kBM, 1>), dim3(1, y, z), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_combine(int dtype, int d, int rows, const ChunkArgs &a, hipStream_t st) {
  const bool f32 = dtype == SPARROW_F32;
#define SPARROW_ROWS(n) \
  if (rows == n && f32) return d == 128 ? launch<float, 128, n>(a, st) : launch<float, 64, n>(a, st); \
  if (rows == n) return d == 128 ? launch<bf16_t, 128, n>(a, st) : launch<bf16_t, 64, n>(a, st);
  SPARROW_ROWS(16)
  SPARROW_ROWS(32)
  SPARROW_ROWS(64)
#undef SPARROW_ROWS
  return d == 128 ? launch<bf16_t, 128, 256>(a, st) : launch<bf16_t, 64, 256>(a, st);
}

}  // namespace sparrow
