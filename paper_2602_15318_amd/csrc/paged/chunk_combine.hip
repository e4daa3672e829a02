// Second pass of the chunk attention: the pieces of a block's keys put together.  kD / 4 lanes take a row's piece, 16 bytes each; the groups of
// kSpread wavefronts (8 or 2) share the pieces of one (row of the batch, query head), the loads of up to 8 pieces of a group on their
// way at once.  Where there are many rows (kSpread 1), each group takes a head of its own.
// Measured, 28/4 heads of 128: one token over 26,112 4.5 us, 48 over up to 8,192 5.0: about a launch and two dependent round trips.  A mixed batch of
// nine, 32/8 heads of 64, 7.2.
#include "chunk_plan.hpp"

namespace sparrow {

namespace {

struct State { float top, l; f32x4 o; };
__device__ __forceinline__ void add(State &s, float m, float l, f32x4 o, float scale_log2) {
  const float t = fmaxf(s.top, m), f = factor(s.top, t, scale_log2), g = factor(m, t, scale_log2);
  s.l = fmaf(s.l, f, l * g);
  s.o = s.o * f + o * g;
  s.top = t;
}

template <typename T, int kD, int kSpread>
__global__ void __launch_bounds__(64 * (kSpread == 1 ? 4 : kSpread)) chunk_combine_kernel(ChunkArgs a) {
  constexpr int kGroup = kD / 4, kGroups = 64 / kGroup, kAtOnce = kSpread == 1 ? 4 : 8, kParts = kSpread * kGroups;
  __shared__ __attribute__((aligned(16))) float sum_o[kParts][kD];
  __shared__ float sum_ml[kParts][2];
  const int lane = threadIdx.x & 63, group = lane / kGroup, at4 = 4 * (lane % kGroup);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.y + 32768 * blockIdx.z;
  if (r >= a.n_rows) return;
  // the row's request, and what the first pass has left of it
  int b = -1, i = 0, n = 0, past = 0, first = 0, n_splits = 0;
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k)
    if (b < 0 && 64 * k < a.B) {
      Request q{};
      int2 plan{};
      if (64 * k + lane < a.B) {
        q = request_of(a, 64 * k + lane);
        plan = ((const int2 *)a.plan)[64 * k + lane];
      }
      const unsigned long long m = __builtin_amdgcn_ballot_w64(r >= q.row0 && r - q.row0 < q.n);
      if (m != 0ull) {
        const int l = __builtin_ctzll(m);
        b = 64 * k + l;
        i = r - lane_value(q.row0, l);
        n = lane_value(q.n, l);
        past = lane_value(q.past, l);
        first = lane_value(plan.x, l);
        n_splits = lane_value(plan.y, l);
      }
    }
  if (b < 0 || n_splits <= 1) return;                      // (in one piece: written already)
  const int n_blocks = blocks_of(a, n);
  if (first < 0 || (int64_t)n_blocks * n_splits > a.slots - first) return;     // (offsets that overlap: a plan that nobody has written)
  const bool none = past + i < 0;
  const int part = w * kGroups + group;                    // kSpread 1: the head; else which of the pieces
  for (int h = kSpread > 1 ? (int)blockIdx.x : part; h < a.Hq; h += kSpread > 1 ? a.Hq : 4 * kGroups) {
    const int c = quotient(h, a.g, a.inv_g), rho = i * a.g + h - c * a.g;
    const int64_t at0 = (((int64_t)(first + n_blocks - 1 - (rho >> a.block_shift)) * a.Hkv + c) << a.block_shift) + (rho & ((1 << a.block_shift) - 1));
    const auto at = [&](int s) { return at0 + ((int64_t)s * n_blocks * a.Hkv << a.block_shift); };
    State st{kNothingSeen, 0.f, {0.f, 0.f, 0.f, 0.f}};
    constexpr int kStep = kSpread > 1 ? kParts : 1;
    for (int s0 = kSpread > 1 ? part : 0; s0 < n_splits; s0 += kStep * kAtOnce) {
      float m[kAtOnce], l[kAtOnce];
      f32x4 o[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int64_t k = at(min(s0 + kStep * u, n_splits - 1));
        const float2 ml = ((const float2 *)a.part_ml)[k];
        m[u] = ml.x;
        l[u] = ml.y;
        o[u] = *(const f32x4 *)(a.part_o + k * kD + at4);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (s0 + kStep * u < n_splits) add(st, m[u], l[u], o[u], a.scale_log2);
    }
    if constexpr (kSpread > 1) {
      *(f32x4 *)&sum_o[part][at4] = st.o;
      if (at4 == 0) { sum_ml[part][0] = st.top; sum_ml[part][1] = st.l; }
      __syncthreads();
      if (part != 0) return;
      const int n = min(kParts, n_splits);                 // those that had a piece
      for (int k = 1; k < n; ++k) st.top = fmaxf(st.top, sum_ml[k][0]);
      st.l = 0.f;
      st.o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float f = factor(sum_ml[k][0], st.top, a.scale_log2);
        st.l = fmaf(sum_ml[k][1], f, st.l);
        st.o += *(const f32x4 *)&sum_o[k][at4] * f;
      }
    }
    const int64_t to = (int64_t)r * a.Hq + h;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (!none) x = st.o / st.l;
    if constexpr (sizeof(T) == 4)
      *(f32x4 *)((float *)a.out + to * kD + at4) = x;
    else
      *(u32x2 *)((bf16_t *)a.out + to * kD + at4) = (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    if (a.lse && at4 == 0) a.lse[to] = none ? -INFINITY : log_sum(st.top, a.scale_log2, st.l);
  }
}

template <typename T, int kD> hipError_t launch(const ChunkArgs &a, hipStream_t st) {
  const int y = a.n_rows < 32768 ? a.n_rows : 32768, z = (a.n_rows + 32767) / 32768;
  // as many wavefronts a (row, head) as the chip holds
  const int64_t rows = (int64_t)a.n_rows * a.Hq;
  if (rows <= 1024) hipLaunchKernelGGL((chunk_combine_kernel<T, kD, 8>), dim3(a.Hq, y, z), dim3(512), 0, st, a);
  else if (rows <= 4096) hipLaunchKernelGGL((chunk_combine_kernel<T, kD, 2>), dim3(a.Hq, y, z), dim3(128), 0, st, a);
  else hipLaunchKernelGGL((chunk_combine_kernel<T, kD, 1>), dim3(1, y, z), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_combine(int dtype, int d, const ChunkArgs &a, hipStream_t st) {
  if (dtype == SPARROW_F32) return d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
  return d == 128 ? launch<bf16_t, 128>(a, st) : launch<bf16_t, 64>(a, st);
}

}  // namespace sparrow
