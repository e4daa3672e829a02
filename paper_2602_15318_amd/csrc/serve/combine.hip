// Second pass of the attention: a row's pieces of what is behind its prefix and of the prefix put together.  As chunk_combine_kernel
// (../paged/chunk_combine.hip): kD / 4 lanes take a row's piece, 16 bytes each; the groups of kSpread wavefronts (8 or 2) share the pieces of one
// (row of the batch, query head), the loads of up to 8 pieces of a group on their way at once.  Where there are many rows (kSpread 1), each group takes
// a head of its own.
//
// Bound by memory and its round trips: 32 single tokens over a shared 26,112 (21 MB of partials) 8.5 us, one token 4.9.
#include "serve_plan.hpp"

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
__global__ void __launch_bounds__(64 * (kSpread == 1 ? 4 : kSpread)) serve_combine_kernel(ServeArgs a) {
  constexpr int kGroup = kD / 4, kGroups = 64 / kGroup, kAtOnce = kSpread == 1 ? 4 : 8, kParts = kSpread * kGroups;
  __shared__ __attribute__((aligned(16))) float sum_o[kSpread][kD];
  __shared__ float sum_ml[kSpread][2];
  const int lane = threadIdx.x & 63, group = lane / kGroup, at4 = 4 * (lane % kGroup);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.y + 32768 * blockIdx.z;
  if (r >= a.n_rows) return;
  // the row's request, and what the first pass has left of it
  int b = -1, i = 0, n = 0, past = 0;
  ServeLeft left{};
#pragma unroll
  for (int k = 0; k < kMaxPerLane; ++k)
    if (b < 0 && 64 * k < a.B) {
      int row0 = 0, rows = 0, before = 0;
      ServeLeft mine{};
      if (64 * k + lane < a.B) {
        const int x = 64 * k + lane, c0 = min(max(a.cu_new[x], 0), a.n_rows), c1 = min(max(a.cu_new[x + 1], 0), a.n_rows);
        row0 = c0;
        rows = min(max(c1 - c0, 0), a.max_new);
        before = max(a.kv_len[x], 0) - max(c1 - c0, 0);
        mine = a.left[x];
      }
      const unsigned long long m = __builtin_amdgcn_ballot_w64(r >= row0 && r - row0 < rows);
      if (m != 0ull) {
        const int l = __builtin_ctzll(m);
        b = 64 * k + l;
        i = r - lane_value(row0, l);
        n = lane_value(rows, l);
        past = lane_value(before, l);
        left = {lane_value(mine.first, l), lane_value(mine.n_splits, l), lane_value(mine.group_first, l), lane_value(mine.group_splits, l),
                lane_value(mine.group_row0, l), lane_value(mine.group_blocks, l), {0, 0}};
      }
    }
  const int n_own = left.n_splits, n_shared = left.group_splits, n_all = n_own + n_shared;
  if (b < 0 || n_own < 1 || n_shared < 0 || (n_own == 1 && n_shared == 0)) return;       // (in one piece: written already)
  const int n_blocks = serve_blocks(a, n);
  // (offsets that overlap: a plan that nobody has written)
  if (left.first < 0 || (int64_t)n_blocks * n_own > a.slots - left.first) return;
  const int64_t group_rho = ((int64_t)r - left.group_row0) * a.g;
  if (n_shared > 0 && (left.group_first < 0 || left.group_blocks < 1 || (int64_t)left.group_blocks * n_shared > a.slots - left.group_first ||
                       group_rho < 0 || (group_rho + a.g - 1) >> a.block_shift >= left.group_blocks))
    return;
  const bool none = past + i < 0;
  const int part = w * kGroups + group;                    // kSpread 1: the head; else which of the pieces
  for (int h = kSpread > 1 ? (int)blockIdx.x : 4 * kGroups * blockIdx.x + part; h < a.Hq; h += kSpread > 1 ? a.Hq : 4 * kGroups * gridDim.x) {
    const int c = quotient(h, a.g, a.inv_g), of_group = h - c * a.g;
    const auto row_of = [&](int first, int blocks, int rho) {
      return (((int64_t)(first + blocks - 1 - (rho >> a.block_shift)) * a.Hkv + c) << a.block_shift) + (rho & ((1 << a.block_shift) - 1));
    };
    const int64_t own0 = row_of(left.first, n_blocks, i * a.g + of_group), shared0 = row_of(left.group_first, left.group_blocks, (int)group_rho + of_group);
    const auto at = [&](int s) {
      return s < n_own ? own0 + ((int64_t)s * n_blocks * a.Hkv << a.block_shift)
                       : shared0 + ((int64_t)(s - n_own) * left.group_blocks * a.Hkv << a.block_shift);
    };
    State st{kNothingSeen, 0.f, {0.f, 0.f, 0.f, 0.f}};
    constexpr int kStep = kSpread > 1 ? kParts : 1;
    for (int s0 = kSpread > 1 ? part : 0; s0 < n_all; s0 += kStep * kAtOnce) {
      float m[kAtOnce], l[kAtOnce];
      f32x4 o[kAtOnce];
      const int left_over = (n_all - 1 - s0) / kStep;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {                  // (behind the last: the last again, which is on its way already)
        const int64_t k = at(s0 + kStep * min(u, left_over));
        const float2 ml = ((const float2 *)a.part_ml)[k];
        m[u] = ml.x;
        l[u] = ml.y;
        o[u] = *(const f32x4 *)(a.part_o + k * kD + at4);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u)
        if (s0 + kStep * u < n_all) add(st, m[u], l[u], o[u], a.scale_log2);
    }
    if constexpr (kSpread > 1) {
#pragma unroll
      for (int x = kGroup; x < 64; x <<= 1) {              // the wavefront's groups, then the wavefronts
        f32x4 other;
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = __shfl_xor(st.o[i], x, 64);
        add(st, __shfl_xor(st.top, x, 64), __shfl_xor(st.l, x, 64), other, a.scale_log2);
      }
      if (group == 0) *(f32x4 *)&sum_o[w][at4] = st.o;
      if (lane == 0) { sum_ml[w][0] = st.top; sum_ml[w][1] = st.l; }
      __syncthreads();
      if (part != 0) return;
#pragma unroll
      for (int k = 1; k < kSpread; ++k) add(st, sum_ml[k][0], sum_ml[k][1], *(const f32x4 *)&sum_o[k][at4], a.scale_log2);
    }
    const int64_t to = (int64_t)r * a.Hq + h;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    if (!none) x = st.o / (st.l * lowered(a));
    if constexpr (sizeof(T) == 4)
      *(f32x4 *)((float *)a.out + to * kD + at4) = x;
    else
      *(u32x2 *)((bf16_t *)a.out + to * kD + at4) = (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    if (a.lse && at4 == 0) a.lse[to] = none ? -INFINITY : log_sum(st.top, a.scale_log2, st.l);
  }
}

template <typename T, int kD> hipError_t launch(const ServeArgs &a, hipStream_t st) {
  const int y = a.n_rows < 32768 ? a.n_rows : 32768, z = (a.n_rows + 32767) / 32768;
  // Wavefronts a (row, head): 8 below 256 of them, 2 below 3,200, else a part of one.  us of a call, rows * heads, with 8 / 2 / less: 896 42.5 / 41.3 / -, 1,344
  // 53.5 / 50.3 / 50.4, 2,688 63.1 / 53.0 / 54.5, 3,584 62.5 / 51.1 / 48.8, 7,168 - / 59.7 / 55.0.
  const int64_t rows = (int64_t)a.n_rows * a.Hq;
  if (rows <= 256) hipLaunchKernelGGL((serve_combine_kernel<T, kD, 8>), dim3(a.Hq, y, z), dim3(512), 0, st, a);
  else if (rows <= 3200) hipLaunchKernelGGL((serve_combine_kernel<T, kD, 2>), dim3(a.Hq, y, z), dim3(128), 0, st, a);
  else hipLaunchKernelGGL((serve_combine_kernel<T, kD, 1>), dim3((a.Hq + 1024 / kD - 1) / (1024 / kD), y, z), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_serve_combine(int dtype, int d, const ServeArgs &a, hipStream_t st) {
  if (dtype == SPARROW_F32) return d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
  return d == 128 ? launch<bf16_t, 128>(a, st) : launch<bf16_t, 64>(a, st);
}

}  // namespace sparrow
