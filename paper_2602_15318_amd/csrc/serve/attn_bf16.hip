// Attention of new tokens in bf16 over a paged cache of bf16 or of 8 bits, prefixes of groups first: a workgroup of eight wavefronts takes a
// piece of an item, of up to 16 rows (attn_few.hpp, bound by memory) or more (attn_many.hpp, bound by the matrix cores and, beside them, by the
// exponentials).  In one launch, so that prefixes run beside what is behind them.
#include "attn_many.hpp"
#include "attn_some.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 8;

template <typename C, int kD>
__global__ void __launch_bounds__(64 * kWaves, 2) serve_attn_kernel(ServeArgs a) {
  constexpr int kFew = FewTiles<C, kD, kWaves>::kBytes, kMany = ManyTiles<kD>::kBytes, kBytes = kFew > kMany ? kFew : kMany;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kBytes];
  __shared__ float ml[kWaves][16][2];
  __shared__ int flags[kWaves];
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  ServePiece pc;
  if (!serve_piece(a, idx, &pc)) return;              // uniform
  if (pc.it.n * a.g <= 16) attend_few<C, kD, kWaves>(a, pc, idx, c, lds, ml);
  else attend_many<C, kD>(a, pc, idx, c, lds, flags);
}

// Calls without groups whose requests have 16 rows at most
template <typename C, int kD, int kW>
__global__ void __launch_bounds__(64 * kW, 2) serve_few_kernel(ServeArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[FewTiles<C, kD, kW>::kBytes];
  __shared__ float ml[kW][16][2];
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  ServePiece pc;
  if (!serve_find_piece(a, idx, &pc)) return;         // uniform
  attend_few<C, kD, kW>(a, pc, idx, c, lds, ml);
}

// Calls without groups whose requests have 64 rows at most.  (A kernel of its own: in the one above it has too few scalar registers.)
template <typename C, int kD>
__global__ void __launch_bounds__(64 * kWaves, 2) serve_some_kernel(ServeArgs a) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[FewTiles<C, kD, kWaves>::kBytes];
  __shared__ float ml[kWaves][32][2];
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  ServePiece pc;
  if (!serve_find_piece(a, idx, &pc)) return;         // uniform
  if (pc.it.n * a.g <= 16) attend_few<C, kD, kWaves>(a, pc, idx, c, lds, (float (*)[16][2])ml);
  else attend_some<C, kD>(a, pc, idx, c, lds, ml);
}

template <typename C, int kD> hipError_t launch(const ServeShape &s, const ServeArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, s.grid < 32768 ? s.grid : 32768, (s.grid + 32767) / 32768);
  const auto run = [&](auto kernel, int waves) { hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), 0, st, a); };
  if (a.G == 0 && s.rows == 64) run(serve_some_kernel<C, kD>, kWaves);
  else if (a.G > 0 || s.rows > 16) run(serve_attn_kernel<C, kD>, kWaves);
  else if (s.waves == 8) run(serve_few_kernel<C, kD, 8>, 8);
  else if (s.waves == 4) run(serve_few_kernel<C, kD, 4>, 4);
  else run(serve_few_kernel<C, kD, 2>, 2);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_serve_bf16(int d, const ServeShape &s, const ServeArgs &a, hipStream_t st) {
  if (a.exponents) return d == 128 ? launch<e4m3_t, 128>(s, a, st) : launch<e4m3_t, 64>(s, a, st);
  return d == 128 ? launch<bf16_t, 128>(s, a, st) : launch<bf16_t, 64>(s, a, st);
}

}  // namespace sparrow
