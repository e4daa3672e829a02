// Attention of new tokens in bf16 over a paged cache of bf16 or of 8 bits, prefixes of groups first: a workgroup of eight wavefronts takes a
// piece of an item, of up to 16 rows (attn_few.hpp, bound by memory) or more (attn_many.hpp, bound by the matrix cores and, beside them, by the
// exponentials).  In one launch, so that prefixes run beside what is behind them.
#include "attn_few.hpp"
#include "attn_many.hpp"

namespace sparrow {

namespace {

template <typename C, int kD>
__global__ void __launch_bounds__(64 * kServeWaves, 2) serve_attn_kernel(ServeArgs a) {
  constexpr int kBytes = FewTiles<C, kD>::kBytes > ManyTiles<kD>::kBytes ? FewTiles<C, kD>::kBytes : ManyTiles<kD>::kBytes;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kBytes];
  __shared__ float ml[kServeWaves][16][2];
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  ServePiece pc;
  if (!serve_piece(a, idx, &pc)) return;              // uniform
  if (pc.it.n * a.g <= 16) attend_few<C, kD>(a, pc, idx, c, lds, ml);
  else attend_many<C, kD>(a, pc, idx, c, lds);
}

}  // namespace

hipError_t launch_serve_bf16(int d, int pieces, const ServeArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, pieces < 32768 ? pieces : 32768, (pieces + 32767) / 32768), block(64 * kServeWaves);
  if (a.exponents) {
    if (d == 128) hipLaunchKernelGGL((serve_attn_kernel<e4m3_t, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((serve_attn_kernel<e4m3_t, 64>), grid, block, 0, st, a);
  } else {
    if (d == 128) hipLaunchKernelGGL((serve_attn_kernel<bf16_t, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((serve_attn_kernel<bf16_t, 64>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sparrow
