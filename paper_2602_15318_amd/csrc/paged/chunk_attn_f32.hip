// Attention of chunks of new tokens over the paged cache, fp32: blocks of 64 rows (new token, query head of the group) per request and KV head, products on
// the matrix cores in fp32 (v_mfma_f32_16x16x4_f32).  Bound by them: 1,000 tokens over 6,000, 28/4 heads
// of 128, 730 us, 108 TFLOP/s (a library's product of 8,192^3 152).
//
// A workgroup of four wavefronts takes one block and piece of keys; wavefront w has rows 16 w .. 16 w + 15.  K and V tiles of 32 keys go memory -> LDS
// past the registers, one tile ahead; two workgroups share a compute unit, so that one's softmax runs beside the other's products.
// Operands as in chunk_attn_few16.hip.
#include "chunk_attn_16.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 4, kTokens = 32, kBM = 64;

template <int kD>
__global__ void __launch_bounds__(64 * kWaves, 2) chunk_f32_kernel(ChunkArgs a) {
  constexpr int kRow = 4 * kD, kChunks = kRow / 16, kDB = kD / 16, kG = kD / 16, kLoadRows = 64 / kChunks, kLoads = 8 / kLoadRows;
  constexpr int kTileBytes = kTokens * kRow, kSlab = 16 * kRow;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTileBytes];      // K0, V0, K1, V1

  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  Piece pc;
  if (!find_piece(a, idx, lane, &pc)) return;         // uniform
  const int R = pc.rq.n * a.g, rho0 = pc.block * kBM;
  const auto table = (const int32_t __attribute__((address_space(4))) *)(uintptr_t)(a.block_table + (int64_t)pc.b * a.table_stride);
  const unsigned char *Kg = (const unsigned char *)((const float *)a.k + c * a.stride_head);
  const unsigned char *Vg = (const unsigned char *)((const float *)a.v + c * a.stride_head);
  const unsigned int row_bytes = (unsigned int)(4 * a.stride_token);
  const int rho = min(rho0 + 16 * w + n16, R - 1);
  const int i_row = quotient(rho, a.g, a.inv_g), head = c * a.g + rho - i_row * a.g;
  const int pos = min(pc.rq.past + i_row, pc.rq.L - 1);
  // what the block's rows see of the piece
  const int last_pos = min(pc.rq.past + quotient(min(rho0 + kBM, R) - 1, a.g), pc.rq.L - 1);
  const int first_pos = pc.rq.past + quotient(rho0, a.g);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;

  const auto swz = [](int row) { return (row & 7) << 1; };
  const unsigned int lds0 = lds_offset(lds) + 8 * w * kRow;
  // rows 8 w .. 8 w + 7 of a tile, on one page; rows past the request's: some of its last page
  auto issue = [&](int tile, int buf) __attribute__((always_inline)) {
    const int t = pc.t0 + tile * kTokens + 8 * w;
    const unsigned int page = min((unsigned int)table[min(t, pc.rq.L - 1) >> a.page_shift], (unsigned int)(a.n_pages - 1));
    const int64_t at = (int64_t)page * a.stride_page * 4 + (int64_t)(t & ((1 << a.page_shift) - 1)) * row_bytes;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = kLoadRows * j + lane / kChunks;
      global_to_lds<false>(Kg + at, row * row_bytes + 16u * ((lane % kChunks) ^ swz(row)), lds0 + 2 * buf * kTileBytes + 1024 * j);
      global_to_lds<false>(Vg + at, row * row_bytes + 16u * (lane % kChunks), lds0 + (2 * buf + 1) * kTileBytes + 1024 * j);
    }
  };

  f32x4 o[kDB];
  float m = kNothingSeen, l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) o[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    issue(0, 0);
    f32x4 q[kG];
    {
      const float *at = (const float *)a.q + (int64_t)(pc.rq.row0 + i_row) * a.q_row + (int64_t)head * kD;
#pragma unroll
      for (int g = 0; g < kG; ++g) q[g] = ((const f32x4 *)at)[4 * g + c4];
    }
    const bool have = rho0 + 16 * w < R;                   // the wavefront has rows
    auto step = [&](int t, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      wait_loads<0>();
      barrier();                                           // tile t is there, and nobody reads tile t - 1
      if (t + 1 < n) issue(t + 1, (t + 1) & 1);
      if (!have) return;
      const unsigned char *K = lds + 2 * (t & 1) * kTileBytes, *V = K + kTileBytes;
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const int at = n16 * kRow + (((4 * g + c4) ^ swz(n16)) << 4);
        const f32x4 k[2] = {*reinterpret_cast<const f32x4 *>(K + at), *reinterpret_cast<const f32x4 *>(K + at + kSlab)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j][i], q[g][i], s[j], 0, 0, 0);
      }
      const int t0 = pc.t0 + t * kTokens;
      float p[2][4], seen[2][4];
      if constexpr (kMasked) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool vis = t0 + 16 * j + 4 * c4 + i <= min(pos, t1 - 1);
            s[j][i] = vis ? s[j][i] : -INFINITY;
            seen[j][i] = vis ? 1.f : 0.f;
          }
      }
      float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int i = 1; i < 4; ++i) mx = fmaxf(fmaxf(mx, s[0][i]), s[1][i]);
      if (__builtin_amdgcn_ballot_w64((mx - m) * a.scale_log2 > kSlack) != 0ull) {
        const float m_new = fmaxf(m, quad_max(mx)), alpha = factor(m, m_new, a.scale_log2);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < kDB; ++db) o[db] *= alpha;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[j][i] = fast_exp2((s[j][i] - m) * a.scale_log2);
        l += (p[j][0] + p[j][1]) + (p[j][2] + p[j][3]);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[kDB];
#pragma unroll
          for (int db = 0; db < kDB; ++db) v[db] = *reinterpret_cast<const float *>(V + j * kSlab + (4 * c4 + i) * kRow + (16 * db + n16) * 4);
          if constexpr (kMasked) {
            add_masked4(v, p[j][i], seen[j][i], o);
          } else {
#pragma unroll
            for (int db = 0; db < kDB; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[db], p[j][i], o[db], 0, 0, 0);
          }
        }
    };
    // the tiles that all rows of the block see whole, then the others
    const int n_full = min(n, max(min(first_pos + 1, t1) - pc.t0, 0) / kTokens);
    int t = 0;
    for (; t < n_full; ++t) step(t, std::false_type());
    for (; t < n; ++t) step(t, std::true_type());
  }
  // ---- the block's rows, or its partial of this piece: elements 16 db + 4 c4 + 0..3 of a row
  l = quad_sum(l);
  if (rho0 + 16 * w + n16 >= R) return;
  if (pc.n_splits == 1) {
    const bool none = pc.rq.past + i_row < 0;
    const int64_t to = (int64_t)(pc.rq.row0 + i_row) * a.Hq + head;
#pragma unroll
    for (int db = 0; db < kDB; ++db) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (!none) x = o[db] / l;
      *reinterpret_cast<f32x4 *>((float *)a.out + to * kD + 16 * db + 4 * c4) = x;
    }
    if (a.lse && c4 == 0) a.lse[to] = none ? -INFINITY : log_sum(m, a.scale_log2, l);
    return;
  }
  if (idx >= a.slots) return;                              // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) * kBM + 16 * w + n16;
#pragma unroll
  for (int db = 0; db < kDB; ++db) *reinterpret_cast<f32x4 *>(a.part_o + part * kD + 16 * db + 4 * c4) = o[db];
  if (c4 == 0) {
    a.part_ml[2 * part] = m;
    a.part_ml[2 * part + 1] = l;
  }
}

}  // namespace

hipError_t launch_chunk_f32(int d, int blocks, const ChunkArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, blocks < 32768 ? blocks : 32768, (blocks + 32767) / 32768), block(64 * kWaves);
  if (d == 128) hipLaunchKernelGGL(chunk_f32_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(chunk_f32_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace sparrow
