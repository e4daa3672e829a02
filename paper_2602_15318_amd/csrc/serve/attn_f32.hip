// Attention of new tokens in fp32 over a paged cache of fp32 or of 8 bits, prefixes of groups first: blocks of up to 64 rows (new token, query head of
// the group) of an item, products on the matrix cores in fp32.  As chunk_f32_kernel (../paged/chunk_attn_f32.hip): four wavefronts of 16 rows, K and
// V tiles of 32 keys one tile ahead, two workgroups per compute unit.  An 8-bit cache's tiles come through registers and are written to LDS as the fp32
// numbers that they are.
// Bound by the fp32 matrix cores from some 64 rows on: a chunk of 256 over 8,192, 28 and 4 heads of 128, 322 us.  Single tokens fill part of a wavefront's 16 rows and
// leave three wavefronts idle: 48 over up to 8,192, 8 bits, 191 us, matrix cores busy for 45 and LDS for 60, a third of it bank conflicts of the tiles' writes and V's
// reads.  Five over 500 (a head of 64) 7 us, round trips.
#include "serve_tiles.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 4, kTokens = 32;

template <typename C, int kD>
__global__ void __launch_bounds__(64 * kWaves, 2) serve_attn_f32_kernel(ServeArgs a) {
  constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  constexpr int kRow = 4 * kD, kChunks = kRow / 16, kDB = kD / 16, kG = kD / 16, kLoadRows = 64 / kChunks, kLoads = 8 / kLoadRows;
  constexpr int kTileBytes = kTokens * kRow, kSlab = 16 * kRow;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[4 * kTileBytes];      // K0, V0, K1, V1

  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  ServePiece pc;
  if (!serve_piece(a, idx, &pc)) return;              // uniform
  const ServePages<C> pages = serve_pages<C>(a, pc.it, c);
  const int block_rows = 1 << a.block_shift, R = pc.it.n * a.g, rho0 = pc.block << a.block_shift;
  const int in_block = 16 * w + n16;
  const int rho = min(rho0 + min(in_block, block_rows - 1), R - 1);
  const int i_row = quotient(rho, a.g, a.inv_g), head = c * a.g + rho - i_row * a.g;
  const int pos = min(pc.it.past + i_row, pc.it.to - 1);
  // what the block's rows see of the piece
  const int last_pos = min(pc.it.past + quotient(min(rho0 + block_rows, R) - 1, a.g), pc.it.to - 1);
  const int first_pos = pc.it.past + quotient(rho0, a.g);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;

  const auto swz = [](int row) { return (row & 7) << 1; };
  // rows 8 w .. 8 w + 7 of a tile, on one page
  const unsigned int lds0 = lds_offset(lds) + 8 * w * kRow;
  const auto issue = [&](int tile, int buf) __attribute__((always_inline)) {
    const auto place = pages.place(pc.t0 + tile * kTokens + 8 * w);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = kLoadRows * j + lane / kChunks;
      global_to_lds<false>(pages.k + place.at, row * pages.stride_token + 16u * ((lane % kChunks) ^ swz(row)), lds0 + 2 * buf * kTileBytes + 1024 * j);
      global_to_lds<false>(pages.v + place.at, row * pages.stride_token + 16u * (lane % kChunks), lds0 + (2 * buf + 1) * kTileBytes + 1024 * j);
    }
  };
  // 8 bits: kD / 8 codes of row lane / 8 of them, and its powers
  typedef __attribute__((ext_vector_type(kD / 32))) unsigned int Codes;
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  Codes kc, vc;
  unsigned int powers = 0u;
  const auto fetch = [&](int tile) __attribute__((always_inline)) {
    const auto place = pages.place(pc.t0 + tile * kTokens + 8 * w);
    const unsigned int off = (lane / 8) * pages.stride_token + (kD / 8) * (lane % 8);
    kc = *(const Codes *)(pages.k + place.at + off);
    vc = *(const Codes *)(pages.v + place.at + off);
    powers = pages.powers_of(place, lane / 8);
  };
  const auto store = [&](int buf) __attribute__((always_inline)) {
    unsigned char *to = lds + 2 * buf * kTileBytes + (8 * w + lane / 8) * kRow;
    const float pk = power_in(powers, lane / 8, false), pv = power_in(powers, lane / 8, true);
#pragma unroll
    for (int i = 0; i < kD / 32; ++i) {                    // 16 bytes of fp32: four codes
      const int chunk = kD / 32 * (lane % 8) + i;
      const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8((int)kc[i], false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)kc[i], true);
      *reinterpret_cast<f32x4 *>(to + ((chunk ^ swz(lane / 8)) << 4)) = (f32x4){x[0] * pk, x[1] * pk, y[0] * pk, y[1] * pk};
      const f32x2 u = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], false), v = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], true);
      *reinterpret_cast<f32x4 *>(to + kTileBytes + (chunk << 4)) = (f32x4){u[0] * pv, u[1] * pv, v[0] * pv, v[1] * pv};
    }
  };

  f32x4 o[kDB];
  float m = kNothingSeen, l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) o[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    if constexpr (k8) fetch(0);
    else issue(0, 0);
    f32x4 q[kG];
    {
      const float *at = (const float *)a.q + (int64_t)(pc.it.row0 + i_row) * a.q_row + (int64_t)head * kD;
#pragma unroll
      for (int g = 0; g < kG; ++g) q[g] = ((const f32x4 *)at)[4 * g + c4];
    }
    const bool have = 16 * w < min(block_rows, R - rho0);  // the wavefront has rows
    const auto step = [&](int t, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      if constexpr (k8) {
        store(t & 1);                                      // (tile t - 2, which was there, has been read: the barrier of step t - 1)
        if (t + 1 < n) fetch(t + 1);
        barrier();
      } else {
        wait_loads<0>();
        barrier();                                         // tile t is there, and nobody reads tile t - 1
        if (t + 1 < n) issue(t + 1, (t + 1) & 1);
      }
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
  if (in_block >= min(block_rows, R - rho0)) return;
  if (pc.direct) {
    const bool none = pc.it.past + i_row < 0;
    const int64_t to = (int64_t)(pc.it.row0 + i_row) * a.Hq + head;
#pragma unroll
    for (int db = 0; db < kDB; ++db) {
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (!none) x = o[db] / (k8 ? l * kLowered : l);
      *reinterpret_cast<f32x4 *>((float *)a.out + to * kD + 16 * db + 4 * c4) = x;
    }
    if (a.lse && c4 == 0) a.lse[to] = none ? -INFINITY : log_sum(m, a.scale_log2, l);
    return;
  }
  if (idx >= a.slots) return;                              // (offsets that overlap)
  const int64_t part = (((int64_t)idx * a.Hkv + c) << a.block_shift) + in_block;
#pragma unroll
  for (int db = 0; db < kDB; ++db) *reinterpret_cast<f32x4 *>(a.part_o + part * kD + 16 * db + 4 * c4) = o[db];
  if (c4 == 0) {
    a.part_ml[2 * part] = m;
    a.part_ml[2 * part + 1] = l;
  }
}

}  // namespace

hipError_t launch_serve_f32(int d, int pieces, const ServeArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, pieces < 32768 ? pieces : 32768, (pieces + 32767) / 32768), block(64 * kWaves);
  if (a.exponents) {
    if (d == 128) hipLaunchKernelGGL((serve_attn_f32_kernel<e4m3_t, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((serve_attn_f32_kernel<e4m3_t, 64>), grid, block, 0, st, a);
  } else {
    if (d == 128) hipLaunchKernelGGL((serve_attn_f32_kernel<float, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((serve_attn_f32_kernel<float, 64>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sparrow
