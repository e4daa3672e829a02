// Attention of new tokens over the paged cache, fp32: products on the matrix cores in fp32 (v_mfma_f32_16x16x4_f32), blocks of 16, 32 or 64 rows
// (new token, query head of the group) per request and KV head.  Bound by memory up to 32 rows, by the matrix cores (157 TFLOP/s) above.
//
// A workgroup of four wavefronts takes one block and piece of keys; the wavefronts take its 16-token tiles in turn and know nothing of each
// other until the end, where their four states of a row are merged through LDS.  A tile lies on one page; it travels memory -> LDS past
// the registers, two tiles ahead.
//   S^T = K Q^T    A (16 x 4: lane = key + 16 * k): a 16-byte read gives a lane four k-steps, columns 16 g + 4 c4 + 0..3; Q^T in registers, cut alike.
//                 D: a lane holds, for row lane % 16, the scores of keys 4 c4 + 0..3.
//   O^T += V^T P^T  k-step i takes keys 4 c4 + i, so P^T is the scores' own register i and V^T a 4-byte read.
#include "chunk_attn_mfma.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 4, kTokens = 16;

// Over lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quad_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quad_sum(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// As add_masked, of one k-step.
__device__ __forceinline__ f32x4 add_masked_f32(float v, float p, float seen, f32x4 o) {
  const bool no = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;
  if (__builtin_amdgcn_ballot_w64(no) == 0ull) return __builtin_amdgcn_mfma_f32_16x16x4f32(v, p, o, 0, 0, 0);
  const bool nan = v != v;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  o = __builtin_amdgcn_mfma_f32_16x16x4f32(no ? 0.f : v, p, o, 0, 0, 0);
  const f32x4 up = __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v > 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0);
  const f32x4 down = __builtin_amdgcn_mfma_f32_16x16x4f32(nan || (no && v < 0.f) ? 1.f : 0.f, seen, zero, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] += (up[i] > 0.f ? INFINITY : 0.f) + (down[i] > 0.f ? -INFINITY : 0.f);
  return o;
}

template <int kD, int kRT>
__global__ void __launch_bounds__(64 * kWaves) chunk_f32_kernel(ChunkArgs a) {
  constexpr int kBM = 16 * kRT, kDB = kD / 16, kG = kD / 16, kRow = 4 * kD, kChunks = kD / 4, kLoadRows = 64 / kChunks;
  constexpr int kTileBytes = kTokens * kRow, kLoads = kTokens / kLoadRows;
  constexpr int kTiles = kWaves * 4 * kTileBytes, kMerge = kWaves * kBM * kRow;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTiles > kMerge ? kTiles : kMerge];   // [wave][K0, V0, K1, V1]
  __shared__ float ml[kWaves][kBM][2];

  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  Piece pc;
  if (!find_piece<kBM>(a, idx, lane, &pc)) return;         // uniform
  const int R = pc.rq.n * a.g, rho0 = pc.block * kBM;
  const auto table = (const int32_t __attribute__((address_space(4))) *)(uintptr_t)(a.block_table + (int64_t)pc.b * a.table_stride);
  const unsigned char *Kg = (const unsigned char *)((const float *)a.k + c * a.stride_head);
  const unsigned char *Vg = (const unsigned char *)((const float *)a.v + c * a.stride_head);
  const unsigned int row_bytes = (unsigned int)(4 * a.stride_token);
  // what the block's rows see of the piece
  const int last_pos = min(pc.rq.past + quotient(min(rho0 + kBM, R) - 1, a.g), pc.rq.L - 1);
  const int first_pos = pc.rq.past + quotient(rho0, a.g);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n_tiles = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;
  const int n = (n_tiles - w + kWaves - 1) / kWaves;       // of this wavefront: w, w + kWaves, ...

  unsigned char *mine = lds + w * 4 * kTileBytes;
  const unsigned int mine_at = lds_offset(mine);
  const auto swz = [](int row) { return (row & 7) << 1; };
  // rows of load j: kLoadRows j + lane / kChunks; lane's chunk by the row's swizzle (V's rows are read 4 bytes a lane and stay as they are)
  auto issue = [&](const unsigned char *src, bool swizzled, int tile, int part) __attribute__((always_inline)) {
    const int t = pc.t0 + tile * kTokens;
    const unsigned int page = min((unsigned int)table[t >> a.page_shift], (unsigned int)(a.n_pages - 1));
    const unsigned char *at = src + (int64_t)page * a.stride_page * 4 + (int64_t)(t & ((1 << a.page_shift) - 1)) * row_bytes;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = kLoadRows * j + lane / kChunks;
      const int chunk = swizzled ? (lane % kChunks) ^ swz(row) : lane % kChunks;
      global_to_lds<true>(at, row * row_bytes + 16u * chunk, mine_at + part * kTileBytes + 1024 * j);
    }
  };

  int pos[kRT], i_row[kRT], rho[kRT];
  f32x4 o[kRT][kDB];
  float m[kRT], l[kRT];
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    rho[rt] = min(rho0 + 16 * rt + n16, R - 1);
    i_row[rt] = quotient(rho[rt], a.g, a.inv_g);
    pos[rt] = min(pc.rq.past + i_row[rt], pc.rq.L - 1);
    m[rt] = kNegBig;
    l[rt] = 0.f;
#pragma unroll
    for (int db = 0; db < kDB; ++db) o[rt][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  if (n > 0) {
    issue(Kg, true, w, 0);
    issue(Vg, false, w, 1);
    f32x4 q[kRT][kG];
#pragma unroll
    for (int rt = 0; rt < kRT; ++rt) {
      const float *at = (const float *)a.q + (int64_t)(pc.rq.row0 + i_row[rt]) * a.q_row + (int64_t)(c * a.g + rho[rt] - i_row[rt] * a.g) * kD + 4 * c4;
#pragma unroll
      for (int g = 0; g < kG; ++g) q[rt][g] = *(const f32x4 *)(at + 16 * g);
    }
    wait_loads<0>();
    if (n > 1) {
      issue(Kg, true, w + kWaves, 2);
      issue(Vg, false, w + kWaves, 3);
    }
    for (int it = 0; it < n; ++it) {
      const int buf = it & 1;
      const bool more = it + 1 < n, more2 = it + 2 < n;
      if (more) wait_loads<3 * kLoads>();
      else wait_loads<kLoads>();
      const unsigned char *K = mine + 2 * buf * kTileBytes, *V = K + kTileBytes;
      f32x4 s[kRT];
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt) s[rt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const f32x4 k = *reinterpret_cast<const f32x4 *>(K + n16 * kRow + (((4 * g + c4) ^ swz(n16)) << 4));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int rt = 0; rt < kRT; ++rt) s[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[rt][g][i], s[rt], 0, 0, 0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(Kg, true, w + (it + 2) * kWaves, 2 * buf);
      const int t = pc.t0 + (w + it * kWaves) * kTokens;
      const bool edge = t + kTokens - 1 > min(first_pos, t1 - 1);          // some row does not see all of the tile
      float p[kRT][4], seen[kRT][4];
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt) {
        if (edge) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool vis = t + 4 * c4 + i <= min(pos[rt], t1 - 1);
            s[rt][i] = vis ? s[rt][i] : -INFINITY;
            seen[rt][i] = vis ? 1.f : 0.f;
          }
        }
        const float mx = fmaxf(fmaxf(s[rt][0], s[rt][1]), fmaxf(s[rt][2], s[rt][3])) * a.scale_log2;
        if (__builtin_amdgcn_ballot_w64(mx > m[rt] + kSlack) != 0ull) {
          const float m_new = fmaxf(m[rt], quad_max(mx)), alpha = fast_exp2(m[rt] - m_new);
          m[rt] = m_new;
          l[rt] *= alpha;
#pragma unroll
          for (int db = 0; db < kDB; ++db) o[rt][db] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[rt][i] = fast_exp2(fmaf(s[rt][i], a.scale_log2, -m[rt]));
        l[rt] += (p[rt][0] + p[rt][1]) + (p[rt][2] + p[rt][3]);
      }
      if (more2) wait_loads<3 * kLoads>();
      else if (more) wait_loads<2 * kLoads>();
      else wait_loads<0>();
#pragma unroll
      for (int db = 0; db < kDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = *reinterpret_cast<const float *>(V + (4 * c4 + i) * kRow + (16 * db + n16) * 4);
#pragma unroll
          for (int rt = 0; rt < kRT; ++rt)
            o[rt][db] = edge ? add_masked_f32(v, p[rt][i], seen[rt][i], o[rt][db])
                             : __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[rt][i], o[rt][db], 0, 0, 0);
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(Vg, false, w + (it + 2) * kWaves, 2 * buf + 1);
    }
  }
  // ---- merge: states of the four wavefronts through LDS
  __syncthreads();
  unsigned char *states = lds + w * kBM * kRow;
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    const int r = 16 * rt + n16;
    l[rt] = quad_sum(l[rt]);
    if (c4 == 0) { ml[w][r][0] = m[rt]; ml[w][r][1] = l[rt]; }
#pragma unroll
    for (int db = 0; db < kDB; ++db)                       // elements 16 db + 4 c4 + 0..3
      *reinterpret_cast<f32x4 *>(states + (r * kChunks + ((4 * db + c4) ^ n16)) * 16) = o[rt][db];
  }
  __syncthreads();
  const bool direct = pc.n_splits == 1;
  if (!direct && idx >= a.slots) return;                   // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) * kBM;
  const int rows = min(kBM, R - rho0);
  for (int x = threadIdx.x; x < rows * kChunks; x += 64 * kWaves) {
    const int r = x / kChunks, chunk = x % kChunks;
    float top = ml[0][r][0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) top = fmaxf(top, ml[k][r][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float ls = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = fast_exp2(ml[k][r][0] - top);
      ls = fmaf(ml[k][r][1], f, ls);
      sum += *reinterpret_cast<const f32x4 *>(lds + k * kBM * kRow + (r * kChunks + (chunk ^ (r & 15))) * 16) * f;
    }
    if (!direct) {
      *reinterpret_cast<f32x4 *>(a.part_o + (part + r) * kD + 4 * chunk) = sum;
      if (chunk == 0) {
        a.part_ml[2 * (part + r)] = top;
        a.part_ml[2 * (part + r) + 1] = ls;
      }
      continue;
    }
    const int i = quotient(rho0 + r, a.g, a.inv_g);
    const int64_t at = (int64_t)(pc.rq.row0 + i) * a.Hq + c * a.g + rho0 + r - i * a.g;
    const bool none = pc.rq.past + i < 0;
    if (none) sum = (f32x4){0.f, 0.f, 0.f, 0.f};
    else sum /= ls;
    *reinterpret_cast<f32x4 *>((float *)a.out + at * kD + 4 * chunk) = sum;
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : (top + fast_log2(ls)) * kLn2;
  }
}

template <int kRT> hipError_t launch(int d, dim3 grid, const ChunkArgs &a, hipStream_t st) {
  if (d == 128) hipLaunchKernelGGL((chunk_f32_kernel<128, kRT>), grid, dim3(64 * kWaves), 0, st, a);
  else hipLaunchKernelGGL((chunk_f32_kernel<64, kRT>), grid, dim3(64 * kWaves), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_f32(int d, int rows, int blocks, const ChunkArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, blocks < 32768 ? blocks : 32768, (blocks + 32767) / 32768);
  return rows == 16 ? launch<1>(d, grid, a, st) : rows == 32 ? launch<2>(d, grid, a, st) : launch<4>(d, grid, a, st);
}

}  // namespace sparrow
