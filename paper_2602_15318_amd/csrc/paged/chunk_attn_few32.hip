// Attention of few new tokens over the paged cache, bf16: 17 to 64 rows (new token, query head of the group) per request and KV head.
// Bound by memory: every key and value is read once, by one workgroup.  Measured a call, 28/4 heads of 128: four tokens over 26,112 (53.5 MB) 18 us,
// eight 23, twelve requests of eight tokens over up to 8,000 34.  Probabilities are rounded to bf16 for the output's product; their sum is not (what a
// second term costs: chunk_attn_few16.hip).
//
// A workgroup of four wavefronts takes one piece of a request's keys for one KV head; the wavefronts take its 32-token tiles in turn
// and know nothing of each other until the end, where their four states of a row are merged through LDS.  A wavefront's tiles travel
// memory -> LDS without passing registers (page by page, two tiles of K and V ahead, 64 KB in flight on a compute unit).
#include <type_traits>

#include "chunk_attn_mfma.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 4, kTokens = 32;

template <int kD, int kRT>
__global__ void __launch_bounds__(64 * kWaves) chunk_few32_kernel(ChunkArgs a) {
  using Rows = Tile<kD, false>;
  constexpr int kBM = 32 * kRT, kDB = kD / 32, kKS = kD / 16;
  constexpr int kTileBytes = kTokens * 2 * kD, kLoads = kTokens / Rows::kLoadRows;   // of a tile of K (or V)
  constexpr int kRowChunks = kD / 4;                       // 16-byte chunks of a row of fp32 outputs
  constexpr int kTiles = kWaves * 4 * kTileBytes, kMerge = kWaves * kBM * kD * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTiles > kMerge ? kTiles : kMerge];   // [wave][K0, V0, K1, V1]
  __shared__ float ml[kWaves][kBM][2];

  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y;
  Piece pc;
  if (!find_piece(a, idx, lane, &pc)) return;         // uniform
  const Pages pages = pages_of(a, pc, c);
  const int rho0 = pc.block * kBM, R = pc.rq.n * a.g - rho0;      // rows of the request from the block's first on

  unsigned char *mine = lds + w * 4 * kTileBytes;
  const unsigned int mine_at = lds_offset(mine);
  unsigned int from_k[2], from_v[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) from_k[j] = Rows::k_from(lane, Rows::kLoadRows * j, pages.stride_token);
#pragma unroll
  for (int j = 0; j < 2; ++j) from_v[j] = Rows::v_from(lane, Rows::kLoadRows * j, pages.stride_token);
  auto issue = [&](bool value, int tile, int part) __attribute__((always_inline)) {
    const int t = pc.t0 + tile * kTokens;
    const int64_t half[2] = {pages.offset(t), pages.offset(t + 16)};
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      global_to_lds<true>((value ? pages.v : pages.k) + half[2 * j / kLoads] + (int64_t)(j % (kLoads / 2) * Rows::kLoadRows) * pages.stride_token,
                          value ? from_v[j & 1] : from_k[j & 1], mine_at + part * kTileBytes + 1024 * j);
  };
  const int n_tiles = (pc.t1 - pc.t0 + kTokens - 1) / kTokens;
  const int n = (n_tiles - w + kWaves - 1) / kWaves;       // of this wavefront: w, w + kWaves, ...

  // rows of the lane
  int pos[kRT];
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    const int rho = rho0 + min(32 * rt + (lane & 31), R - 1);
    pos[rt] = min(pc.rq.past + (int)(((float)rho + 0.5f) * a.inv_g), pc.rq.L - 1);
  }
  f32x16 o[kRT][kDB];
  float m[kRT], l[kRT];
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    m[rt] = kNothingSeen;
    l[rt] = 0.f;
#pragma unroll
    for (int db = 0; db < kDB; ++db) o[rt][db] = (f32x16){0.f};
  }
  if (n > 0) {
    // Q through the second tile's place, ahead of the first tile
    constexpr int kQLoads = kRT * kLoads;
#pragma unroll
    for (int j = 0; j < kQLoads; ++j) {
      const int rho = rho0 + min(j * Rows::kLoadRows + lane / Rows::kChunks, R - 1);
      const int i = (int)(((float)rho + 0.5f) * a.inv_g);
      const unsigned char *at = (const unsigned char *)a.q + 2 * ((int64_t)(pc.rq.row0 + i) * a.q_row + (int64_t)(c * a.g + rho - i * a.g) * kD);
      const int row = j * Rows::kLoadRows + lane / Rows::kChunks;
      global_to_lds_each(at + 16 * ((lane % Rows::kChunks) ^ Rows::swz_k(row)), mine_at + 2 * kTileBytes + 1024 * j);
    }
    issue(false, w, 0);
    issue(true, w, 1);
    wait_loads<2 * kLoads>();
    bf16x8 q[kRT][kKS];
#pragma unroll
    for (int rt = 0; rt < kRT; ++rt)
#pragma unroll
      for (int ks = 0; ks < kKS; ++ks) q[rt][ks] = lds_b128(mine + 2 * kTileBytes + Rows::k(32 * rt + (lane & 31), 2 * ks + h));
    wait_loads<2 * kLoads>();                              // (the reads are done: their place may be written)
    if (n > 1) {
      issue(false, w + kWaves, 2);
      issue(true, w + kWaves, 3);
    }
    auto step = [&](int it, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      const int buf = it & 1;
      const bool more = it + 1 < n, more2 = it + 2 < n;
      if (more) wait_loads<3 * kLoads>();
      else wait_loads<kLoads>();
      const unsigned char *K = mine + 2 * buf * kTileBytes, *V = K + kTileBytes;
      f32x16 s[kRT];
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt) s[rt] = (f32x16){0.f};
#pragma unroll
      for (int ks = 0; ks < kKS; ++ks) {
        const bf16x8 k = lds_b128(K + (k_at<kD, false>(lane) ^ ks << 5));
#pragma unroll
        for (int rt = 0; rt < kRT; ++rt) s[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[rt][ks], s[rt], 0, 0, 0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(false, w + (it + 2) * kWaves, 2 * buf);
      const int t = pc.t0 + (w + it * kWaves) * kTokens;
      bf16x8 pb[kRT][2], seen[kRT][2];
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt) {
        if constexpr (kMasked) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int key = t + 8 * (e >> 2) + 4 * h + (e & 3);
            const bool vis = key <= min(pos[rt], pc.t1 - 1);
            s[rt][e] = vis ? s[rt][e] : -INFINITY;
            seen[rt][e >> 3][e & 7] = (__bf16)(vis ? 1.f : 0.f);
          }
        }
        float mx = s[rt][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[rt][e]);
        if (__builtin_amdgcn_ballot_w64((mx - m[rt]) * a.scale_log2 > kSlack) != 0ull) {
          const float m_new = fmaxf(m[rt], pair_max(mx)), alpha = factor(m[rt], m_new, a.scale_log2);
          m[rt] = m_new;
          l[rt] *= alpha;
#pragma unroll
          for (int db = 0; db < kDB; ++db) o[rt][db] *= alpha;
        }
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = fast_exp2((s[rt][e] - m[rt]) * a.scale_log2);
          sum += p;
          pb[rt][e >> 3][e & 7] = (__bf16)p;
        }
        l[rt] += sum;
      }
      if (more2) wait_loads<3 * kLoads>();
      else if (more) wait_loads<2 * kLoads>();
      else wait_loads<0>();
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        bf16x8 v[kDB];
#pragma unroll
        for (int db = 0; db < kDB; ++db) v[db] = read_vt<kD>(V + (vt_at<kD>(lane) ^ db << 6), st);
#pragma unroll
        for (int rt = 0; rt < kRT; ++rt) {
          if constexpr (kMasked) {
            add_masked(v, pb[rt][st], seen[rt][st], o[rt]);
          } else {
#pragma unroll
            for (int db = 0; db < kDB; ++db) o[rt][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db], pb[rt][st], o[rt][db], 0, 0, 0);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(true, w + (it + 2) * kWaves, 2 * buf + 1);
    };
    // the tiles that all rows of the block see whole, then the others
    const int first_pos = pc.rq.past + quotient(rho0, a.g);
    const int full = max(min(first_pos + 1, pc.t1) - pc.t0, 0) / kTokens, n_full = max(full - w + kWaves - 1, 0) / kWaves;
    int it = 0;
    for (; it < n_full; ++it) step(it, std::false_type());
    for (; it < n; ++it) step(it, std::true_type());
  }
  // ---- merge: states of the four wavefronts, fp32, through LDS
  __syncthreads();
  unsigned char *states = lds + w * kBM * kD * 4;
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    const int r = 32 * rt + (lane & 31);
    l[rt] = pair_sum(l[rt]);
    if (h == 0) { ml[w][r][0] = m[rt]; ml[w][r][1] = l[rt]; }
#pragma unroll
    for (int db = 0; db < kDB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int chunk = 8 * db + 2 * j + h;              // elements 32 db + 8 j + 4 h + 0..3
        const f32x4 x = {o[rt][db][4 * j], o[rt][db][4 * j + 1], o[rt][db][4 * j + 2], o[rt][db][4 * j + 3]};
        *reinterpret_cast<f32x4 *>(states + (r * kRowChunks + (chunk ^ (r & (kRowChunks - 1)))) * 16) = x;
      }
  }
  __syncthreads();
  const bool direct = pc.n_splits == 1;
  if (!direct && idx >= a.slots) return;                   // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) * kBM;
  for (int x = threadIdx.x; x < min(R, kBM) * kRowChunks; x += 64 * kWaves) {
    const int r = x / kRowChunks, chunk = x % kRowChunks;
    float top = ml[0][r][0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) top = fmaxf(top, ml[k][r][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float ls = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = factor(ml[k][r][0], top, a.scale_log2);
      ls = fmaf(ml[k][r][1], f, ls);
      sum += *reinterpret_cast<const f32x4 *>(lds + k * kBM * kD * 4 + (r * kRowChunks + (chunk ^ (r & (kRowChunks - 1)))) * 16) * f;
    }
    if (!direct) {
      *reinterpret_cast<f32x4 *>(a.part_o + (part + r) * kD + 4 * chunk) = sum;
      if (chunk == 0) {
        a.part_ml[2 * (part + r)] = top;
        a.part_ml[2 * (part + r) + 1] = ls;
      }
      continue;
    }
    const int rho = rho0 + r, i = (int)(((float)rho + 0.5f) * a.inv_g);
    const int64_t at = (int64_t)(pc.rq.row0 + i) * a.Hq + c * a.g + rho - i * a.g;
    const bool none = pc.rq.past + i < 0;
    const float inv = 1.f / ls;
    if (none) sum = (f32x4){0.f, 0.f, 0.f, 0.f};
    else sum *= inv;
    *reinterpret_cast<u32x2 *>((bf16_t *)a.out + at * kD + 4 * chunk) = (u32x2){pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : log_sum(top, a.scale_log2, ls);
  }
}

}  // namespace

hipError_t launch_chunk_few32(int d, int rows, int blocks, const ChunkArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, blocks), block(64 * kWaves);
  if (d == 128) {
    if (rows == 32) hipLaunchKernelGGL((chunk_few32_kernel<128, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((chunk_few32_kernel<128, 2>), grid, block, 0, st, a);
  } else {
    if (rows == 32) hipLaunchKernelGGL((chunk_few32_kernel<64, 1>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((chunk_few32_kernel<64, 2>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace sparrow
