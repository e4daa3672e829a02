// Attention of up to 16 rows (new token, query head of the group) of an item by a workgroup of eight wavefronts, each with every eighth tile of 16
// keys; their states of a row are merged at the end.  As chunk_few16_kernel (../paged/chunk_attn_few16.hip), whose operands it has: S^T = K Q^T by
// 16x16x32 products, P^T the scores' own registers, V^T by transposing reads.
//
// A bf16 cache's tiles go memory -> LDS past the registers, two tiles ahead.  An 8-bit cache's go through registers, kAhead tiles ahead, and are
// written to LDS as the bf16 numbers that they are, so that scores and outputs see no powers.
#pragma once
#include "serve_tiles.hpp"

namespace sparrow {

constexpr int kServeWaves = 8;

template <typename C, int kD> struct FewTiles {
  static constexpr int kTokens = 16, kRow = 2 * kD, kTileBytes = kTokens * kRow, kBytes = kServeWaves * 4 * kTileBytes;
};

template <typename C, int kD>
__device__ __forceinline__ void attend_few(const ServeArgs &a, const ServePiece &pc, int idx, int c, unsigned char *lds, float (*ml)[16][2]) {
  constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  constexpr int kWaves = kServeWaves, kTokens = FewTiles<C, kD>::kTokens, kRow = FewTiles<C, kD>::kRow, kTileBytes = FewTiles<C, kD>::kTileBytes;
  constexpr int kDB = kD / 16, kChunks = kRow / 16, kG = kRow / 64, kLoadRows = 64 / kChunks, kLoads = kTokens / kLoadRows, kOut = kD / 4;
  constexpr int kAhead = 4, kCodes = kD / 64;              // 8 bits: tiles in flight; 16-byte loads of a tile
  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R = pc.it.n * a.g;                             // (at most 16: one block)
  const ServePages<C> pages = serve_pages<C>(a, pc.it, c);
  const int last_pos = min(pc.it.past + quotient(R - 1, a.g), pc.it.to - 1), first_pos = pc.it.past;
  const int t1 = min(pc.t1, last_pos + 1);
  const int n_tiles = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;
  const int n = (n_tiles - w + kWaves - 1) / kWaves;       // of this wavefront: w, w + kWaves, ...
  unsigned char *mine = lds + w * 4 * kTileBytes;
  // Row r's 16-byte chunk x is kept at x ^ swz(r): eight rows read at one chunk, or four groups of four rows read transposed, fall on
  // different banks.
  const auto swz = [](int row) { return kRow == 128 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; };

  const int rho = min(n16, R - 1), i_row = quotient(rho, a.g, a.inv_g), pos = min(pc.it.past + i_row, pc.it.to - 1);
  f32x4 o[kDB];
  float m = kNothingSeen, l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) o[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    u32x4 q[kG];
    const auto load_q = [&]() __attribute__((always_inline)) {
      const bf16_t *at = (const bf16_t *)a.q + (int64_t)(pc.it.row0 + i_row) * a.q_row + (int64_t)(c * a.g + rho - i_row * a.g) * kD;
#pragma unroll
      for (int g = 0; g < kG; ++g) q[g] = ((const u32x4 *)at)[4 * g + c4];
    };
    // of the tile at K, from token t on: scores and softmax, then the output
    float p[4], seen[4];
    const auto scores = [&](const unsigned char *K, int t, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        const u32x4 k = *reinterpret_cast<const u32x4 *>(K + n16 * kRow + (((4 * g + c4) ^ swz(n16)) << 4));
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[g]), s, 0, 0, 0);
      }
      if constexpr (kMasked) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool vis = t + 4 * c4 + i <= min(pos, t1 - 1);
          s[i] = vis ? s[i] : -INFINITY;
          seen[i] = vis ? 1.f : 0.f;
        }
      }
      return s;
    };
    // the row's reference score moves only when a score of the wavefront's lies more than kSlack above it
    const auto softmax = [&](f32x4 s) __attribute__((always_inline)) {
      const float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      if (__builtin_amdgcn_ballot_w64((mx - m) * a.scale_log2 > kSlack) != 0ull) {
        const float m_new = fmaxf(m, quad_max(mx)), alpha = factor(m, m_new, a.scale_log2);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < kDB; ++db) o[db] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = fast_exp2((s[i] - m) * a.scale_log2);
      l += (p[0] + p[1]) + (p[2] + p[3]);
    };
    const auto output = [&](const unsigned char *V, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      const int row = 4 * c4 + (n16 >> 2);
      bf16x4 v[kDB], pb, ones;
#pragma unroll
      for (int db = 0; db < kDB; ++db) v[db] = lds_tr(V + row * kRow + (((2 * db + ((n16 >> 1) & 1)) ^ swz(row)) << 4) + 8 * (n16 & 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pb[i] = (__bf16)p[i];
        if (kMasked) ones[i] = (__bf16)seen[i];
      }
      if constexpr (kMasked) {
        add_masked16(v, pb, ones, o);
      } else {
#pragma unroll
        for (int db = 0; db < kDB; ++db) o[db] = mul16(v[db], pb, o[db]);
      }
    };
    // the tiles that all rows see whole, then the others
    const int full = max(min(first_pos + 1, t1) - pc.t0, 0) / kTokens, n_full = max(full - w + kWaves - 1, 0) / kWaves;
    if constexpr (!k8) {
      const unsigned int mine_at = lds_offset(mine);
      // load j of a tile: rows kLoadRows j + lane / kChunks
      const auto issue = [&](const unsigned char *src, int tile, int part) __attribute__((always_inline)) {
        const unsigned char *at = src + pages.place(pc.t0 + tile * kTokens).at;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int row = kLoadRows * j + lane / kChunks;
          global_to_lds<true>(at, row * pages.stride_token + 16u * ((lane % kChunks) ^ swz(row)), mine_at + part * kTileBytes + 1024 * j);
        }
      };
      issue(pages.k, w, 0);
      issue(pages.v, w, 1);
      if (n > 1) {
        issue(pages.k, w + kWaves, 2);
        issue(pages.v, w + kWaves, 3);
      }
      load_q();
      wait_loads<0>();
      const auto step = [&](int it, auto masked) __attribute__((always_inline)) {
        const int buf = it & 1;
        const bool more = it + 1 < n, more2 = it + 2 < n;
        if (more) wait_loads<3 * kLoads>();
        else wait_loads<kLoads>();
        const unsigned char *K = mine + 2 * buf * kTileBytes;
        const f32x4 s = scores(K, pc.t0 + (w + it * kWaves) * kTokens, masked);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more2) issue(pages.k, w + (it + 2) * kWaves, 2 * buf);
        softmax(s);
        if (more2) wait_loads<3 * kLoads>();
        else if (more) wait_loads<2 * kLoads>();
        else wait_loads<0>();
        output(K + kTileBytes, masked);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more2) issue(pages.v, w + (it + 2) * kWaves, 2 * buf + 1);
      };
      int it = 0;
      for (; it < n_full; ++it) step(it, std::false_type());
      for (; it < n; ++it) step(it, std::true_type());
    } else {
      // A lane has 16 codes of row kCodeRows j + lane / kCodeLanes, and that row's powers.
      constexpr int kCodeLanes = kD / 16, kCodeRows = 64 / kCodeLanes;
      u32x4 kc[kAhead][kCodes], vc[kAhead][kCodes];
      unsigned short pw[kAhead][kCodes];
      const auto fetch = [&](int tile, int u) __attribute__((always_inline)) {
        const auto place = pages.place(pc.t0 + tile * kTokens);
#pragma unroll
        for (int j = 0; j < kCodes; ++j) {
          const int row = kCodeRows * j + lane / kCodeLanes;
          const unsigned int off = row * pages.stride_token + 16u * (lane % kCodeLanes);
          kc[u][j] = __builtin_nontemporal_load((const u32x4 *)(pages.k + place.at + off));
          vc[u][j] = __builtin_nontemporal_load((const u32x4 *)(pages.v + place.at + off));
          pw[u][j] = pages.powers[place.token + row];
        }
      };
      const auto store = [&](unsigned char *to, const u32x4 *codes, const unsigned short *powers, int shift) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kCodes; ++j) {
          const int row = kCodeRows * j + lane / kCodeLanes;
          const float power = power_of((powers[j] >> shift) & 0xffu);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x2 x = four_of(codes[j][2 * h], power), y = four_of(codes[j][2 * h + 1], power);
            *reinterpret_cast<u32x4 *>(to + row * kRow + (((2 * (lane % kCodeLanes) + h) ^ swz(row)) << 4)) = (u32x4){x[0], x[1], y[0], y[1]};
          }
        }
      };
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (u < n) fetch(w + u * kWaves, u);
      load_q();
      const auto step = [&](int it, int u, auto masked) __attribute__((always_inline)) {
        store(mine, kc[u], pw[u], 0);
        store(mine + kTileBytes, vc[u], pw[u], 8);
        if (it + kAhead < n) fetch(w + (it + kAhead) * kWaves, u);
        asm volatile("" ::: "memory");
        softmax(scores(mine, pc.t0 + (w + it * kWaves) * kTokens, masked));
        output(mine + kTileBytes, masked);
        asm volatile("" ::: "memory");
      };
      for (int it = 0; it < n; it += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (it + u < n_full) step(it + u, u, std::false_type());
          else if (it + u < n) step(it + u, u, std::true_type());
        }
      }
    }
  }
  // ---- merge: states of the wavefronts through LDS
  __syncthreads();
  unsigned char *states = lds + w * 16 * kD * 4;
  l = quad_sum(l);
  if (c4 == 0) { ml[w][n16][0] = m; ml[w][n16][1] = l; }
#pragma unroll
  for (int db = 0; db < kDB; ++db)                         // elements 16 db + 4 c4 + 0..3
    *reinterpret_cast<f32x4 *>(states + (n16 * kOut + ((4 * db + c4) ^ n16)) * 16) = o[db];
  __syncthreads();
  if (!pc.direct && idx >= a.slots) return;                // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) << a.block_shift;
  for (int x = threadIdx.x; x < R * kOut; x += 64 * kWaves) {
    const int r = x / kOut, chunk = x % kOut;
    float top = ml[0][r][0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) top = fmaxf(top, ml[k][r][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float ls = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = factor(ml[k][r][0], top, a.scale_log2);
      ls = fmaf(ml[k][r][1], f, ls);
      sum += *reinterpret_cast<const f32x4 *>(lds + k * 16 * kD * 4 + (r * kOut + (chunk ^ (r & 15))) * 16) * f;
    }
    if (!pc.direct) {
      *reinterpret_cast<f32x4 *>(a.part_o + (part + r) * kD + 4 * chunk) = sum;
      if (chunk == 0) {
        a.part_ml[2 * (part + r)] = top;
        a.part_ml[2 * (part + r) + 1] = ls;
      }
      continue;
    }
    const int i = quotient(r, a.g, a.inv_g);
    const int64_t at = (int64_t)(pc.it.row0 + i) * a.Hq + c * a.g + r - i * a.g;
    const bool none = pc.it.past + i < 0;
    if (none) sum = (f32x4){0.f, 0.f, 0.f, 0.f};
    else sum /= ls;
    *reinterpret_cast<u32x2 *>((bf16_t *)a.out + at * kD + 4 * chunk) = (u32x2){pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : log_sum(top, a.scale_log2, ls);
  }
}

}  // namespace sparrow
