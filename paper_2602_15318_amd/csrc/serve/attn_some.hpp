// Attention of 17 to 64 rows (new token, query head of the group) of a request by eight wavefronts: chains of draft tokens.  As attn_few.hpp, with products of 32 rows: a wavefront has up to 32 rows and every eighth tile of 32 keys, or, of more rows, half of the
// rows and every fourth tile; the states of a row are merged at the end.
//
// S^T = K Q^T by 32x32x16 products, P^T the scores' own registers (../paged/chunk_attn_mfma.hpp).  Tiles go memory -> LDS past the registers.  A bf16 cache's
// have one place of K and one of V a wavefront: K of the next is asked for behind the scores, V behind the output, and the other wavefronts
// fill the time.  An 8-bit cache's have two, and their codes lie in LDS as they come; they become bf16 numbers in the operands, K's times its power, V's as they are, V's power in the probability.  A 16-byte read of K is a lane's part of two k-steps, Q^T cut alike; V^T of
// eight keys is one transposing read of bytes (attn_few.hpp).
//
// Bound by waiting: a workgroup fills a compute unit's LDS, two wavefronts a SIMD.  Twelve chains of 8 over up to 8,000, 28 and 4 heads of 128, 8 bits, 35.4 us, 29 of
// them here: the vector ALU works some 11 (of more than 32 rows, each half converts a tile for itself), the matrix cores 4, and 77 MB are fetched where 52 are
// held.  Over bf16 pages, twice the bytes, 35.0.  In blocks of 256 rows 44.4 either way; one chain over 26,112 22.3 (24.7), with heads of 64 eight chains 27.7
// (36.4).
#pragma once
#include "attn_few.hpp"

namespace sparrow {

template <typename C, int kD>
__device__ __forceinline__ void attend_some(const ServeArgs &a, const ServePiece &pc, int idx, int c, unsigned char *lds, float (*ml)[32][2]) {
  constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  constexpr int kWaves = 8, kTokens = 32, kRow = kD * (int)sizeof(C), kTileBytes = kTokens * kRow, kPlace = 4 * kTokens * kD;
  constexpr int kPowers = FewTiles<e4m3_t, kD, kWaves>::kPowers, kDB = kD / 32, kChunks = kRow / 16, kLoadRows = 64 / kChunks, kLoads = kTokens / kLoadRows;
  constexpr int kReads = kD / 32, kOut = kD / 4;
  const int lane = threadIdx.x & 63, n32 = lane & 31, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R = pc.it.n * a.g, shift = R > 32 ? 1 : 0, half = w & shift, stream = w >> shift, streams = kWaves >> shift;
  const int rho = min(32 * half + n32, R - 1), i_row = quotient(rho, a.g, a.inv_g);
  const int t1 = min(pc.t1, min(pc.it.past + pc.it.n, pc.it.to)), last_seen = min(min(pc.it.past + i_row, pc.it.to - 1), t1 - 1);
  const auto mine_of = [&](int tiles) { return max(tiles - stream + streams - 1, 0) >> (3 - shift); };
  const int n = mine_of(max(t1 - pc.t0 + kTokens - 1, 0) / kTokens), n_full = mine_of(max(min(pc.it.past + 1, t1) - pc.t0, 0) / kTokens);
  unsigned char *const mine = lds + w * kPlace, *const powers = lds + kWaves * kPlace + w * 2 * kPowers;
  f32x16 o[kDB];
  float m = kNothingSeen, l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) o[db] = (f32x16){0.f};
  if (n > 0) {
    const ServePages<C> pages = serve_pages<C>(a, pc.it, c);
    // Row r's 16-byte chunk x is kept at x ^ swz(r): eight rows of K read at one chunk, or of V at two neighbours transposed (0..3 and 8..11 of 16), fall on
    // different banks.
    const auto swz_k = [](int row) { return !k8 ? Tile<kD>::swz_k(row) : kD == 128 ? row & 7 : (row >> 2) & 1; };
    const auto swz_v = [](int row) { return !k8 ? Tile<kD>::swz_v(row) : kD == 128 ? ((row >> 1) & 1) << 1 | ((row >> 3) & 1) << 2 : ((row >> 3) & 1) << 1; };
    const unsigned int mine_at = lds_offset(mine), powers_at = lds_offset(powers);
    const auto token_of = [&](int it) __attribute__((always_inline)) { return pc.t0 + (stream + it * streams) * kTokens; };
    const auto issue = [&](const unsigned char *src, const auto &swz, int it, int part) __attribute__((always_inline)) {
      const unsigned char *at[2] = {src + pages.place(token_of(it)).at, src + pages.place(token_of(it) + 16).at};       // 16 tokens lie on one page
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = kLoadRows * j + lane / kChunks;
        global_to_lds<false>(at[kLoadRows * j / 16], (row & 15) * pages.stride_token + 16u * ((lane % kChunks) ^ swz(row)), mine_at + part * kTileBytes + 1024 * j);
      }
    };
    const auto issue_k = [&](int it) __attribute__((always_inline)) {     // the powers of two tokens a lane, and K
      if constexpr (k8) {
        const int64_t x = pages.place(token_of(it)).token, y = pages.place(token_of(it) + 16).token;
        global_to_lds_4(pages.powers + 2 * ((lane & 8) ? y : x) + 4 * (lane & 7), powers_at + (it & 1) * kPowers);
      }
      issue(pages.k, swz_k, it, k8 ? 2 * (it & 1) : 0);
    };
    const auto issue_v = [&](int it) __attribute__((always_inline)) { issue(pages.v, swz_v, it, k8 ? 2 * (it & 1) + 1 : 1); };
    issue_k(0);
    issue_v(0);
    if (k8 && n > 1) {
      issue_k(1);
      issue_v(1);
    }
    bf16x8 q[kReads][2];
    const bf16x8 *from = (const bf16x8 *)((const bf16_t *)a.q + (int64_t)(pc.it.row0 + i_row) * a.q_row + (int64_t)(c * a.g + rho - i_row * a.g) * kD);
#pragma unroll
    for (int g = 0; g < kReads; ++g)
#pragma unroll
      for (int i = 0; i < 2; ++i) q[g][i] = from[k8 ? 2 * (2 * g + h) + i : 2 * (2 * g + i) + h];
    wait_loads<0>();
#pragma unroll
    for (int g = 0; g < kReads; ++g) asm volatile("" : "+v"(q[g][0]), "+v"(q[g][1]));    // (waited for here, and not in the loop)
    const auto step = [&](int it, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
      int l64 = lane;
      if constexpr (kMasked) asm volatile("" : "+v"(l64));  // (worked out again in the last tiles: kept, there are too few registers)
      const int n32 = l64 & 31, h = l64 >> 5;
      const int buf = k8 ? it & 1 : 0, seen = last_seen - token_of(it) - 4 * h;
      const bool more = it + 1 < n, more2 = it + 2 < n;
      if (k8 && more) wait_loads<3 * kLoads + 1>();
      else wait_loads<kLoads>();
      const unsigned char *K = mine + 2 * buf * kTileBytes, *V = K + kTileBytes, *P = powers + buf * kPowers;
      f32x16 s = (f32x16){0.f};
      u32x2 pv[4];                                         // K's and V's bytes of keys 8 j + 4 h + 0..3
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if constexpr (k8) pv[j] = *reinterpret_cast<const u32x2 *>(P + 16 * j + 8 * h);
      const float power = k8 ? power_of(P[2 * n32]) : 1.f;
#pragma unroll
      for (int g = 0; g < kReads; ++g) {
        if constexpr (!k8) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_b128(K + (k_at<kD>(l64) ^ (2 * g + i) << 5)), q[g][i], s, 0, 0, 0);
          continue;
        }
        const u32x4 codes = *reinterpret_cast<const u32x4 *>(K + n32 * kRow + (((2 * g + h) ^ swz_k(n32)) << 4));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x2 lo = four_of(codes[2 * i], power), hi = four_of(codes[2 * i + 1], power);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]}), q[g][i], s, 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (k8 ? more2 : more) issue_k(it + (k8 ? 2 : 1));
      if constexpr (kMasked) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) <= seen ? s[e] : -INFINITY;
      }
      // the reference score moves only when a score of the wavefront's lies more than kSlack above it
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; e += 3) mx = fmaxf(fmaxf(fmaxf(mx, s[e]), s[e + 1]), s[e + 2]);
      if (__builtin_amdgcn_ballot_w64((mx - m) * a.scale_log2 > kSlack) != 0ull) {
        const float m_new = fmaxf(m, pair_max(mx)), alpha = factor(m, m_new, a.scale_log2);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int db = 0; db < kDB; ++db) o[db] *= alpha;
      }
      bf16x8 pb[2], ones[2];
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = fast_exp2((s[e] - m) * a.scale_log2);
        sum[e & 1] += p;
        pb[e >> 3][e & 7] = (__bf16)(k8 ? p * power_in(pv[e >> 2][(e & 3) >> 1], e, true) : p);
        if (kMasked) ones[e >> 3][e & 7] = (__bf16)(8 * (e >> 2) + (e & 3) <= seen ? 1.f : 0.f);
      }
      l += sum[0] + sum[1];
      if (!more) wait_loads<0>();
      else if (!k8) wait_loads<kLoads>();
      else if (more2) wait_loads<3 * kLoads + 2>();
      else wait_loads<2 * kLoads + 1>();
      const int j = (l64 & 15) >> 1, of_16 = 4 * h + (j & 3) + 8 * (j >> 2), which = (l64 >> 4) & 1;
      const auto read_v = [&](int st, int db) __attribute__((always_inline)) {
        if constexpr (!k8) return read_vt<kD>(V + (vt_at<kD>(l64) ^ db << 6), st);
        typedef __attribute__((ext_vector_type(2))) int i32x2;
        const int row = 16 * st + of_16;
        const i32x2 codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) i32x2 *)(V + row * kRow + (((2 * db + which) ^ swz_v(row)) << 4) + 8 * (l64 & 1)));
        const u32x2 lo = four_of((unsigned int)codes[0], 1.f), hi = four_of((unsigned int)codes[1], 1.f);
        return __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]});
      };
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        if constexpr (kMasked) {
          bf16x8 v[kDB];
#pragma unroll
          for (int db = 0; db < kDB; ++db) v[db] = read_v(st, db);
          add_masked(v, pb[st], ones[st], o);
        } else {
#pragma unroll
          for (int db = 0; db < kDB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(st, db), pb[st], o[db], 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (k8 ? more2 : more) issue_v(it + (k8 ? 2 : 1));
    };
    int it = 0;
    for (; it < n_full; ++it) step(it, std::false_type());
    for (; it < n; ++it) step(it, std::true_type());
  }
  // ---- merge: states of the wavefronts through LDS, each in the place of its tiles; rows of kD numbers, 16-byte chunks swizzled by the row
  const float lsum = pair_sum(l);
  if (h == 0) {
    ml[w][n32][0] = m;
    ml[w][n32][1] = lsum;
  }
#pragma unroll
  for (int db = 0; db < kDB; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4 *>(mine + (n32 * kOut + ((8 * db + 2 * j + h) ^ (n32 & (kOut - 1)))) * 16) =
          (f32x4){o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]};
  __syncthreads();
  if (!pc.direct && idx >= a.slots) return;                // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) << a.block_shift;
  for (int x = threadIdx.x; x < R * kOut; x += 64 * kWaves) {
    const int r = x / kOut, chunk = x % kOut, n = r & 31, first = r >> 5;                // (its wavefronts: first, first + 2, ... of more than 32 rows)
    float top = ml[first][n][0];
    for (int k = 1; k < streams; ++k) top = fmaxf(top, ml[(k << shift) + first][n][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float ls = 0.f;
    for (int k = 0; k < streams; ++k) {
      const int wave = (k << shift) + first;
      const float f = factor(ml[wave][n][0], top, a.scale_log2);
      ls = fmaf(ml[wave][n][1], f, ls);
      sum += *reinterpret_cast<const f32x4 *>(lds + wave * kPlace + (n * kOut + (chunk ^ (n & (kOut - 1)))) * 16) * f;
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
    else sum /= k8 ? ls * kLowered : ls;
    *reinterpret_cast<u32x2 *>((bf16_t *)a.out + at * kD + 4 * chunk) = (u32x2){pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : log_sum(top, a.scale_log2, ls);
  }
}

}  // namespace sparrow
