// Attention of up to 16 rows (new token, query head of the group) of an item by a workgroup of kWaves wavefronts, each with every kWaves-th tile of 16
// keys; their states of a row are merged at the end.  As chunk_few16_kernel (../paged/chunk_attn_few16.hip), whose operands it has: S^T = K Q^T by
// 16x16x32 products, P^T the scores' own registers, V^T by transposing reads.
//
// Tiles go memory -> LDS past the registers, two tiles ahead.  An 8-bit cache's are tiles of 32 keys (the same bytes); their codes become bf16 numbers
// in the operands, K's times its power, V's as they are: V's power multiplies the probability instead, which is exact too.  A 16-byte read of K gives
// a lane its part of two k-steps (columns 16 x .. 16 x + 15 of chunk x, Q^T cut alike), a transposing read of bytes (ds_read_b64_tr_b8: within 16
// lanes, lane i receives byte i % 8 of the 8-byte words addressed by lanes 2 j + i / 8, j = 0..7) V^T of eight keys.  (Products of 8-bit numbers, the
// query as a sum of two e4m3 terms, take as many cycles and no conversion of K, but their sums were off by 2^-15 of the terms' sizes: 2^-24 in bf16.)
//
// Bound by memory where there are many requests: 48 single tokens over up to 8,192, four KV heads of 128, 8 bits, 44.7 us, 231 MB, 5.2 TB/s; a ring of registers
// in the place of LDS 54 -> 67 at that step.  One token over 26,112 10.4 us, of which 4 are the bytes: the rest are the round trips of the plan, the table and the
// first tiles.
#pragma once
#include "serve_tiles.hpp"

namespace sparrow {

template <typename C, int kD, int kWaves> struct FewTiles {
  static constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  static constexpr int kTokens = k8 ? 32 : 16, kRow = kD * (int)sizeof(C), kTileBytes = kTokens * kRow;
  static constexpr int kPowers = k8 ? 256 : 0;             // bytes of a tile's powers
  static constexpr int kAtPowers = kWaves * 4 * kTileBytes, kBytes = kAtPowers + kWaves * 2 * kPowers;     // [wave][K0, V0, K1, V1], [wave][powers 0, 1]
};

__device__ __forceinline__ f32x4 mul32(bf16x8 v, bf16x8 p, f32x4 o) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0); }

// A wavefront's part of an item: its tiles w, w + kWaves, ... of the piece, its lane's row and what that has seen.
struct FewPart {
  int w, n, n_full, t0, t1, pos;     // tiles; those that all rows see whole; the piece's first token, last one seen + 1; the row's position
  const bf16_t *q;                   // the row
  // No other request reads the pages, as far as is known: they need not stay in the caches.  48 single tokens 51 us, otherwise 56; three groups of ten over a
  // prefix that is not read once for them 58 us, otherwise 32.
  bool once;
};
template <int kD> struct FewState {
  f32x4 o[kD / 16];
  float m, l;
  // The reference score moves only when a score of the wavefront's lies more than kSlack above it.
  template <int kN> __device__ __forceinline__ void softmax(const f32x4 (&s)[kN], float (&p)[kN][4], float scale_log2) {
    float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
    for (int k = 1; k < kN; ++k) mx = fmaxf(mx, fmaxf(fmaxf(s[k][0], s[k][1]), fmaxf(s[k][2], s[k][3])));
    if (__builtin_amdgcn_ballot_w64((mx - m) * scale_log2 > kSlack) != 0ull) {
      const float m_new = fmaxf(m, quad_max(mx)), alpha = factor(m, m_new, scale_log2);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < kD / 16; ++db) o[db] *= alpha;
    }
#pragma unroll
    for (int k = 0; k < kN; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[k][i] = fast_exp2((s[k][i] - m) * scale_log2);
      l += (p[k][0] + p[k][1]) + (p[k][2] + p[k][3]);
    }
  }
};

template <int kD, int kWaves>
__device__ __forceinline__ void few_of_bf16(const FewPart &x, const ServePages<bf16_t> &pages, float scale_log2, unsigned char *mine, FewState<kD> &st) {
  constexpr int kTokens = 16, kRow = 2 * kD, kTileBytes = kTokens * kRow;
  constexpr int kDB = kD / 16, kChunks = kRow / 16, kG = kRow / 64, kLoadRows = 64 / kChunks, kLoads = kTokens / kLoadRows;
  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  // Row r's 16-byte chunk x is kept at x ^ swz(r): eight rows read at one chunk, or four groups of four rows read transposed, fall on
  // different banks.
  const auto swz = [](int row) { return kRow == 128 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; };
  const unsigned int mine_at = lds_offset(mine);
  // load j of a tile: rows kLoadRows j + lane / kChunks
  const auto issue = [&](const unsigned char *src, int it, int part) __attribute__((always_inline)) {
    const unsigned char *at = src + pages.place(x.t0 + (x.w + it * kWaves) * kTokens).at;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = kLoadRows * j + lane / kChunks;
      const unsigned int off = row * pages.stride_token + 16u * ((lane % kChunks) ^ swz(row)), to = mine_at + part * kTileBytes + 1024 * j;
      if (x.once) global_to_lds<true>(at, off, to);
      else global_to_lds<false>(at, off, to);
    }
  };
  issue(pages.k, 0, 0);
  issue(pages.v, 0, 1);
  if (x.n > 1) {
    issue(pages.k, 1, 2);
    issue(pages.v, 1, 3);
  }
  u32x4 q[kG];
#pragma unroll
  for (int g = 0; g < kG; ++g) q[g] = ((const u32x4 *)x.q)[4 * g + c4];
  wait_loads<0>();
#pragma unroll
  for (int g = 0; g < kG; ++g) asm volatile("" : "+v"(q[g]));              // (waited for here, and not in the loop)
  const auto step = [&](int it, auto masked) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked)::value;
    const int buf = it & 1;
    const bool more = it + 1 < x.n, more2 = it + 2 < x.n;
    if (more) wait_loads<3 * kLoads>();
    else wait_loads<kLoads>();
    const unsigned char *K = mine + 2 * buf * kTileBytes, *V = K + kTileBytes;
    f32x4 s[1] = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      const u32x4 k = *reinterpret_cast<const u32x4 *>(K + n16 * kRow + (((4 * g + c4) ^ swz(n16)) << 4));
      s[0] = mul32(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[g]), s[0]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more2) issue(pages.k, it + 2, 2 * buf);
    const int t = x.t0 + (x.w + it * kWaves) * kTokens;
    const auto sees = [&](int i) __attribute__((always_inline)) { return t + 4 * c4 + i <= min(x.pos, x.t1 - 1); };
    if constexpr (kMasked) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][i] = sees(i) ? s[0][i] : -INFINITY;
    }
    float p[1][4];
    st.softmax(s, p, scale_log2);
    bf16x4 pb, ones;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      pb[i] = (__bf16)p[0][i];
      if (kMasked) ones[i] = (__bf16)(sees(i) ? 1.f : 0.f);
    }
    if (more2) wait_loads<3 * kLoads>();
    else if (more) wait_loads<2 * kLoads>();
    else wait_loads<0>();
    const int row = 4 * c4 + (n16 >> 2);
    bf16x4 v[kDB];
#pragma unroll
    for (int db = 0; db < kDB; ++db) v[db] = lds_tr(V + row * kRow + (((2 * db + ((n16 >> 1) & 1)) ^ swz(row)) << 4) + 8 * (n16 & 1));
    if constexpr (kMasked) {
      add_masked16(v, pb, ones, st.o);
    } else {
#pragma unroll
      for (int db = 0; db < kDB; ++db) st.o[db] = mul16(v[db], pb, st.o[db]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more2) issue(pages.v, it + 2, 2 * buf + 1);
  };
  int it = 0;
  for (; it < x.n_full; ++it) step(it, std::false_type());
  for (; it < x.n; ++it) step(it, std::true_type());
}

// As add_masked16 (../paged/chunk_attn_16.hpp), of 32 keys and one block of columns.
__device__ __forceinline__ void add_masked32(bf16x8 v, bf16x8 p, bf16x8 seen, f32x4 *o) {
  u32x4 fine = __builtin_bit_cast(u32x4, v), up, down;
  if (__builtin_amdgcn_ballot_w64((not_finite(fine[0]) | not_finite(fine[1]) | not_finite(fine[2]) | not_finite(fine[3])) != 0u) == 0ull) {
    *o = mul32(v, p, *o);
    return;
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    up[i] = ones_of(fine[i], false);
    down[i] = ones_of(fine[i], true);
    fine[i] &= ~no_numbers(fine[i]);
  }
  *o = infinities(mul32(__builtin_bit_cast(bf16x8, fine), p, *o), mul32(__builtin_bit_cast(bf16x8, up), seen, zero),
                  mul32(__builtin_bit_cast(bf16x8, down), seen, zero));
}

template <int kD, int kWaves>
__device__ __forceinline__ void few_of_8bit(const FewPart &x, const ServePages<e4m3_t> &pages, float scale_log2, unsigned char *mine, unsigned char *powers,
                                            FewState<kD> &st) {
  constexpr int kTokens = 32, kRow = kD, kTileBytes = kTokens * kRow, kPowers = FewTiles<e4m3_t, kD, kWaves>::kPowers;
  constexpr int kDB = kD / 16, kChunks = kRow / 16, kLoadRows = 64 / kChunks, kLoads = kTokens / kLoadRows, kReads = kChunks / 4;
  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  // Row r's 16-byte chunk x is kept at x ^ swz(r): eight rows of K read at one chunk, or of V at one chunk transposed (four of either half of the tile),
  // fall on different banks.
  const auto swz_k = [](int row) { return kD == 128 ? row & 7 : (row >> 2) & 1; };
  const auto swz_v = [](int row) { return kD == 128 ? (row & 3) | ((row >> 4) & 1) << 2 : (row >> 4) & 1; };
  const unsigned int mine_at = lds_offset(mine), powers_at = lds_offset(powers);
  // load j of a tile: rows kLoadRows j + lane / kChunks; 16 tokens lie on one page
  const auto token_of = [&](int it) __attribute__((always_inline)) { return x.t0 + (x.w + it * kWaves) * kTokens; };
  const auto issue = [&](const unsigned char *src, const auto &swz, int it, int part) __attribute__((always_inline)) {
    const unsigned char *at[2] = {src + pages.place(token_of(it)).at, src + pages.place(token_of(it) + 16).at};
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = kLoadRows * j + lane / kChunks;
      const unsigned int off = (row & 15) * pages.stride_token + 16u * ((lane % kChunks) ^ swz(row)), to = mine_at + part * kTileBytes + 1024 * j;
      if (x.once) global_to_lds<true>(at[kLoadRows * j / 16], off, to);
      else global_to_lds<false>(at[kLoadRows * j / 16], off, to);
    }
  };
  const auto issue_k = [&](int it) __attribute__((always_inline)) {       // the powers of two tokens a lane, and K
    const int64_t a = pages.place(token_of(it)).token, b = pages.place(token_of(it) + 16).token;
    global_to_lds_4(pages.powers + 2 * ((lane & 8) ? b : a) + 4 * (lane & 7), powers_at + (it & 1) * kPowers);
    issue(pages.k, swz_k, it, 2 * (it & 1));
  };
  const auto issue_v = [&](int it) __attribute__((always_inline)) { issue(pages.v, swz_v, it, 2 * (it & 1) + 1); };
  issue_k(0);
  issue_v(0);
  if (x.n > 1) {
    issue_k(1);
    issue_v(1);
  }
  bf16x8 q[kReads][2];
#pragma unroll
  for (int g = 0; g < kReads; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i) q[g][i] = ((const bf16x8 *)x.q)[2 * (4 * g + c4) + i];
  wait_loads<0>();
#pragma unroll
  for (int g = 0; g < kReads; ++g) asm volatile("" : "+v"(q[g][0]), "+v"(q[g][1]));      // (waited for here, and not in the loop)
  const auto step = [&](int it, auto masked) __attribute__((always_inline)) {
    constexpr bool kMasked = decltype(masked)::value;
    const int buf = it & 1;
    const bool more = it + 1 < x.n, more2 = it + 2 < x.n;
    if (more) wait_loads<3 * kLoads + 1>();
    else wait_loads<kLoads>();
    const unsigned char *K = mine + 2 * buf * kTileBytes, *V = K + kTileBytes, *P = powers + buf * kPowers;
    f32x4 s[2];
    u32x2 pv[2];                                           // K's and V's bytes of tokens 4 c4 + 0..3 of either half
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      pv[k] = *reinterpret_cast<const u32x2 *>(P + 32 * k + 8 * c4);
      const int row = 16 * k + n16;
      const float power = power_of(P[2 * row]);
      s[k] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < kReads; ++g) {
        const u32x4 codes = *reinterpret_cast<const u32x4 *>(K + row * kRow + (((4 * g + c4) ^ swz_k(row)) << 4));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x2 lo = four_of(codes[2 * i], power), hi = four_of(codes[2 * i + 1], power);
          s[k] = mul32(__builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]}), q[g][i], s[k]);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more2) issue_k(it + 2);
    const auto sees = [&](int k, int i) __attribute__((always_inline)) { return token_of(it) + 16 * k + 4 * c4 + i <= min(x.pos, x.t1 - 1); };
    if constexpr (kMasked) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[k][i] = sees(k, i) ? s[k][i] : -INFINITY;
    }
    float p[2][4];
    st.softmax(s, p, scale_log2);
    bf16x8 pb, ones;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pb[4 * k + i] = (__bf16)(p[k][i] * power_in(pv[k][i >> 1], i, true));
        if (kMasked) ones[4 * k + i] = (__bf16)(sees(k, i) ? 1.f : 0.f);
      }
    if (more2) wait_loads<3 * kLoads + 2>();
    else if (more) wait_loads<2 * kLoads + 1>();
    else wait_loads<0>();
    const int j = n16 >> 1, row = 4 * c4 + (j & 3) + 16 * (j >> 2);
    const auto read_v = [&](int db) __attribute__((always_inline)) {
      typedef __attribute__((ext_vector_type(2))) int i32x2;
      const i32x2 codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(V + row * kRow + ((db ^ swz_v(row)) << 4) + 8 * (n16 & 1)));
      const u32x2 lo = four_of((unsigned int)codes[0], 1.f), hi = four_of((unsigned int)codes[1], 1.f);
      return __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]});
    };
#pragma unroll
    for (int db = 0; db < kDB; ++db) {
      if constexpr (kMasked) add_masked32(read_v(db), pb, ones, &st.o[db]);
      else st.o[db] = mul32(read_v(db), pb, st.o[db]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more2) issue_v(it + 2);
  };
  int it = 0;
  for (; it < x.n_full; ++it) step(it, std::false_type());
  for (; it < x.n; ++it) step(it, std::true_type());
}

template <typename C, int kD, int kWaves>
__device__ __forceinline__ void attend_few(const ServeArgs &a, const ServePiece &pc, int idx, int c, unsigned char *lds, float (*ml)[16][2]) {
  using Tiles = FewTiles<C, kD, kWaves>;
  constexpr int kTokens = Tiles::kTokens, kDB = kD / 16, kOut = kD / 4;
  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int R = pc.it.n * a.g;                             // (at most 16: one block)
  const int rho = min(n16, R - 1), i_row = quotient(rho, a.g, a.inv_g);
  const int last_pos = min(pc.it.past + quotient(R - 1, a.g), pc.it.to - 1);
  FewPart x;
  x.w = w;
  x.t0 = pc.t0;
  x.t1 = min(pc.t1, last_pos + 1);
  x.pos = min(pc.it.past + i_row, pc.it.to - 1);
  x.once = a.once != 0;
  x.q = (const bf16_t *)a.q + (int64_t)(pc.it.row0 + i_row) * a.q_row + (int64_t)(c * a.g + rho - i_row * a.g) * kD;
  const int n_tiles = max(x.t1 - x.t0 + kTokens - 1, 0) / kTokens;
  x.n = (n_tiles - w + kWaves - 1) / kWaves;
  const int full = max(min(pc.it.past + 1, x.t1) - x.t0, 0) / kTokens;
  x.n_full = max(full - w + kWaves - 1, 0) / kWaves;
  FewState<kD> st;
  st.m = kNothingSeen;
  st.l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) st.o[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  if (x.n > 0) {
    const ServePages<C> pages = serve_pages<C>(a, pc.it, c);
    unsigned char *mine = lds + w * 4 * Tiles::kTileBytes;
    if constexpr (Tiles::k8) few_of_8bit<kD, kWaves>(x, pages, a.scale_log2, mine, lds + Tiles::kAtPowers + w * 2 * Tiles::kPowers, st);
    else few_of_bf16<kD, kWaves>(x, pages, a.scale_log2, mine, st);
  }
  // ---- merge: states of the wavefronts through LDS
  __syncthreads();
  unsigned char *states = lds + w * 16 * kD * 4;
  const float l = quad_sum(st.l);
  if (c4 == 0) { ml[w][n16][0] = st.m; ml[w][n16][1] = l; }
#pragma unroll
  for (int db = 0; db < kDB; ++db)                         // elements 16 db + 4 c4 + 0..3
    *reinterpret_cast<f32x4 *>(states + (n16 * kOut + ((4 * db + c4) ^ n16)) * 16) = st.o[db];
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
    else sum /= Tiles::k8 ? ls * kLowered : ls;
    *reinterpret_cast<u32x2 *>((bf16_t *)a.out + at * kD + 4 * chunk) = (u32x2){pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : log_sum(top, a.scale_log2, ls);
  }
}

}  // namespace sparrow
