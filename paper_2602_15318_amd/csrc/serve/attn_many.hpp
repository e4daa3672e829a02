// Attention of more rows of an item: blocks of up to 256 rows (new token, query head of the group), 32 per wavefront, K and V tiles of 64 keys that
// the workgroup shares.  As chunk_many_kernel (../paged/chunk_attn_many.hip): wavefronts w and w + 4 share a SIMD and run half a step apart, one in
// the products of a step (scores of a tile, output of the tile before) while the other is in its softmax; four tiles of K and of V in LDS.
//
// A bf16 cache's tiles go memory -> LDS past the registers.  An 8-bit cache's are asked for a step ahead into registers, made the bf16 numbers that they
// are in the softmax's half step, 1/8 by each wavefront, and written to LDS.
//
// Probabilities are rounded to bf16 for the output's product, half a step 2^-9 to 2^-8 of a term; the row's sum takes them unrounded.
//
// Bound by the matrix cores beside the exponentials: 2,048 tokens over 26,112, 28 and 4 heads of 128, 630 us in bf16 and 667 in 8 bits (1.17 and 1.10 PFLOP/s;
// a product of 8,192^3 on that card 1.27; up to 650 and 716 on others), matrix cores busy 45 to 57 % of the cycles by the card's clock.  With heads of 64 a tile has the same softmax for half the
// products.  A piece of a prefix (224 rows, 576 tokens) takes some 10 us beside its tiles: the first loads, and up to 128 KB of partial output.
#pragma once
#include "serve_tiles.hpp"

namespace sparrow {

template <int kD> struct ManyTiles {
  static constexpr int kTokens = 64, kStages = 4, kTileBytes = kTokens * kD * 2;
  static constexpr int kBytes = 2 * kStages * kTileBytes;  // K tiles, V tiles
};

template <typename C, int kD>
__device__ __forceinline__ void attend_many(const ServeArgs &a, const ServePiece &pc, int idx, int c, unsigned char *lds, int *flags) {
  constexpr bool k8 = std::is_same<C, e4m3_t>::value;
  using Tiles = ManyTiles<kD>;
  constexpr int kTokens = Tiles::kTokens, kStages = Tiles::kStages, kTileBytes = Tiles::kTileBytes;
  constexpr int kDB = kD / 32, kKS = kD / 16, kHalf = kKS / 2;
  // The requests in the half step that has time left, the vector one with heads of 128, the matrix one with heads of 64.
  constexpr bool kLate = kD == 128;
  // Tiles that some rows do not see whole need care where V holds what is no number: 0 times it is none.  An 8-bit cache's tiles come through registers, so
  // that every wavefront can tell of its rows, and with heads of 128 such tiles without one are taken as all others are, their weights 0 where nothing is
  // seen: 256 tokens over 8,192 55.0 -> 51.2 us, three chunks of 60 24.5 -> 22.9.  (With heads of 64, 17.9 instead of 18.9 for a chunk of 75, but 75.5
  // instead of 72.5 for one of 777 beside 8 tokens; bf16 tiles read again for it 638 -> 659 for 2,048 over 26,112.)
  constexpr bool kOneLoop = k8 && kD == 128;
  constexpr int kLoads = 8 / Tile<kD>::kLoadRows;          // of a wavefront: eight rows of a tile
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ServePages<C> pages = serve_pages<C>(a, pc.it, c);
  const int R = pc.it.n * a.g, rho0 = pc.block << a.block_shift, block_rows = 1 << a.block_shift;
  const bool have = 32 * w < min(block_rows, R - rho0);    // the wavefront has rows
  // this lane's row, and how far the block's rows see
  const int rho = min(rho0 + min(32 * w, block_rows - 1) + (lane & 31), R - 1);
  const int i_row = quotient(rho, a.g, a.inv_g), head = c * a.g + rho - i_row * a.g;
  const int pos = min(pc.it.past + i_row, pc.it.to - 1);
  const int last_pos = min(pc.it.past + quotient(min(rho0 + block_rows, R) - 1, a.g), pc.it.to - 1);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;
  // tiles that all rows of the block see whole
  const int n_full = min(n, max(min(t1, pc.it.past + quotient(rho0, a.g) + 1) - pc.t0, 0) / kTokens);

  // About scaled points r below 2^20 an exponent is one operation, fma(score, scale, -r): the weights are then 2^c of those about m, c what
  // the rounding of r took off (2^-5 at most), which is taken out where the states leave the workgroup.  Farther points, and a row that has seen
  // nothing, let every score past their limit and into the branch of the points that move, which takes the difference first.
  const auto far = [&](float r) __attribute__((always_inline)) { return fabsf(r) >= 0x1p20f; };
  const auto excess = [&](float m) __attribute__((always_inline)) {
    const float r = m * a.scale_log2;
    return far(r) ? 0.f : fmaf(m, a.scale_log2, -r);
  };
  f32x16 o[kDB];
  float m = kNothingSeen, r = kNothingSeen, limit = -INFINITY, l = 0.f;
#pragma unroll
  for (int db = 0; db < kDB; ++db) o[db] = (f32x16){0.f};
  if (n > 0) {
    const auto place = [&](int tile) __attribute__((always_inline)) { return pages.place(pc.t0 + min(tile, n - 1) * kTokens + 8 * w); };
    using Place = typename ServePages<C>::Place;
    const auto stage = [&](int t) { return t & (kStages - 1); };
    // ---- bf16: straight to LDS
    const unsigned int lds0 = lds_offset(lds) + 1024 * kLoads * w;
    unsigned int from_k[kLoads], from_v[kLoads];
    if constexpr (!k8) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = Tile<kD>::kLoadRows * j;
        from_k[j] = row * pages.stride_token + Tile<kD>::k_from(lane, 8 * w + row, pages.stride_token);
        from_v[j] = row * pages.stride_token + Tile<kD>::v_from(lane, 8 * w + row, pages.stride_token);
      }
    }
    const auto load_k = [&](Place at, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) global_to_lds<false>(pages.k + at.at, from_k[j], lds0 + stage(t) * kTileBytes + 1024 * j);
    };
    const auto load_v = [&](Place at, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) global_to_lds<false>(pages.v + at.at, from_v[j], lds0 + (kStages + stage(t)) * kTileBytes + 1024 * j);
    };
    // ---- 8 bits: kD / 8 codes of row 8 w + lane / 8
    typedef __attribute__((ext_vector_type(kD / 32))) unsigned int Codes;
    const int row = 8 * w + lane / 8;
    const unsigned int off = (lane / 8) * pages.stride_token + (kD / 8) * (lane % 8);
    const auto fetch = [&](const unsigned char *src, Place at) __attribute__((always_inline)) { return *(const Codes *)(src + at.at + off); };
    const auto powers = [&](Place at) __attribute__((always_inline)) { return pages.powers_of(at, lane / 8); };
    const auto store = [&](Codes x, unsigned int bytes, bool is_v, int t) __attribute__((always_inline)) {
      const float p = power_in(bytes, lane / 8, is_v);
      unsigned char *to = lds + ((is_v ? kStages : 0) + stage(t)) * kTileBytes;
#pragma unroll
      for (int i = 0; i < kD / 64; ++i) {                  // 16 bytes of bf16: eight codes
        const u32x2 y = four_of(x[2 * i], p), z = four_of(x[2 * i + 1], p);
        const int chunk = kD / 64 * (lane % 8) + i;
        *reinterpret_cast<u32x4 *>(to + (is_v ? Tile<kD>::v(row, chunk) : Tile<kD>::k(row, chunk))) = (u32x4){y[0], y[1], z[0], z[1]};
        if (kOneLoop && is_v && t >= n_full) {             // (before the barrier that gives the tile to the others)
          const unsigned int any = not_finite(y[0]) | not_finite(y[1]) | not_finite(z[0]) | not_finite(z[1]);
          if (__builtin_amdgcn_ballot_w64(any != 0u) != 0ull) flags[w] = 1;
        }
      }
    };
    if constexpr (kOneLoop) flags[w] = 0;
    Codes kc, vc;
    unsigned int kp = 0u, vp = 0u;

    const Place p0 = place(0), p1 = place(1), p2 = place(2);
    if constexpr (!k8) {
      load_k(p0, 0);
      load_v(p0, 0);
      load_k(p1, 1);
      load_v(p1, 1);
      load_k(p2, 2);
    } else {
      const Codes k0 = fetch(pages.k, p0), v0 = fetch(pages.v, p0), k1 = fetch(pages.k, p1), v1 = fetch(pages.v, p1);
      const Codes k2 = fetch(pages.k, p2);
      const unsigned int b0 = powers(p0), b1 = powers(p1);
      vc = fetch(pages.v, p2);
      vp = powers(p2);
      const Place p3 = place(3);
      kc = fetch(pages.k, p3);
      kp = powers(p3);
      store(k0, b0, false, 0);
      store(v0, b0, true, 0);
      store(k1, b1, false, 1);
      store(v1, b1, true, 1);
      store(k2, vp, false, 2);
    }
    bf16x8 q[kKS];
    {
      const unsigned char *at = (const unsigned char *)a.q + 2 * ((int64_t)(pc.it.row0 + i_row) * a.q_row + (int64_t)head * kD) + 16 * h;
#pragma unroll
      for (int ks = 0; ks < kKS; ++ks) q[ks] = *(const bf16x8 *)(at + 32 * ks);
    }
    // Half steps of tile t: A(t), its scores (and the output of tile t - 1), then B(t), its softmax; a barrier ends each.  A(t) or B(t) asks for K of
    // tile t + 3 and V of t + 2, whose places A(t - 1) was the last to read; a wavefront ends B(t) when all but its last requests are done, those of this
    // step: K of t + 2 and V of t + 1 are there before either half of the workgroup begins A(t + 1).  8 bits: B(t) writes K of t + 3 and V of t + 2,
    // asked for in B(t - 1), and asks for their successors.
    Place at_v = k8 ? place(3) : p2, at_k = place(k8 ? 4 : 3);
    if constexpr (!k8) wait_loads<0>();
    barrier();
    if (w >= 4) barrier();                                 // half a step behind
    const auto request = [&](int t) __attribute__((always_inline)) {
      load_k(at_k, t + 3);
      load_v(at_v, t + 2);
    };
    const auto begin_a = [&](int t) __attribute__((always_inline)) {
      if constexpr (!k8 && !kLate) request(t);
    };
    const auto begin_b = [&](int t) __attribute__((always_inline)) {
      if constexpr (!k8) {
        if (kLate) request(t);
        at_v = at_k;
        at_k = place(t + 4);
      }
    };
    // (8 bits behind the softmax: before it the chunk of 2,048 tokens over 26,112 takes 781 us instead of 685)
    const auto end_b = [&](int t) __attribute__((always_inline)) {
      if constexpr (!k8) {
        wait_loads<2 * kLoads>();
      } else {
        asm volatile("" : "+v"(kp), "+v"(vp));             // (what is made of them is made here: earlier, the loads would be waited for earlier)
        store(kc, kp, false, t + 3);
        store(vc, vp, true, t + 2);
        vc = fetch(pages.v, at_v);
        vp = kp;
        kc = fetch(pages.k, at_k);
        kp = powers(at_k);
        at_v = at_k;
        at_k = place(t + 5);
      }
      barrier();
    };
    if (!have) {
      begin_a(0);
      barrier();
      for (int t = 0; t < n; ++t) {
        begin_b(t);
        end_b(t);
        begin_a(t + 1);
        barrier();
      }
    } else {
      f32x16 s[2];
      bf16x8 pb[4], kf[2][kHalf];                          // kf: the first half of the columns of the next tile's K
      const auto tile = [&](int t, int stage0, int at) __attribute__((always_inline)) {
        at += (stage0 + stage(t)) * kTileBytes;
        asm volatile("" : "+v"(at));                       // (worked out here: kept, the offsets cost more registers than there are)
        return at;
      };
      const auto read_k = [&](int at, int ks0, bf16x8 (*k)[kHalf]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kHalf; ++ks)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) k[kb][ks] = lds_b128(lds + (at ^ (ks0 + ks) << 5) + 32 * kb * Tile<kD>::kRow);
      };
      const auto multiply = [&](int ks0, bf16x8 (*k)[kHalf]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kHalf; ++ks)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][ks], q[ks0 + ks], s[kb], 0, 0, 0);
      };
      const auto read_v = [&](int at, int db, bf16x8 *v) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 4; ++st) v[st] = read_vt<kD>(lds + (at ^ db << 6), st);
      };
      // the scores' exponentials about the row's reference score, which moves only when a score of the wavefront's lies more than
      // kSlack above it
      const auto softmax = [&]() __attribute__((always_inline)) {
        float x[2][16];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[kb][e] = fmaf(s[kb][e], a.scale_log2, -r);
        float top = fmaxf(x[0][0], x[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, x[0][e]), x[1][e]);
        if (__builtin_amdgcn_ballot_w64(top > limit) != 0ull) {
          float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
          for (int e = 1; e < 16; ++e) mx = fmaxf(fmaxf(mx, s[0][e]), s[1][e]);
          const float m_new = fmaxf(m, pair_max(mx)), alpha = fast_exp2(fmaf(m - m_new, a.scale_log2, excess(m_new) - excess(m)));
          m = m_new;
          r = scaled(m, a.scale_log2);
          limit = far(r) ? -INFINITY : kSlack;
          l *= alpha;
#pragma unroll
          for (int db = 0; db < kDB; ++db) o[db] *= alpha;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[kb][e] = far(r) ? (s[kb][e] - m) * a.scale_log2 : fmaf(s[kb][e], a.scale_log2, -r);
        }
        float sum[2] = {0.f, 0.f};
        u32x4 pw[4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float p0 = fast_exp2(x[kb][e]), p1 = fast_exp2(x[kb][e + 1]);
            sum[0] += p0;
            sum[1] += p1;
            pw[2 * kb + (e >> 3)][(e & 7) >> 1] = pack_bf16x2(p0, p1);
          }
        l += sum[0] + sum[1];
        asm volatile("" : "+v"(pw[0]), "+v"(pw[1]), "+v"(pw[2]), "+v"(pw[3]), "+v"(l));     // (done here, not where they are used)
#pragma unroll
        for (int st = 0; st < 4; ++st) pb[st] = __builtin_bit_cast(bf16x8, pw[st]);
      };
      const int k0 = k_at<kD>(lane), v0 = vt_at<kD>(lane);
      // the scores of tile t, the first half of whose K is there; `then` between the two
      const auto scores = [&](int t, auto then) __attribute__((always_inline)) {
        bf16x8 k2[2][kHalf];
        read_k(tile(t, 0, k0), kHalf, k2);
        s[0] = s[1] = (f32x16){0.f};
        __builtin_amdgcn_sched_barrier(0);
        multiply(0, kf);
        __builtin_amdgcn_sched_barrier(0);
        then();
        multiply(kHalf, k2);
      };
      read_k(tile(0, 0, k0), 0, kf);
      begin_a(0);
      scores(0, [] {});
      barrier();
      int t = 0;
      for (; t < (kOneLoop ? n : n_full); ++t) {
        if (kOneLoop && t >= n_full) {
          if (__builtin_amdgcn_ballot_w64(flags[lane & 7] != 0) != 0ull) break;
          const int seen = min(pos, t1 - 1) - (pc.t0 + t * kTokens) - 4 * h;
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = 32 * kb + 8 * (e >> 2) + (e & 3) <= seen ? s[kb][e] : -INFINITY;
        }
        read_k(tile(t + 1, 0, k0), 0, kf);                 // (behind the last tile: of one that nothing is done with)
        begin_b(t);
        softmax();
        end_b(t);
        begin_a(t + 1);
        const int vt = tile(t, kStages, v0);
        bf16x8 v[2][4];
        scores(t + 1, [&]() __attribute__((always_inline)) { read_v(vt, 0, v[0]); });
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int db = 0; db < kDB; ++db) {
          if (db + 1 < kDB) read_v(vt, db + 1, v[(db + 1) & 1]);
#pragma unroll
          for (int st = 0; st < 4; ++st) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[db & 1][st], pb[st], o[db], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        barrier();
      }
      for (; t < n; ++t) {                                 // tiles that some rows do not see whole: the output in the vector half step
        begin_b(t);
        const int seen = min(pos, t1 - 1) - (pc.t0 + t * kTokens) - 4 * h;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[kb][e] = 32 * kb + 8 * (e >> 2) + (e & 3) <= seen ? s[kb][e] : -INFINITY;
        softmax();
        const int vt = tile(t, kStages, v0);
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          bf16x8 ones;
#pragma unroll
          for (int e = 0; e < 8; ++e) ones[e] = (__bf16)(16 * st + 8 * (e >> 2) + (e & 3) <= seen ? 1.f : 0.f);
          bf16x8 v[kDB];
#pragma unroll
          for (int db = 0; db < kDB; ++db) v[db] = read_vt<kD>(lds + (vt ^ db << 6), st);
          add_masked(v, pb[st], ones, o);
          __builtin_amdgcn_sched_barrier(0);
        }
        read_k(tile(t + 1, 0, k0), 0, kf);
        end_b(t);
        begin_a(t + 1);
        scores(t + 1, [] {});
        barrier();
      }
    }
    if (w < 4) barrier();
    if constexpr (!k8) wait_loads<0>();                    // (no load may land once the workgroup's LDS is another's)
  }
  // ---- the block's rows, or its partial of this piece
  const float near = fast_exp2(-excess(m));                // (1 where nothing was seen)
  l = pair_sum(l) * near;
  const int in_block = 32 * w + (lane & 31);
  if (in_block >= min(block_rows, R - rho0)) return;
  if (pc.direct) {
    const bool none = pc.it.past + i_row < 0;
    const int64_t to = (int64_t)(pc.it.row0 + i_row) * a.Hq + head;
    const float inv = none ? 0.f : near / (k8 ? l * kLowered : l);
#pragma unroll
    for (int db = 0; db < kDB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : o[db][4 * j + e] * inv;
        *reinterpret_cast<u32x2 *>((bf16_t *)a.out + to * kD + 32 * db + 8 * j + 4 * h) = (u32x2){pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
      }
    if (a.lse && h == 0) a.lse[to] = none ? -INFINITY : log_sum(m, a.scale_log2, l);
    return;
  }
  if (idx >= a.slots) return;                              // (offsets that overlap)
  const int64_t part = (((int64_t)idx * a.Hkv + c) << a.block_shift) + in_block;
#pragma unroll
  for (int db = 0; db < kDB; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4 *>(a.part_o + part * kD + 32 * db + 8 * j + 4 * h) = (f32x4){o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]} * near;
  if (h == 0) {
    a.part_ml[2 * part] = m;
    a.part_ml[2 * part + 1] = l;
  }
}

}  // namespace sparrow
