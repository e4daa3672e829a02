// Attention of chunks of new tokens over the paged cache, bf16: blocks of 256 rows (new token, query head of the group) per request and KV
// head.  Bound by the matrix cores and, beside them, by the exponentials: of a tile of 64 keys a wavefront's 32 MFMAs (heads of 128)
// take 1,024 cycles of its SIMD's matrix core, its softmax as many of the vector ALU.
//
// A workgroup of eight wavefronts takes one block and piece of keys; wavefront w has rows 32 w .. 32 w + 31.  Wavefronts w and w + 4 share
// a SIMD and run half a step apart: while one is in the products of a step (scores of a tile, output of the tile before), the other is in
// its softmax.  K and V tiles of 64 keys go memory -> LDS past the registers, four of each, asked for four to six half steps
// ahead.  Half a step apart against one barrier a tile: chunk of 2,048 tokens over 26,112, 28/4 heads of 128, 672 / 738 us.
//
// Probabilities are rounded to bf16 for the output's product, half a step 2^-9 to 2^-8 of a term; the row's sum takes them unrounded.
//
// Measured: that chunk 625 to 690 us by card (1,070 to 1,180 TFLOP/s; matrix cores busy 56 % of the cycles), prompt of 7,001 tokens 325 to 365
// (960 to 1,080; 53 %), prompt of 6,000 with 32/8 heads of 64 190 to 204.
#include "chunk_attn_mfma.hpp"

namespace sparrow {

namespace {

constexpr int kWaves = 8, kTokens = 64, kBM = 256, kStages = 4;

template <int kD>
__global__ void __launch_bounds__(64 * kWaves, 2) chunk_many_kernel(ChunkArgs a) {
  constexpr int kDB = kD / 32, kKS = kD / 16, kHalf = kKS / 2;
  // The requests in the half step that has time left, the vector one with heads of 128 (prompt of 7,001 tokens 364 -> 357 us), the matrix one
  // with heads of 64 (of 6,000 206 -> 198).
  constexpr bool kLate = kD == 128;
  constexpr int kTileBytes = kTokens * 2 * kD, kLoads = 8 / Tile<kD>::kLoadRows;      // of a wavefront: eight rows of a tile
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * kStages * kTileBytes];    // K tiles, V tiles
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  Piece pc;
  if (!find_piece(a, idx, lane, &pc)) return;         // uniform
  const Pages pages = pages_of(a, pc, c);
  const int R = pc.rq.n * a.g, rho0 = pc.block * kBM;
  const bool have = rho0 + 32 * w < R;                     // the wavefront has rows
  // this lane's row, and how far the block's rows see
  const int rho = min(rho0 + 32 * w + (lane & 31), R - 1);
  const int i_row = quotient(rho, a.g, a.inv_g), head = c * a.g + rho - i_row * a.g;
  const int pos = min(pc.rq.past + i_row, pc.rq.L - 1);
  const int last_pos = min(pc.rq.past + quotient(min(rho0 + kBM, R) - 1, a.g), pc.rq.L - 1);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;
  // tiles that all rows of the block see whole
  const int n_full = min(n, max(min(t1, pc.rq.past + quotient(rho0, a.g) + 1) - pc.t0, 0) / kTokens);

  // About scaled points r below 2^20 an exponent is one operation, fma(score, scale, -r): the weights are then 2^c of those about m, c what
  // the rounding of r took off (2^-5 at most), which is taken out where the states leave the workgroup.  Farther points, and a row that has seen
  // nothing, let every score past their limit and into the branch of the points that move, which takes the difference first.  (Everywhere
  // the difference first: chunk of 2,048 over 26,112 tokens 651 -> 677 us, prompt of 6,000 with heads of 64 187 -> 205.)
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
    const unsigned int lds0 = lds_offset(lds) + 1024 * kLoads * w;
    unsigned int from_k[kLoads], from_v[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = Tile<kD>::kLoadRows * j;
      from_k[j] = row * pages.stride_token + Tile<kD>::k_from(lane, 8 * w + row, pages.stride_token);
      from_v[j] = row * pages.stride_token + Tile<kD>::v_from(lane, 8 * w + row, pages.stride_token);
    }
    auto place = [&](int tile) __attribute__((always_inline)) { return pages.offset(pc.t0 + min(tile, n - 1) * kTokens + 8 * w); };
    auto load_k = [&](int64_t at, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) global_to_lds<false>(pages.k + at, from_k[j], lds0 + (t & (kStages - 1)) * kTileBytes + 1024 * j);
    };
    auto load_v = [&](int64_t at, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        global_to_lds<false>(pages.v + at, from_v[j], lds0 + (kStages + (t & (kStages - 1))) * kTileBytes + 1024 * j);
    };
    const int64_t p0 = place(0), p1 = place(1), p2 = place(2);
    load_k(p0, 0);
    load_v(p0, 0);
    load_k(p1, 1);
    load_v(p1, 1);
    load_k(p2, 2);
    bf16x8 q[kKS];
    {
      const unsigned char *at = (const unsigned char *)a.q + 2 * ((int64_t)(pc.rq.row0 + i_row) * a.q_row + (int64_t)head * kD) + 16 * h;
#pragma unroll
      for (int ks = 0; ks < kKS; ++ks) q[ks] = *(const bf16x8 *)(at + 32 * ks);
    }
    // Half steps of tile t: A(t), its scores (and the output of tile t - 1), then B(t), its softmax; a barrier ends each.  A(t), or B(t),
    // asks for K of tile t + 3 and V of t + 2, whose places A(t - 1) was the last to read.  A wavefront ends B(t) when all but its last
    // requests are done, those of this step: K of t + 2 and V of t + 1 are there before either half of the workgroup begins A(t + 1).
    int64_t at_v = p2, at_k = place(3);
    wait_loads<0>();
    barrier();
    if (w >= 4) barrier();                                 // half a step behind
    auto request = [&](int t) __attribute__((always_inline)) {
      load_k(at_k, t + 3);
      load_v(at_v, t + 2);
    };
    auto begin_a = [&](int t) __attribute__((always_inline)) {
      if (!kLate) request(t);
    };
    auto begin_b = [&](int t) __attribute__((always_inline)) {
      if (kLate) request(t);
      at_v = at_k;
      at_k = place(t + 4);
    };
    if (!have) {
      begin_a(0);
      barrier();
      for (int t = 0; t < n; ++t) {
        begin_b(t);
        wait_loads<2 * kLoads>();
        barrier();
        begin_a(t + 1);
        barrier();
      }
    } else {
      f32x16 s[2];
      bf16x8 pb[4], kf[2][kHalf];                          // kf: the first half of the columns of the next tile's K
      auto tile = [&](int t, int stage0, int at) __attribute__((always_inline)) {
        at += (stage0 + (t & (kStages - 1))) * kTileBytes;
        asm volatile("" : "+v"(at));                       // (worked out here: kept, the offsets cost more registers than there are)
        return at;
      };
      auto read_k = [&](int at, int ks0, bf16x8 (*k)[kHalf]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kHalf; ++ks)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) k[kb][ks] = lds_b128(lds + (at ^ (ks0 + ks) << 5) + 32 * kb * Tile<kD>::kRow);
      };
      auto multiply = [&](int ks0, bf16x8 (*k)[kHalf]) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < kHalf; ++ks)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb][ks], q[ks0 + ks], s[kb], 0, 0, 0);
      };
      auto read_v = [&](int at, int db, bf16x8 *v) __attribute__((always_inline)) {
#pragma unroll
        for (int st = 0; st < 4; ++st) v[st] = read_vt<kD>(lds + (at ^ db << 6), st);
      };
      // the scores' exponentials about the row's reference score, which moves only when a score of the wavefront's lies more than
      // kSlack above it
      auto softmax = [&]() __attribute__((always_inline)) {
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
      auto scores = [&](int t) __attribute__((always_inline)) {       // from kf on
        bf16x8 k2[2][kHalf];
        read_k(tile(t, 0, k0), kHalf, k2);
        s[0] = s[1] = (f32x16){0.f};
        __builtin_amdgcn_sched_barrier(0);
        multiply(0, kf);
        __builtin_amdgcn_sched_barrier(0);
        multiply(kHalf, k2);
      };
      // Where the loop below lies in the 64-byte lines of instructions makes 1 %: of 16 places 657 to 665 us (chunk of 2,048 over 26,112), this one 657.
      asm volatile(".p2align 6\n\t.rept 15\n\ts_nop 0\n\t.endr");
      read_k(tile(0, 0, k0), 0, kf);
      begin_a(0);
      scores(0);
      barrier();
      int t = 0;
      for (; t < n_full; ++t) {
        read_k(tile(t + 1, 0, k0), 0, kf);                 // (behind the last tile: of one that nothing is done with)
        begin_b(t);
        softmax();
        wait_loads<2 * kLoads>();
        barrier();
        begin_a(t + 1);
        const int vt = tile(t, kStages, v0);
        bf16x8 k2[2][kHalf], v[2][4];
        read_k(tile(t + 1, 0, k0), kHalf, k2);
        s[0] = s[1] = (f32x16){0.f};
        __builtin_amdgcn_sched_barrier(0);
        multiply(0, kf);
        __builtin_amdgcn_sched_barrier(0);
        read_v(vt, 0, v[0]);
        multiply(kHalf, k2);
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
        wait_loads<2 * kLoads>();
        barrier();
        begin_a(t + 1);
        scores(t + 1);
        barrier();
      }
    }
    if (w < 4) barrier();
    wait_loads<0>();                                       // (no load may land once the workgroup's LDS is another's)
  }
  // ---- the block's rows, or its partial of this piece
  const float near = fast_exp2(-excess(m));                // (1 where nothing was seen)
  l = pair_sum(l) * near;
  if (rho0 + 32 * w + (lane & 31) >= R) return;
  if (pc.n_splits == 1) {
    const bool none = pc.rq.past + i_row < 0;
    const int64_t to = (int64_t)(pc.rq.row0 + i_row) * a.Hq + head;
    const float inv = none ? 0.f : near / l;
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
  const int64_t part = ((int64_t)idx * a.Hkv + c) * kBM + 32 * w + (lane & 31);
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

}  // namespace

hipError_t launch_chunk_many(int d, int blocks, const ChunkArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, blocks < 32768 ? blocks : 32768, (blocks + 32767) / 32768), block(64 * kWaves);
  if (d == 128) hipLaunchKernelGGL(chunk_many_kernel<128>, grid, block, 0, st, a);
  else hipLaunchKernelGGL(chunk_many_kernel<64>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace sparrow
