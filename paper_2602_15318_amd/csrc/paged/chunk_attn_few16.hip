// Attention of few new tokens over the paged cache by 16-row tiles: up to 16 rows (new token, query head of the group) per request and KV head, in
// fp32 up to 32.  Bound by memory: 28/4 heads of 128, 48 single tokens over up to 8,192 (405 MB) 69 us, 5.9 TB/s; one over 26,112 (53.5 MB) 11, 4.9
// TB/s with launch, plan and first tile in it; the second pass takes 4.5 to 5 more.  16-row tiles against 32-row ones for up to 16 rows: 79 / 83 and
// 17.3 / 18.1 us a call; for 28 rows over 26,112 tokens 27 / 18, so that more rows take 32-row tiles (chunk_attn_few32.hip).
//
// A workgroup takes one block and piece of keys; its wavefronts take the 16-token tiles in turn and know nothing of each other until the
// end, where their states of a row are merged through LDS.  A tile lies on one page; it travels memory -> LDS past the registers, two
// tiles of K and V ahead.
//   S^T = K Q^T    v_mfma_f32_16x16x32_bf16 / 16x16x4_f32 (A: lane = key + 16 * c4).  A 16-byte read of K gives a lane its part of one k-step (bf16) or
//                 of four (fp32, columns 16 g + 4 c4 + 0..3); Q^T in registers, cut alike.  D: a lane holds, for row lane % 16, the scores
//                 of keys 4 c4 + 0..3.
//   O^T += V^T P^T  the scores' own registers are P^T: of one 16x16x16 product whose V^T comes by a transposing read (bf16), or of four 16x16x4
//                 ones, step i taking keys 4 c4 + i (fp32).
#include <type_traits>

#include "chunk_attn_16.hpp"

namespace sparrow {

namespace {

constexpr int kTokens = 16;

template <typename T, int kD, int kRT, int kWaves>
__global__ void __launch_bounds__(64 * kWaves) chunk_few16_kernel(ChunkArgs a) {
  constexpr bool kF32 = std::is_same<T, float>::value;
  constexpr int kBM = 16 * kRT, kDB = kD / 16, kRow = kD * (int)sizeof(T), kChunks = kRow / 16, kG = kRow / 64, kLoadRows = 64 / kChunks;
  constexpr int kTileBytes = kTokens * kRow, kLoads = kTokens / kLoadRows;
  constexpr int kTiles = kWaves * 4 * kTileBytes, kMerge = kWaves * kBM * kD * 4, kOut = kD / 4;      // kOut: 16-byte chunks of a row of fp32 outputs
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kTiles > kMerge ? kTiles : kMerge];   // [wave][K0, V0, K1, V1]
  __shared__ float ml[kWaves][kBM][2];

  const int lane = threadIdx.x & 63, n16 = lane & 15, c4 = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = blockIdx.x, idx = blockIdx.y + 32768 * blockIdx.z;
  Piece pc;
  if (!find_piece(a, idx, lane, &pc)) return;         // uniform
  const int R = pc.rq.n * a.g, rho0 = pc.block * kBM;
  const auto table = (const int32_t __attribute__((address_space(4))) *)(uintptr_t)(a.block_table + (int64_t)pc.b * a.table_stride);
  const unsigned char *Kg = (const unsigned char *)((const T *)a.k + c * a.stride_head);
  const unsigned char *Vg = (const unsigned char *)((const T *)a.v + c * a.stride_head);
  const unsigned int row_bytes = (unsigned int)(sizeof(T) * a.stride_token);
  // what the block's rows see of the piece
  const int last_pos = min(pc.rq.past + quotient(min(rho0 + kBM, R) - 1, a.g), pc.rq.L - 1);
  const int first_pos = pc.rq.past + quotient(rho0, a.g);
  const int t1 = min(pc.t1, last_pos + 1);
  const int n_tiles = max(t1 - pc.t0 + kTokens - 1, 0) / kTokens;
  const int n = (n_tiles - w + kWaves - 1) / kWaves;       // of this wavefront: w, w + kWaves, ...

  unsigned char *mine = lds + w * 4 * kTileBytes;
  const unsigned int mine_at = lds_offset(mine);
  // Row r's 16-byte chunk x is kept at x ^ swz(r): eight rows read at one chunk, or four groups of four rows read transposed, fall on
  // different banks.  (V of fp32 is read 4 bytes a lane, whole rows: kept as it is.)
  const auto swz = [](int row) { return kRow == 128 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; };
  // load j of a tile: rows kLoadRows j + lane / kChunks
  auto issue = [&](const unsigned char *src, bool swizzled, int tile, int part) __attribute__((always_inline)) {
    const int t = pc.t0 + tile * kTokens;
    const unsigned int page = min((unsigned int)table[t >> a.page_shift], (unsigned int)(a.n_pages - 1));
    const unsigned char *at = src + (int64_t)page * a.stride_page * (int64_t)sizeof(T) + (int64_t)(t & ((1 << a.page_shift) - 1)) * row_bytes;
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
    m[rt] = kNothingSeen;
    l[rt] = 0.f;
#pragma unroll
    for (int db = 0; db < kDB; ++db) o[rt][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }
  if (n > 0) {
    issue(Kg, true, w, 0);
    issue(Vg, !kF32, w, 1);
    if (n > 1) {
      issue(Kg, true, w + kWaves, 2);
      issue(Vg, !kF32, w + kWaves, 3);
    }
    u32x4 q[kRT][kG];
#pragma unroll
    for (int rt = 0; rt < kRT; ++rt) {
      const T *at = (const T *)a.q + (int64_t)(pc.rq.row0 + i_row[rt]) * a.q_row + (int64_t)(c * a.g + rho[rt] - i_row[rt] * a.g) * kD;
#pragma unroll
      for (int g = 0; g < kG; ++g) q[rt][g] = ((const u32x4 *)at)[4 * g + c4];
    }
    wait_loads<0>();
    auto step = [&](int it, auto masked) __attribute__((always_inline)) {
      constexpr bool kMasked = decltype(masked)::value;
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
        const u32x4 k = *reinterpret_cast<const u32x4 *>(K + n16 * kRow + (((4 * g + c4) ^ swz(n16)) << 4));
        if constexpr (kF32) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt)
              s[rt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i]), __uint_as_float(q[rt][g][i]), s[rt], 0, 0, 0);
        } else {
#pragma unroll
          for (int rt = 0; rt < kRT; ++rt)
            s[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[rt][g]), s[rt], 0, 0, 0);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(Kg, true, w + (it + 2) * kWaves, 2 * buf);
      const int t = pc.t0 + (w + it * kWaves) * kTokens;
      float p[kRT][4], seen[kRT][4];
#pragma unroll
      for (int rt = 0; rt < kRT; ++rt) {
        if constexpr (kMasked) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool vis = t + 4 * c4 + i <= min(pos[rt], t1 - 1);
            s[rt][i] = vis ? s[rt][i] : -INFINITY;
            seen[rt][i] = vis ? 1.f : 0.f;
          }
        }
        // the row's reference score moves only when a score of the wavefront's lies more than kSlack above it
        const float mx = fmaxf(fmaxf(s[rt][0], s[rt][1]), fmaxf(s[rt][2], s[rt][3]));
        if (__builtin_amdgcn_ballot_w64((mx - m[rt]) * a.scale_log2 > kSlack) != 0ull) {
          const float m_new = fmaxf(m[rt], quad_max(mx)), alpha = factor(m[rt], m_new, a.scale_log2);
          m[rt] = m_new;
          l[rt] *= alpha;
#pragma unroll
          for (int db = 0; db < kDB; ++db) o[rt][db] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[rt][i] = fast_exp2((s[rt][i] - m[rt]) * a.scale_log2);
        l[rt] += (p[rt][0] + p[rt][1]) + (p[rt][2] + p[rt][3]);
      }
      if (more2) wait_loads<3 * kLoads>();
      else if (more) wait_loads<2 * kLoads>();
      else wait_loads<0>();
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v[kDB];
#pragma unroll
          for (int db = 0; db < kDB; ++db) v[db] = *reinterpret_cast<const float *>(V + (4 * c4 + i) * kRow + (16 * db + n16) * 4);
#pragma unroll
          for (int rt = 0; rt < kRT; ++rt) {
            if constexpr (kMasked) {
              add_masked4(v, p[rt][i], seen[rt][i], o[rt]);
            } else {
#pragma unroll
              for (int db = 0; db < kDB; ++db) o[rt][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[db], p[rt][i], o[rt][db], 0, 0, 0);
            }
          }
        }
      } else {
        // Probabilities are rounded to bf16 for the product (their sum is not): 2^-9 of a term on average, of the result less.  A second bf16 term of
        // each, with the test for values that are no numbers that it needs in every tile: 48 single tokens 73.0 -> 74.5 us, 200 90 -> 95, forty over
        // 500 13.1 -> 15.9, twelve chains in 32-row tiles 33.5 -> 55.7.
        const int row = 4 * c4 + (n16 >> 2);
        bf16x4 v[kDB];
#pragma unroll
        for (int db = 0; db < kDB; ++db) v[db] = lds_tr(V + row * kRow + (((2 * db + ((n16 >> 1) & 1)) ^ swz(row)) << 4) + 8 * (n16 & 1));
#pragma unroll
        for (int rt = 0; rt < kRT; ++rt) {
          bf16x4 pb, ones;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pb[i] = (__bf16)p[rt][i];
            if (kMasked) ones[i] = (__bf16)seen[rt][i];
          }
          if constexpr (kMasked) {
            add_masked16(v, pb, ones, o[rt]);
          } else {
#pragma unroll
            for (int db = 0; db < kDB; ++db) o[rt][db] = mul16(v[db], pb, o[rt][db]);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more2) issue(Vg, !kF32, w + (it + 2) * kWaves, 2 * buf + 1);
    };
    // the tiles that all rows of the block see whole, then the others
    const int full = max(min(first_pos + 1, t1) - pc.t0, 0) / kTokens, n_full = max(full - w + kWaves - 1, 0) / kWaves;
    int it = 0;
    for (; it < n_full; ++it) step(it, std::false_type());
    for (; it < n; ++it) step(it, std::true_type());
  }
  // ---- merge: states of the wavefronts through LDS
  __syncthreads();
  unsigned char *states = lds + w * kBM * kD * 4;
#pragma unroll
  for (int rt = 0; rt < kRT; ++rt) {
    const int r = 16 * rt + n16;
    l[rt] = quad_sum(l[rt]);
    if (c4 == 0) { ml[w][r][0] = m[rt]; ml[w][r][1] = l[rt]; }
#pragma unroll
    for (int db = 0; db < kDB; ++db)                       // elements 16 db + 4 c4 + 0..3
      *reinterpret_cast<f32x4 *>(states + (r * kOut + ((4 * db + c4) ^ n16)) * 16) = o[rt][db];
  }
  __syncthreads();
  const bool direct = pc.n_splits == 1;
  if (!direct && idx >= a.slots) return;                   // (offsets that overlap)
  const int64_t part = ((int64_t)idx * a.Hkv + c) * kBM;
  const int rows = min(kBM, R - rho0);
  for (int x = threadIdx.x; x < rows * kOut; x += 64 * kWaves) {
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
      sum += *reinterpret_cast<const f32x4 *>(lds + k * kBM * kD * 4 + (r * kOut + (chunk ^ (r & 15))) * 16) * f;
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
    if constexpr (kF32)
      *reinterpret_cast<f32x4 *>((float *)a.out + at * kD + 4 * chunk) = sum;
    else
      *reinterpret_cast<u32x2 *>((bf16_t *)a.out + at * kD + 4 * chunk) = (u32x2){pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
    if (a.lse && chunk == 0) a.lse[at] = none ? -INFINITY : log_sum(top, a.scale_log2, ls);
  }
}

template <typename T, int kRT, int kWaves> hipError_t launch(int d, dim3 grid, const ChunkArgs &a, hipStream_t st) {
  if (d == 128) hipLaunchKernelGGL((chunk_few16_kernel<T, 128, kRT, kWaves>), grid, dim3(64 * kWaves), 0, st, a);
  else hipLaunchKernelGGL((chunk_few16_kernel<T, 64, kRT, kWaves>), grid, dim3(64 * kWaves), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_few16(int dtype, int d, int rows, int waves, int blocks, const ChunkArgs &a, hipStream_t st) {
  const dim3 grid(a.Hkv, blocks < 32768 ? blocks : 32768, (blocks + 32767) / 32768);
  if (dtype == SPARROW_F32)
    return rows == 16 ? launch<float, 1, 4>(d, grid, a, st) : launch<float, 2, 4>(d, grid, a, st);
  return waves == 8 ? launch<bf16_t, 1, 8>(d, grid, a, st) : waves == 2 ? launch<bf16_t, 1, 2>(d, grid, a, st) : launch<bf16_t, 1, 4>(d, grid, a, st);
}

}  // namespace sparrow
