// Decode attention over a paged latent cache: a sliding window with a few first rows (sinks), and a prefix that the
// sequences of a batch share.
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v
//
// One workgroup takes a unit (up to four key/value heads, two where the key rank is above 256), up to 16 query rows of each
// (query heads, and sequences where the tokens are shared) and a run of tiles of 32 tokens.
// Eight wavefronts, two per SIMD; FQ of them share a head: each has 64 / FQ of its rotation pairs, the weights for which stay
// in up to 128 accumulation registers.
//   keys    K^T = B_k^T H_k^T of 16 tokens at a time, from latents in LDS; rotated in float32 and multiplied by the
//           rotated queries on the matrix cores.  The scores over a wavefront's features go to LDS.
//   softmax eight lanes per row, eight rows per wavefront: adds the partial scores, masks, keeps the running maximum and sum in
//           float32.
//   values  every wavefront contracts the probabilities of all rows with its 32 columns of the value latents (read as two
//           columns of eight tokens per lane: the transposition that the matrix operand wants is a byte permute).
//   angles  of a tile's tokens, a 512th part by every lane, in LDS: all heads' keys are rotated by them.
// One barrier per tile: in interval n are the keys of tile n, the softmax of n - 1 and the values of n - 2 (WHOLE), or two of them, one per
// 16 tokens' keys, where LDS does not hold two tiles' scores, angles and probabilities.  With two, 16 sequences of 8192 rows take 390 us,
// with one 374.  One wavefront of a SIMD begins with the keys, the other ends with them: the matrix instructions of one run beside
// the vector instructions of the other.  Latents, page-table entries and the angles' anchors come by loads that write to LDS
// directly, n_stages - 1 tiles ahead, counted and never drained while tiles follow: 5.3 TB/s at 2 us latency take 40 KB in flight
// per compute unit.
// What bounds it: rank 256 of 4 heads takes 2048 cycles of matrix instructions per SIMD and tile for the keys, about 400 for the scores, and
// 500 vector instructions of 4 cycles; two wavefronts per SIMD leave half of either unused.  Measured, 32 heads in groups of 4, rank 256, float16:
// 16 sequences of 8192 rows 374 us (2.9 TB/s; the loads alone 199 us); 8 sequences behind 16384 shared rows 81 us.
// Partial results (unnormalised sums, maxima, row sums) are merged, normalised and multiplied by B_v in paged_merge_kernel.
//
// Rotation.  The angle of position t0 + i is that of t0 plus that of i: a lane keeps cos and sin of two i < 16 and one pair, and those of
// each 16 tokens' first position follow from those before.  These products are right to 8e-7 (PagedAngles), which moves a logit by as
// much of sum(|q k|) / sqrt(d_h).  Rotated keys are made once for all query rows; turning the queries of few rows to the tiles instead
// was no faster.
// Rounding.  The matrix instructions take 16-bit operands.  The rotated keys and queries enter as pairs of float16 numbers hi + lo
// (2^-21 relative; the second has steps of 2^-24, so keys below 1 to 2^-22 and queries below 1/8 to 2^-25), the probabilities as pairs of
// the latents' type (2^-21 or 2^-40 of the largest, bfloat16 2^-16), so that the error is that of the output's rounding (2^-11, bfloat16
// 2^-8).  (One float16 number each for a bfloat16 layer's keys and queries left outputs 1.3e-3 from these in the 2-norm, beside 1.66e-3
// of rounding them.)  Keys are scaled by 1/8 and the queries by 8 (exact): magnitudes up to 524032 stay in range.

#include "paged_dev.h"

namespace palu {

template <typename T, int FQ, int KS, int PT, int VB>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_kernel(PagedArgs a) {
  constexpr int NH = 8 / FQ;
  constexpr int FT = 8 / FQ;                   // tiles of 16 features per wavefront: low halves of the rotation pairs, then high halves
  constexpr bool WHOLE = paged_whole(FQ, PT);  // one barrier per tile
  constexpr int NP = 16 / FQ, NT = NP / 4;     // rotation pairs per lane, contraction steps of the score product
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  const PagedWork w(a);
  if (w.idle()) return;
  const int i0 = w.i0, i1 = w.i1, nr = w.nr, n_packed = w.n_packed;
  const int NB = a.n_stages;
  const int max_packed = PT > 1 ? PT * 16 : a.max_packed;    // rows that LDS is laid out for
  const PagedLds ld = paged_lds(w.un.n_groups(), KS, w.v_cols, max_packed, PT, FQ, NB);
  const int plane = (max_packed + 1) * kPagedScorePitch;     // floats: a wavefront's part of 16 tokens' scores, of all rows and none
  const uint32_t lds0 = lds_addr(lds);
  const bool works = wave % NH < w.nh;                       // else: the same instructions, results nowhere
  const int hh = works ? wave % NH : 0, fq = wave / NH;
  const int fbase = (64 / FQ) * fq;                          // first rotation pair of this wavefront
  const bool front = wave >= 4;                              // of the two of a SIMD: the one that ends with the keys (not that with rows
                                                             // of the softmax, where there are few)
  const int hg = w.un.n_groups() > 1 ? hh / w.per_group : 0; // the head's group inside the unit
  const int E = 2 * NB - 1;                                  // entries are requested so many tiles ahead: early enough to be there when rows are made of them
  // the lane, once more: where accumulators take the registers, what is made of it is made anew, not kept in registers of the loop, which spill
  auto fresh_lane = [&]() __attribute__((always_inline)) {
    int l = lane;
    if (PT > 1) asm volatile("" : "+v"(l));
    return l;
  };
  int* const entries = reinterpret_cast<int*>(lds + ld.entries);
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  auto make_row = [&](int i, int x) __attribute__((always_inline)) {
    rows[(i & (ld.slots - 1)) * kPagedTile + x] = w.row_of(i, x, entries[(i & (2 * ld.slots - 1)) * kPagedTile + x]);
  };

  // ---- requests of interval n: keys of tile n + NB - 1, values of n + NB - 1 - LAG, entries of n + E; the rows of tile n + NB.  An
  // operation moves 64 16-byte pieces, lane i the i-th of them; a wavefront takes every eighth.
  const int id0 = wave * 64 + lane, x_k = id0 / ld.k_pieces, x_v = id0 / ld.v_pieces;
  const int p_k = (id0 % ld.k_pieces) ^ paged_key_swizzle(x_k);
  const unsigned char* const src_k = paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k);
  const unsigned char* const src_k1 = FQ == 4 ? paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k ^ 2) : src_k;   // (64 pieces: eight tokens on)
  const unsigned char* const src_v = paged_source(a.hv, a.meta.v_off[w.g], w.v_cols, (id0 % ld.v_pieces) ^ paged_value_swizzle(x_v));
  const uint32_t k_pitch = (uint32_t)a.R_k * 2, v_pitch = (uint32_t)a.R_v * 2;
  auto request_keys = [&](int j, int stage) __attribute__((always_inline)) {
    const int* r = rows + (j & (ld.slots - 1)) * kPagedTile + x_k;
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (FQ == 4) {                                           // rows of 64 pieces
      const uint32_t r0 = r[0], r1 = r[8], r2 = r[16], r3 = r[24];
      load_to_lds(src_k + (uint64_t)r0 * k_pitch, dst);
      load_to_lds(src_k1 + (uint64_t)r1 * k_pitch, dst + 8192);
      load_to_lds(src_k + (uint64_t)r2 * k_pitch, dst + 16384);
      load_to_lds(src_k1 + (uint64_t)r3 * k_pitch, dst + 24576);
    } else if (ld.k_pieces == 32) {
      const uint32_t r0 = r[0], r1 = r[16];
      load_to_lds(src_k + (uint64_t)r0 * k_pitch, dst);
      load_to_lds(src_k + (uint64_t)r1 * k_pitch, dst + 8192);
    } else if (ld.k_pieces == 16 || wave < 4) {
      load_to_lds(src_k + (uint64_t)(uint32_t)r[0] * k_pitch, dst);
    }
  };
  auto request_values = [&](int j, int stage) __attribute__((always_inline)) {
    const int* r = rows + (j & (ld.slots - 1)) * kPagedTile + x_v;
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (VB == 2) {                                           // rows of 64 pieces
      const uint32_t r0 = r[0], r1 = r[8], r2 = r[16], r3 = r[24];
      load_to_lds(src_v + (uint64_t)r0 * v_pitch, dst);
      load_to_lds(src_v + (uint64_t)r1 * v_pitch, dst + 8192);
      load_to_lds(src_v + (uint64_t)r2 * v_pitch, dst + 16384);
      load_to_lds(src_v + (uint64_t)r3 * v_pitch, dst + 24576);
    } else if (ld.v_pieces == 32) {
      const uint32_t r0 = r[0], r1 = r[16];
      load_to_lds(src_v + (uint64_t)r0 * v_pitch, dst);
      load_to_lds(src_v + (uint64_t)r1 * v_pitch, dst + 8192);
    } else {
      load_to_lds(src_v + (uint64_t)(uint32_t)r[0] * v_pitch, dst);
    }
  };
  const int per_k = (ld.k_pieces / 2 + 7 - wave) / 8, per_v = ld.v_pieces / 16;    // operations of this wavefront
  // Stages in use, as LDS offsets: keys of tile n and values of tile n - LAG (the stage before is requested into).
  const PagedRing ring_k{ld.k, ld.stage_k, NB}, ring_v{ld.v, ld.stage_v, NB};
  int k_at = ring_k.stage(i0), v_at = ring_v.stage(i0 + 2 * NB - (WHOLE ? 2 : 1));

  // ---- prologue
  for (int x = tid; x < kPagedTile * E; x += kPagedThreads) {   // entries of the first tiles, and rows of those that are requested at once
    const int i = i0 + x / kPagedTile;
    if (i < i1) {
      entries[(i & (2 * ld.slots - 1)) * kPagedTile + x % kPagedTile] = *w.entry_of(i, x % kPagedTile);
      if (i < i0 + NB) make_row(i, x % kPagedTile);
    }
  }
  lds_barrier();
  PagedAngles angles{w, lds, lds0, ld.anchors, ld.slots, lane, 0.f, 0.f, 0.f, 0.f};
  if (wave == 1) angles.begin(NB);
  for (int j = i0; j < min(i0 + NB - 1, i1); ++j) request_keys(j, ring_k.stage(j));
  for (int j = i0; j < min(i0 + NB - (WHOLE ? 3 : 2), i1); ++j) request_values(j, ring_v.stage(j));

  // weights.  FQ = 2: rotation pair fbase + 2 m + j is row m of tile j (low half) and 2 + j (high half); FQ = 4: pair fbase + m of tiles
  // 0 and 1.  A lane reads its features from eight rows of B_k and transposes them.  They stay in the accumulation registers, which the
  // matrix instructions read as they are.
  uint4v W[KS][FT];
  {
    const int width = w.per_group * kDHead;
    const uint16_t* B = a.Bk + w.weights_of(hh, hg) + fbase;
    constexpr int AHEAD = KS < 4 ? KS : (PT > 1 ? 3 : 4);    // steps whose rows are in flight (of many query rows fewer: registers)
    uint32_t v[AHEAD][2][8];
    auto fetch = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint16_t* row = B + (size_t)min(32 * ks + 8 * kg + e, w.rk - 1) * width;
#pragma unroll
        for (int side = 0; side < 2; ++side)
          v[ks % AHEAD][side][e] = FQ == 2 ? *reinterpret_cast<const uint32_t*>(row + side * kHalf + 2 * col) : (uint32_t)row[side * kHalf + col];
      }
    };
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) fetch(ks);
    w.rotate_queries<T, PT == 4 ? 2 : 1>(lds + ld.q, ld.q_pitch);
    // angles of positions 0 .. 15, scaled, where those of a tile's other tokens come later
    float* const in = reinterpret_cast<float*>(lds + ld.ang) + (WHOLE ? 3 : 1) * 16 * kPagedAngPitch;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = tid + i * kPagedThreads;
      in[(x & 15) * kPagedAngPitch + (x >> 4)] = kKeyScale * a.rope[rope_f32_index(x & 15, (x >> 4) & 63, x >> 10, kRopeTableStride)];
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint32_t keep = 32 * ks < w.rk ? 0xffffffffu : 0u;           // rows behind the rank: zero
#pragma unroll
      for (int side = 0; side < 2; ++side) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = v[ks % AHEAD][side][2 * i], y = v[ks % AHEAD][side][2 * i + 1];
          W[ks][side * (FT / 2)][i] = keep & __builtin_amdgcn_perm(y, x, 0x05040100u);
          if (FQ == 2) W[ks][side * (FT / 2) + FT / 2 - 1][i] = keep & __builtin_amdgcn_perm(y, x, 0x07060302u);
        }
      }
#pragma unroll
      for (int j = 0; j < FT; ++j) asm volatile("" : "+a"(W[ks][j]));
      if (ks + AHEAD < KS) fetch(ks + AHEAD);
    }
  }

  const int n_blocks = w.v_cols / 32;                        // of 32 value columns: block wave + 8 v is this wavefront's
  const int n_pt = (n_packed + 15) / 16;
  float4v O[VB][PT][2];
#pragma unroll
  for (int v = 0; v < VB; ++v)
#pragma unroll
    for (int p = 0; p < PT; ++p) O[v][p][0] = O[v][p][1] = float4v{0, 0, 0, 0};

  // softmax: this lane has four tokens of packed row srow; its state (the sum: over these tokens)
  const int srow = 8 * wave + (lane >> 3);
  float run_max = -INFINITY, run_sum = 0.f;
  const int limit = srow < n_packed ? w.limit_of(srow % nr) : w.L;       // rows of the cache that it may see
  int all_see = limit;                                       // rows that every row of the wavefront sees
#pragma unroll
  for (int d = 8; d < 64; d *= 2) all_see = min(all_see, __shfl_xor(all_see, d));
  all_see = __builtin_amdgcn_readfirstlane(all_see);

  wait_vm(0);
  lds_barrier();
  const int steady = (NB - 2) * (per_k + per_v);

  // queries of row col: of a contraction step, low halves of four pairs, high halves
  uint4v qh[NT], ql[NT];
  {
    const unsigned char* q = lds + ld.q + (hh * nr + min(col, nr - 1)) * ld.q_pitch + 2 * (fbase + NP * kg);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint2v x = *reinterpret_cast<const uint2v*>(q + 8 * t), y = *reinterpret_cast<const uint2v*>(q + 128 + 8 * t);
      qh[t] = uint4v{x.x, x.y, y.x, y.y};
      const uint2v z = *reinterpret_cast<const uint2v*>(q + 256 + 8 * t), u = *reinterpret_cast<const uint2v*>(q + 384 + 8 * t);
      ql[t] = uint4v{z.x, z.y, u.x, u.y};
    }
  }
  // angles: this lane makes those of rotation pair `lane` of tokens wave and wave + 8 of 16
  const float* const in = reinterpret_cast<const float*>(lds + ld.ang) + ((WHOLE ? 48 : 16) + wave) * kPagedAngPitch + lane;
  const float in_c0 = in[0], in_s0 = in[kHalf], in_c1 = in[8 * kPagedAngPitch], in_s1 = in[8 * kPagedAngPitch + kHalf];
  auto ang_slot = [&](int n, int sub) __attribute__((always_inline)) { return (WHOLE ? 2 * ((n - i0) & 1) + sub : sub) * 16; };
  auto make_angles = [&](int n, int sub) __attribute__((always_inline)) {
    const int lane = fresh_lane();
    float* at = reinterpret_cast<float*>(lds + ld.ang) + (ang_slot(n, sub) + wave) * kPagedAngPitch + lane;
    const float c = angles.c, s = angles.s;
    at[0] = __builtin_fmaf(in_c0, c, -(in_s0 * s));
    at[kHalf] = __builtin_fmaf(in_s0, c, in_c0 * s);
    at[8 * kPagedAngPitch] = __builtin_fmaf(in_c1, c, -(in_s1 * s));
    at[8 * kPagedAngPitch + kHalf] = __builtin_fmaf(in_s1, c, in_c1 * s);
    angles.turn();
  };
  angles.start();
  make_angles(i0, 0);
  if (WHOLE) make_angles(i0, 1);
  lds_barrier();                                             // (scores and probabilities take the queries' place, other angles that of the first 16)

  const int my_row = works && col < nr ? hh * nr + col : max_packed;   // where this lane's scores go; of no row: behind the last
  const int tok = paged_token(col);
  const int h_key = paged_key_swizzle(tok);
  const int h_lane = tok * ld.k_pieces * 16 + hg * KS * 64, off0 = h_lane + (kg ^ h_key) * 16, off1 = h_lane + ((4 + kg) ^ h_key) * 16;
  const float* const my_ang = reinterpret_cast<const float*>(lds + ld.ang) + tok * kPagedAngPitch + fbase + NP * kg;
  float* const my_score = reinterpret_cast<float*>(lds + ld.s) + fq * plane + my_row * kPagedScorePitch + 4 * kg;
  // scores of 16 tokens: of two tiles, in turn; with two barriers per tile, of its last 16 tokens those of one
  auto score_slot = [&](int n, int sub) __attribute__((always_inline)) { return (WHOLE ? 2 * (n & 1) + sub : (sub == 0 ? n & 1 : 2)) * FQ * plane; };
  float minus_one = -1.f;                                    // (not a constant to the compiler, which would make a conversion and a subtraction of `less`)
  asm("" : "+s"(minus_one));

  // Keys of sub-tile `sub` of tile n, staged at k_stage; rotated, split and multiplied by the queries.
  auto keys = [&](auto sub_c, int n, int k_stage) __attribute__((always_inline)) {
    constexpr int sub = decltype(sub_c)::value;
    const unsigned char* h0p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off0;
    const unsigned char* h1p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off1;
    const float* ang = my_ang + ang_slot(n, sub) * kPagedAngPitch;
    float4v acc[FT], c4[NT], s4[NT];
    uint4v af[3];
    af[0] = *reinterpret_cast<const uint4v*>(h0p);
    af[1] = *reinterpret_cast<const uint4v*>(h1p);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) {
        af[(ks + 2) % 3] = *reinterpret_cast<const uint4v*>(((ks & 1) ? h1p : h0p) + ((ks + 2) >> 1) * 128);
      } else if (ks + 2 == KS) {
        c4[0] = *reinterpret_cast<const float4v*>(ang);
        s4[0] = *reinterpret_cast<const float4v*>(ang + kHalf);
      }
#pragma unroll
      for (int j = 0; j < FT; ++j) acc[j] = mma<T>(W[ks][j], af[ks % 3], ks == 0 ? float4v{0, 0, 0, 0} : acc[j]);
    }
    float4v dot = {0, 0, 0, 0};
    if (NT > 1) {
      c4[NT - 1] = *reinterpret_cast<const float4v*>(ang + 4);
      s4[NT - 1] = *reinterpret_cast<const float4v*>(ang + 4 + kHalf);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {                           // contraction steps: low halves of four pairs, high halves
      uint4v hi, lo;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float x[2], y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int p = 4 * t + 2 * u + i;
          const float l = FQ == 2 ? acc[p & 1][p >> 1] : acc[0][p], h = FQ == 2 ? acc[FT / 2 + (p & 1)][p >> 1] : acc[1][p];
          const float c = c4[t][2 * u + i], sn = s4[t][2 * u + i];
          x[i] = __builtin_fmaf(l, c, -(h * sn));
          y[i] = __builtin_fmaf(h, c, l * sn);
        }
        // (the empty statements: a product and its rounding stay two instructions.  As one, they would round the exact product to hi
        // where lo is measured from the float32 one, and take one instruction per number instead of one per two.)
        asm("" : "+v"(x[0]), "+v"(x[1]), "+v"(y[0]), "+v"(y[1]));
        uint32_t xh = pack2<F16>(x[0], x[1]), yh = pack2<F16>(y[0], y[1]);
        asm("" : "+v"(xh), "+v"(yh));
        lo[u] = pack2<F16>(less<F16>(x[0], xh, minus_one), less<F16>(x[1], xh >> 16, minus_one));
        lo[2 + u] = pack2<F16>(less<F16>(y[0], yh, minus_one), less<F16>(y[1], yh >> 16, minus_one));
        hi[u] = xh;
        hi[2 + u] = yh;
      }
      dot = mma<F16>(hi, qh[t], dot);
      dot = mma<F16>(hi, ql[t], dot);
      dot = mma<F16>(lo, qh[t], dot);
    }
    *reinterpret_cast<float4v*>(my_score + score_slot(n, sub)) = dot;   // lane: query row col, tokens kg + 4 i
  };

  // ---- softmax of tile n: this lane has tokens 16 stile + squad + 4 i
  auto softmax = [&](int n) __attribute__((always_inline)) {
    if (8 * wave >= n_packed) return;
    const int at = fresh_lane();
    const int srow = 8 * wave + (at >> 3), stile = at >> 2 & 1, squad = at & 3;
    const int t0 = w.tile_pos(n);
    const float* row = reinterpret_cast<const float*>(lds + ld.s) + score_slot(n, 0) + (stile ? score_slot(n, 1) - score_slot(n, 0) : 0) +
                       min(srow, n_packed) * kPagedScorePitch + 4 * squad;
    float4v s = *reinterpret_cast<const float4v*>(row);
#pragma unroll
    for (int f = 1; f < FQ; ++f) s += *reinterpret_cast<const float4v*>(row + f * plane);
    const bool whole = t0 + kPagedTile <= all_see && (t0 + kPagedTile <= w.span.sink || t0 >= w.span.lo);
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + 16 * stile + squad + 4 * e;
        if (t >= limit || (t >= w.span.sink && t < w.span.lo)) s[e] = -INFINITY;
      }
    }
    const float now = fmaxf(run_max, max_of_8(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
    const float zero = now == -INFINITY ? 0.f : now;         // no row seen yet: exp2(-inf) = 0 below
    const float alpha = __builtin_amdgcn_exp2f(run_max - zero);
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = kProbScale<T> * __builtin_amdgcn_exp2f(s[e] - zero);
    uint2v hi, lo;
    uint32_t h0, l0, h1, l1;
    split2<T>(p[0], p[1], &h0, &l0);
    split2<T>(p[2], p[3], &h1, &l1);
    hi = uint2v{h0, h1};
    lo = uint2v{l0, l1};
    run_max = now;
    run_sum = run_sum * alpha + ((p[0] + p[1]) + (p[2] + p[3]));
    // in the order of the value product's contraction: lane group squad, tokens squad + 4 e
    unsigned char* P = lds + ld.p + ((WHOLE ? (n & 1) * (PT * 16 + 1) : 0) + min(srow, PT * 16)) * kPagedProbPitch + 16 * squad + 8 * stile;
    *reinterpret_cast<uint2v*>(P) = hi;
    *reinterpret_cast<uint2v*>(P + 64) = lo;
    reinterpret_cast<float*>(lds + ld.alpha)[(WHOLE ? (n & 1) * (PT * 16) : 0) + srow] = alpha;
  };

  // ---- values of tile n, staged at v_stage
  auto values = [&](int n, int v_stage) __attribute__((always_inline)) {
    const int l = fresh_lane(), col = l & 15, kg = l >> 4, v_lane = kg * ld.v_pieces * 16 + (col & 3) * 4, v_pitch16 = 4 * ld.v_pieces * 16;
#pragma unroll
    for (int v = 0; v < VB; ++v) {
      const int block = wave + 8 * v;
      if (block >= n_blocks) break;
      uint32_t x[8];                                         // tokens kg + 4 e
      const unsigned char* row = lds + v_stage + v_lane + ((block * 4 + (col >> 2)) ^ (4 * kg)) * 16;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const uint32_t*>(row + e * v_pitch16);
      uint4v f0, f1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f0[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);
        f1[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);
      }
#pragma unroll
      for (int p = 0; p < PT; ++p) {
        if (p > 0 && p >= n_pt) break;
        const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + ((WHOLE ? (n & 1) * (PT * 16) : 0) + 16 * p + 4 * kg) * 4);
        const unsigned char* P = lds + ld.p + ((WHOLE ? (n & 1) * (PT * 16 + 1) : 0) + 16 * p + col) * kPagedProbPitch + 16 * kg;
        const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 64);
        O[v][p][0] = mma<T>(hi, f0, O[v][p][0] * al);
        O[v][p][1] = mma<T>(hi, f1, O[v][p][1] * al);
        O[v][p][0] = mma<T>(lo, f0, O[v][p][0]);
        O[v][p][1] = mma<T>(lo, f1, O[v][p][1]);
      }
    }
  };

  constexpr int LAG = WHOLE ? 2 : 1;                         // values follow the keys so many intervals later
  for (int n = i0; n < i1 + LAG; ++n) {
    auto first_half = [&]() __attribute__((always_inline)) {
      if (n + NB - 1 < i1) request_keys(n + NB - 1, ring_k.before(k_at));
      if (n > i0 && n <= i1) softmax(n - 1);
    };
    auto second_half = [&]() __attribute__((always_inline)) {
      const int j = n + NB - 1 - LAG;
      if (j >= i0 && j < i1) request_values(j, ring_v.before(v_at));
      if (n >= i0 + LAG) values(n - LAG, v_at);
    };
    if (wave == 3 && n + E < i1 && lane < kPagedTile)
      load_to_lds4(w.entry_of(n + E, lane), lds0 + ld.entries + ((n + E) & (2 * ld.slots - 1)) * (kPagedTile * 4));
    if (wave == 2 && n + NB < i1 && lane < kPagedTile) make_row(n + NB, lane);
    if (wave == 1) angles.request(n + NB);
    if (WHOLE) {
      if (n + 1 < i1) {
        angles.reach(n + 1);
        make_angles(n + 1, 0);
        make_angles(n + 1, 1);
      }
      if (front) {
        first_half();
        second_half();
      }
      if (n < i1) {
        keys(IntC<0>(), n, k_at);
        keys(IntC<1>(), n, k_at);
      }
      if (!front) {
        first_half();
        second_half();
      }
    } else {
      if (n < i1) make_angles(n, 1);
      if (front) first_half();
      if (n < i1) keys(IntC<0>(), n, k_at);
      if (!front) first_half();
      lds_barrier();
      if (n + 1 < i1) {
        angles.reach(n + 1);
        make_angles(n + 1, 0);
      }
      if (front) second_half();
      if (n < i1) keys(IntC<1>(), n, k_at);
      if (!front) second_half();
    }
    k_at = ring_k.behind(k_at);
    v_at = ring_v.behind(v_at);
    // what interval n + 1 reads was requested in n - NB + 2; the NB - 2 intervals since then may be outstanding where all of them
    // requested whole tiles
    if (n + NB - 1 < i1) wait_vm(steady);
    else wait_vm(0);
    lds_barrier();
  }

  // ---- partial results
#pragma unroll
  for (int d = 1; d < 8; d *= 2) run_sum += __shfl_xor(run_sum, d);
  if (srow < n_packed && (lane & 7) == 0) w.store_ml(srow / nr, srow % nr, run_max, run_sum);
#pragma unroll
  for (int v = 0; v < VB; ++v) {
    const int block = wave + 8 * v;
    if (block >= n_blocks) continue;
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * p + 4 * kg + e < n_packed) w.store_o(16 * p + 4 * kg + e, block * 32 + 2 * col, O[v][p][0][e], O[v][p][1][e]);
  }
}

namespace {
template <typename T, int FQ, int KS>
PagedFn pick(const PagedForm& f) {
  if (f.many) return f.vb == 1 ? paged_kernel<T, FQ, KS, 4, 1> : paged_kernel<T, FQ, KS, 2, 2>;
  return f.vb == 1 ? paged_kernel<T, FQ, KS, 1, 1> : paged_kernel<T, FQ, KS, 1, 2>;
}
}  // namespace

template <typename T> PagedFn paged_form(const PagedForm& f) {
  switch (f.ks) {
    case 2: return pick<T, 2, 2>(f);
    case 4: return pick<T, 2, 4>(f);
    case 6: return pick<T, 2, 6>(f);
    case 8: return pick<T, 2, 8>(f);
    case 12: return f.vb == 1 ? paged_kernel<T, 4, 12, 1, 1> : paged_kernel<T, 4, 12, 1, 2>;
    default: return f.vb == 1 ? paged_kernel<T, 4, 16, 1, 1> : paged_kernel<T, 4, 16, 1, 2>;
  }
}
template PagedFn paged_form<PALU_PAGED_ACT>(const PagedForm&);

}  // namespace palu
