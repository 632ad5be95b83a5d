// Decode attention over a paged latent cache with many query rows per key/value head: a prefix that a batch shares, large groups of
// query heads.  The arithmetic is paged.hip's; up to 16 rows per head and 64 in all share a key.
//
// Four wavefronts, one per SIMD and one per head, whose 128 x r weights stay in the accumulation registers.
//   keys    K^T = B_k^T H_k^T of 16 tokens at a time, from latents in LDS; rotated in float32 and multiplied by the
//           rotated queries on the matrix cores, both between the matrix instructions of the next 16 tokens' keys.
//   softmax in the wavefront: a lane holds one row's scores of 8 of the tile's tokens, four lanes the row.
//   values  every wavefront contracts the probabilities of all heads' rows (through LDS) with its share of the value columns.
// One barrier per tile: in interval n are the keys of tile n, the softmax of n - 1 and the values of n - 2.

#include "paged_dev.h"

namespace palu {

template <typename T, int KS, int PT, int VB>
__global__ __launch_bounds__(kPagedRowsThreads) void paged_rows_kernel(PagedArgs a) {
  constexpr bool PAIR = __is_same(T, F16);     // queries and keys as pairs hi + lo
  constexpr int NB_V = 2 * VB;                 // blocks of 32 value columns per wavefront
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  const PagedWork w(a);
  if (w.idle()) return;
  const int i0 = w.i0, i1 = w.i1, nr = w.nr, n_packed = w.n_packed;
  const int NB = a.n_stages;
  const PagedLds ld = paged_lds(w.un.n_groups(), KS, w.v_cols, n_packed, PT, 0, false, PAIR, NB);
  const uint32_t lds0 = lds_addr(lds);
  const bool works = wave < w.nh;                            // else: the same instructions, results nowhere
  const int hh = works ? wave : 0;
  const int hg = w.un.n_groups() > 1 ? hh / w.per_group : 0; // the head's group inside the unit
  const int E = 2 * NB - 1;                                  // entries are requested so many tiles ahead: early enough to be there when rows are made of them
  int* const entries = reinterpret_cast<int*>(lds + ld.entries);
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  auto make_row = [&](int i, int x) __attribute__((always_inline)) {
    rows[(i % kPagedRowSlots) * kPagedTile + x] = w.row_of(i, x, entries[(i % kPagedEntrySlots) * kPagedTile + x]);
  };

  // ---- requests of interval n: keys of tile n + NB - 1, values of n + NB - 3, entries of n + E; the rows of tile
  // n + NB.  An operation moves 64 16-byte pieces, lane i the i-th of them; a wavefront takes every fourth.
  const int ops_k = ld.k_pieces / 8, ops_v = ld.v_pieces / 8;   // per wavefront, each 256 / pieces tokens on
  const int id0 = wave * 64 + lane, x_k = id0 / ld.k_pieces, x_v = id0 / ld.v_pieces;
  const int p_k = (id0 % ld.k_pieces) ^ paged_key_swizzle(x_k);
  const unsigned char* const src_k0 = paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k);
  const unsigned char* const src_k1 = paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k ^ 2);    // (32 pieces: eight tokens on)
  const unsigned char* const src_v = paged_source(a.hv, a.meta.v_off[w.g], w.v_cols, (id0 % ld.v_pieces) ^ paged_value_swizzle(x_v));
  const uint32_t k_pitch = (uint32_t)a.R_k * 2, v_pitch = (uint32_t)a.R_v * 2;
  auto request_keys = [&](int j, int stage) __attribute__((always_inline)) {
    const int* r = rows + (j % kPagedRowSlots) * kPagedTile + x_k;
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (ops_k == 4) {
      const uint32_t r0 = r[0], r1 = r[8], r2 = r[16], r3 = r[24];
      load_to_lds(src_k0 + (uint64_t)r0 * k_pitch, dst);
      load_to_lds(src_k1 + (uint64_t)r1 * k_pitch, dst + 4096);
      load_to_lds(src_k0 + (uint64_t)r2 * k_pitch, dst + 8192);
      load_to_lds(src_k1 + (uint64_t)r3 * k_pitch, dst + 12288);
    } else if (ops_k == 2) {
      const uint32_t r0 = r[0], r1 = r[16];
      load_to_lds(src_k0 + (uint64_t)r0 * k_pitch, dst);
      load_to_lds(src_k0 + (uint64_t)r1 * k_pitch, dst + 4096);
    } else {
      load_to_lds(src_k0 + (uint64_t)(uint32_t)r[0] * k_pitch, dst);
    }
  };
  auto request_values = [&](int j, int stage) __attribute__((always_inline)) {
    const int* r = rows + (j % kPagedRowSlots) * kPagedTile + x_v;
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (VB == 2) {                                           // rows of 64 pieces
      uint32_t y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = r[4 * k];
#pragma unroll
      for (int k = 0; k < 8; ++k) load_to_lds(src_v + (uint64_t)y[k] * v_pitch, dst + 4096 * k);
    } else if (ops_v == 4) {
      const uint32_t r0 = r[0], r1 = r[8], r2 = r[16], r3 = r[24];
      load_to_lds(src_v + (uint64_t)r0 * v_pitch, dst);
      load_to_lds(src_v + (uint64_t)r1 * v_pitch, dst + 4096);
      load_to_lds(src_v + (uint64_t)r2 * v_pitch, dst + 8192);
      load_to_lds(src_v + (uint64_t)r3 * v_pitch, dst + 12288);
    } else {
      const uint32_t r0 = r[0], r1 = r[16];
      load_to_lds(src_v + (uint64_t)r0 * v_pitch, dst);
      load_to_lds(src_v + (uint64_t)r1 * v_pitch, dst + 4096);
    }
  };
  auto request_entries = [&](int n) __attribute__((always_inline)) {
    const int je = n + E;
    if (wave == 3 && je < i1 && lane < kPagedTile)
      load_to_lds4(w.entry_of(je, lane), lds0 + ld.entries + (je % kPagedEntrySlots) * (kPagedTile * 4));
    if (wave == 2 && n >= i0 && n + NB < i1 && lane < kPagedTile) make_row(n + NB, lane);
  };
  const int per_interval = ops_k + ops_v;
  // Stages in use, as LDS offsets: keys of tile n and values of tile n - 2 (the stage before is requested into), angles of n and n - 1.
  const PagedRing ring_k{ld.k, ld.stage_k, NB}, ring_v{ld.v, ld.stage_v, NB}, ring_b{ld.base, (kPagedTile / 16) * kDHead * 4, kPagedBaseSlots};
  int k_at = ring_k.stage(i0), v_at = ring_v.stage(i0 + 2 * NB - 2), b_at = ring_b.stage(i0), b_old = ring_b.before(b_at);

  // ---- prologue
  for (int x = tid; x < kPagedTile * E; x += kPagedRowsThreads) {   // entries of the first tiles, and rows of those that are requested at once
    const int i = i0 + x / kPagedTile;
    if (i < i1) {
      entries[(i % kPagedEntrySlots) * kPagedTile + x % kPagedTile] = *w.entry_of(i, x % kPagedTile);
      if (i < i0 + NB) make_row(i, x % kPagedTile);
    }
  }
  lds_barrier();
  for (int j = i0; j < min(i0 + NB - 1, i1); ++j) request_keys(j, ring_k.stage(j));
  for (int j = i0; j < min(i0 + NB - 3, i1); ++j) request_values(j, ring_v.stage(j));

  PagedAngles angles{w, lds, lds0, ld.base, ld.anchors, lane, 0.f, 0.f, 0.f, 0.f};
  if (wave == 1) angles.begin(NB);

  const int tok = paged_token(col);
  // angles of position tok, of this lane's 16 rotation pairs 16 kg ..; scaled
  float ang_c[16], ang_s[16];
#pragma unroll
  for (int p = 0; p < 16; ++p) {
    ang_c[p] = kKeyScale * a.rope[rope_f32_index(tok, 16 * kg + p, 0, kRopeTableStride)];
    ang_s[p] = kKeyScale * a.rope[rope_f32_index(tok, 16 * kg + p, 1, kRopeTableStride)];
  }
  w.rotate_queries<T, false>(lds + ld.q, ld.q_pitch, kPagedRowsThreads);

  // weights: feature 4 m + j (j < 4) or 64 + 4 m + j - 4 is row m of tile j, so that a lane holds both features of a rotation
  // pair.  A lane reads its four features of either half from eight rows of B_k and transposes them.  They stay in the
  // accumulation registers, which the matrix instructions read as they are.
  uint4v W[KS][8];
  {
    const int width = w.per_group * kDHead;
    const uint16_t* B = a.Bk + w.weights_of(hh, hg) + 4 * col;
    constexpr int AHEAD = KS < 3 ? KS : 3;                   // steps whose rows are in flight
    uint2v v[AHEAD][2][8];
    auto fetch = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint16_t* row = B + (size_t)min(32 * ks + 8 * kg + e, w.rk - 1) * width;
        v[ks % AHEAD][0][e] = *reinterpret_cast<const uint2v*>(row);
        v[ks % AHEAD][1][e] = *reinterpret_cast<const uint2v*>(row + kHalf);
      }
    };
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) fetch(ks);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const uint32_t keep = 32 * ks < w.rk ? 0xffffffffu : 0u;           // rows behind the rank: zero
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          W[ks][j][i] = keep & __builtin_amdgcn_perm(v[ks % AHEAD][j >> 2][2 * i + 1][(j >> 1) & 1], v[ks % AHEAD][j >> 2][2 * i][(j >> 1) & 1],
                                                     (j & 1) ? 0x07060302u : 0x05040100u);
        asm volatile("" : "+a"(W[ks][j]));
      }
      if (ks + AHEAD < KS) fetch(ks + AHEAD);
    }
  }

  const int n_blocks = w.v_cols / 32;                          // of 32 value columns: block wave + 4 v is this wavefront's
  const int n_pt = (n_packed + 15) / 16;
  float4v O[NB_V][PT][2];
#pragma unroll
  for (int v = 0; v < NB_V; ++v)
#pragma unroll
    for (int p = 0; p < PT; ++p) O[v][p][0] = O[v][p][1] = float4v{0, 0, 0, 0};

  // softmax state of row col (the sum: over this lane's tokens); rows of the cache it may see
  float run_max = -INFINITY, run_sum = 0.f;
  const bool live = works && col < nr;
  const int limit = live ? w.limit_of(col) : w.L;
  int all_see = limit;                                       // rows that every row of the wavefront sees
#pragma unroll
  for (int d = 1; d < 16; d *= 2) all_see = min(all_see, __shfl_xor(all_see, d));
  all_see = __builtin_amdgcn_readfirstlane(all_see);
  const int prow = live ? hh * nr + col : PT * 16;           // where its probabilities go; of no row: behind the last

  wait_vm(0);
  lds_barrier();
  const int steady = (NB - 2) * per_interval;

  const unsigned char* const q_row = lds + ld.q + (hh * nr + min(col, nr - 1)) * ld.q_pitch + 32 * kg;
  const int h_key = paged_key_swizzle(tok);
  const int h_lane = tok * ld.k_pieces * 16 + hg * KS * 64, off0 = h_lane + (kg ^ h_key) * 16, off1 = h_lane + ((4 + kg) ^ h_key) * 16;
  const int v_lane = kg * ld.v_pieces * 16, v_pitch16 = 4 * ld.v_pieces * 16;

  float minus_one = -1.f;                                    // (not a constant to the compiler, which would make a conversion and a subtraction of `less`)
  asm("" : "+s"(minus_one));
  float4v acc[2][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[0][j] = acc[1][j] = float4v{0, 0, 0, 0};
  float4v score[2];

  // Keys of sub-tile `sub` of the tile staged at k_stage into acc[sub]; between their matrix instructions the previous sub-tile's, whose
  // tile has its angles at b_stage, are rotated, split and multiplied by the queries into score[1 - sub].  The vector work is 64 steps of
  // about three instructions (a matrix instruction takes the issue slots of four), a step or more behind every matrix instruction.
  auto keys = [&](auto sub_c, int k_stage, int b_stage) __attribute__((always_inline)) {
    constexpr int sub = decltype(sub_c)::value, old = 1 - sub;
    constexpr int kSlots = KS * 8;
    const unsigned char* h0p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off0;
    const unsigned char* h1p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off1;
    const float* bas = reinterpret_cast<const float*>(lds + b_stage) + old * kDHead + 16 * kg;
    uint4v af[3];
    af[0] = *reinterpret_cast<const uint4v*>(h0p);
    af[1] = *reinterpret_cast<const uint4v*>(h1p);
    float4v bc[2], bs[2];                                    // angles of four pairs, and of the next four
    bc[0] = *reinterpret_cast<const float4v*>(bas);
    bs[0] = *reinterpret_cast<const float4v*>(bas + kHalf);
    uint32_t khi[4][4], klo[4][4];                           // [2 side + half][pairs]: contraction steps, feature 64 side + 16 kg + 8 half + ..
    float4v dot[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    float t1, t2, c, s, lo[2], hi[2], l0, l1, l2;
    uint32_t x, y;
    auto step = [&](int e) __attribute__((always_inline)) {
      const int pa = 2 * (e >> 3), pb = pa + 1, q4 = pa >> 2, at = (e >> 3) & 3, half = e >> 5;   // pairs pa and pb
      const float4v c0 = bc[q4 & 1], s0 = bs[q4 & 1];
      if ((e & 15) == 0 && q4 + 1 < 4) {
        bc[(q4 + 1) & 1] = *reinterpret_cast<const float4v*>(bas + 4 * (q4 + 1));
        bs[(q4 + 1) & 1] = *reinterpret_cast<const float4v*>(bas + 4 * (q4 + 1) + kHalf);
      }
      const float kl0 = acc[old][pa & 3][pa >> 2], kh0 = acc[old][4 + (pa & 3)][pa >> 2], kl1 = acc[old][pb & 3][pb >> 2], kh1 = acc[old][4 + (pb & 3)][pb >> 2];
      switch (e & 7) {
        case 0:
          t1 = ang_s[pa] * s0[pa & 3];
          t2 = ang_c[pa] * s0[pa & 3];
          c = __builtin_fmaf(ang_c[pa], c0[pa & 3], -t1);
          break;
        case 1:
          s = __builtin_fmaf(ang_s[pa], c0[pa & 3], t2);
          t1 = kh0 * s;
          t2 = kl0 * s;
          break;
        case 2:
          lo[0] = __builtin_fmaf(kl0, c, -t1);
          hi[0] = __builtin_fmaf(kh0, c, t2);
          t1 = ang_s[pb] * s0[pb & 3];
          break;
        case 3:
          t2 = ang_c[pb] * s0[pb & 3];
          c = __builtin_fmaf(ang_c[pb], c0[pb & 3], -t1);
          s = __builtin_fmaf(ang_s[pb], c0[pb & 3], t2);
          break;
        case 4:
          t1 = kh1 * s;
          t2 = kl1 * s;
          lo[1] = __builtin_fmaf(kl1, c, -t1);
          break;
        case 5:
          hi[1] = __builtin_fmaf(kh1, c, t2);
          // (the empty statements: a product and its rounding stay two instructions.  As one, they would round the exact product to hi
          // where lo is measured from the float32 one, and take one instruction per number instead of one per two.)
          asm("" : "+v"(lo[0]), "+v"(lo[1]), "+v"(hi[0]), "+v"(hi[1]));
          x = pack2<F16>(lo[0], lo[1]);
          y = pack2<F16>(hi[0], hi[1]);
          if (PAIR) asm("" : "+v"(x), "+v"(y));
          khi[half][at] = x;
          khi[2 + half][at] = y;
          break;
        case 6:
          if (PAIR) {
            l0 = less<F16>(lo[0], x, minus_one);
            l1 = less<F16>(lo[1], x >> 16, minus_one);
            l2 = less<F16>(hi[0], y, minus_one);
          }
          break;
        case 7:
          if (PAIR) {
            klo[half][at] = pack2<F16>(l0, l1);
            klo[2 + half][at] = pack2<F16>(l2, less<F16>(hi[1], y >> 16, minus_one));
          }
          break;
      }
    };
    auto products = [&](int half) __attribute__((always_inline)) {
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const int k = 2 * side + half;
        const uint4v kh = {khi[k][0], khi[k][1], khi[k][2], khi[k][3]};
        const uint4v qh = *reinterpret_cast<const uint4v*>(q_row + side * 128 + half * 16);
        dot[side] = mma<F16>(kh, qh, dot[side]);
        if (PAIR) {
          const uint4v kl = {klo[k][0], klo[k][1], klo[k][2], klo[k][3]};
          const uint4v ql = *reinterpret_cast<const uint4v*>(q_row + 256 + side * 128 + half * 16);
          dot[side] = mma<F16>(kh, ql, dot[side]);
          dot[side] = mma<F16>(kl, qh, dot[side]);
        }
      }
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) af[(ks + 2) % 3] = *reinterpret_cast<const uint4v*>(((ks & 1) ? h1p : h0p) + ((ks + 2) >> 1) * 128);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int slot = ks * 8 + j;
        acc[sub][j] = mma<T>(W[ks][j], af[ks % 3], ks == 0 ? float4v{0, 0, 0, 0} : acc[sub][j]);
#pragma unroll
        for (int e = slot * 64 / kSlots; e < (slot + 1) * 64 / kSlots; ++e) {
          step(e);
          if (e == 31) products(0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    products(1);
    score[old] = dot[0] + dot[1];
  };

  // ---- softmax of tile n: this lane has tokens kg + 4 i and 16 + kg + 4 i of row col
  auto softmax = [&](int n) __attribute__((always_inline)) {
    const int buf = n & 1, t0 = w.tile_pos(n);
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = score[e >> 2][e & 3];
    const bool whole = t0 + kPagedTile <= all_see && (t0 + kPagedTile <= w.span.sink || t0 >= w.span.lo);
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = t0 + 4 * e + kg;
        if (t >= limit || (t >= w.span.sink && t < w.span.lo)) s[e] = -INFINITY;
      }
    }
    float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    top = max_of_4(top);
    const float now = fmaxf(run_max, top);
    const float zero = now == -INFINITY ? 0.f : now;         // no row seen yet: exp2(-inf) = 0 below
    const float alpha = __builtin_amdgcn_exp2f(run_max - zero);
    float sum = 0.f;
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float p0 = __builtin_amdgcn_exp2f(s[e] - zero), p1 = __builtin_amdgcn_exp2f(s[e + 1] - zero);
      sum += p0 + p1;
      split2<T>(p0, p1, &ph[e / 2], &pl[e / 2]);
    }
    run_max = now;
    run_sum = run_sum * alpha + sum;
    // in the order of the value product's contraction: lane group kg, token kg + 4 i
    unsigned char* P = lds + ld.p + (buf * (PT * 16 + 1) + prow) * kPagedProbPitch + 16 * kg;
    *reinterpret_cast<uint4v*>(P) = uint4v{ph[0], ph[1], ph[2], ph[3]};
    *reinterpret_cast<uint4v*>(P + 64) = uint4v{pl[0], pl[1], pl[2], pl[3]};
    reinterpret_cast<float*>(lds + ld.alpha)[buf * (PT * 16 + 4) + prow] = alpha;
  };

  // ---- values of tile n, staged at v_stage
  auto values = [&](int n, int v_stage) __attribute__((always_inline)) {
    const int buf = n & 1;
#pragma unroll
    for (int v = 0; v < NB_V; ++v) {
      if (v > 0 && 4 * v >= n_blocks) break;                 // (a block behind the last, of a wavefront whose neighbours have one: nothing that is stored)
      const int block = wave + 4 * v;
      uint32_t x[8];                                         // tokens kg + 4 e
      const unsigned char* row = lds + v_stage + v_lane + ((block * 4 + (col >> 2)) ^ (4 * kg)) * 16 + (col & 3) * 4;
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
        const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (buf * (PT * 16 + 4) + 16 * p + 4 * kg) * 4);
        const unsigned char* P = lds + ld.p + (buf * (PT * 16 + 1) + 16 * p + col) * kPagedProbPitch + 16 * kg;
        const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 64);
        O[v][p][0] = mma<T>(hi, f0, O[v][p][0] * al);
        O[v][p][1] = mma<T>(hi, f1, O[v][p][1] * al);
        O[v][p][0] = mma<T>(lo, f0, O[v][p][0]);
        O[v][p][1] = mma<T>(lo, f1, O[v][p][1]);
      }
    }
  };

  for (int n = i0; n < i1 + 2; ++n) {
    if (n + NB - 1 < i1) request_keys(n + NB - 1, ring_k.before(k_at));
    if (n + NB - 3 >= i0 && n + NB - 3 < i1) request_values(n + NB - 3, ring_v.before(v_at));
    request_entries(n);
    if (wave == 1) {
      angles.request(n + NB);
      if (n + 1 < i1) angles.make(n + 1);
    }
    if (n <= i1) keys(IntC<0>(), k_at, b_old);               // (behind the last tile, and of the one before the first: nothing that is used)
    if (n >= i0 + 2) values(n - 2, v_at);
    if (n > i0 && n <= i1) softmax(n - 1);
    if (n < i1) keys(IntC<1>(), k_at, b_at);
    k_at = ring_k.behind(k_at);
    v_at = ring_v.behind(v_at);
    b_old = b_at;
    b_at = ring_b.behind(b_at);
    // what interval n + 1 reads was requested in n - NB + 2; the NB - 2 intervals since then may be outstanding where all of them
    // requested whole tiles
    if (n + NB - 1 < i1) wait_vm(steady);
    else wait_vm(0);
    lds_barrier();
  }

  // ---- partial results
  run_sum += __shfl_xor(run_sum, 16);
  run_sum += __shfl_xor(run_sum, 32);
  if (live && kg == 0) w.store_ml(hh, col, run_max, run_sum);
#pragma unroll
  for (int v = 0; v < NB_V; ++v) {
    const int block = wave + 4 * v;
    if (block >= n_blocks) continue;
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (16 * p + 4 * kg + e < n_packed) w.store_o(16 * p + 4 * kg + e, block * 32 + 2 * col, O[v][p][0][e], O[v][p][1][e]);
  }
}

namespace {
template <typename T, int KS>
PagedFn pick(int vb) { return vb == 1 ? paged_rows_kernel<T, KS, 4, 1> : paged_rows_kernel<T, KS, 2, 2>; }
}  // namespace

template <typename T> PagedFn paged_rows_form(const PagedForm& f) {
  return f.ks == 2 ? pick<T, 2>(f.vb) : f.ks == 4 ? pick<T, 4>(f.vb) : f.ks == 6 ? pick<T, 6>(f.vb) : pick<T, 8>(f.vb);
}
template PagedFn paged_rows_form<PALU_PAGED_ACT>(const PagedForm&);

}  // namespace palu
