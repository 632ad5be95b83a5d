// Decode attention over a paged latent cache: a sliding window with a few first rows (sinks), and a prefix that the
// sequences of a batch share.  Up to 16 query rows (heads x rows) per workgroup; paged_rows.hip takes more.
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v
//
// One workgroup takes a unit (up to four key/value heads, two where the key rank is above 256) and a run of tiles of 32 tokens.
// Eight wavefronts, two per SIMD; FQ of them share a head: each has 64 / FQ of its rotation pairs, the weights for which stay
// in 128 accumulation registers.
//   keys    K^T = B_k^T H_k^T of 16 tokens at a time, from latents in LDS; rotated in float32 and multiplied by the
//           rotated queries on the matrix cores, both between the matrix instructions of the next 16 tokens' keys.  The
//           scores over a wavefront's features go to LDS.
//   softmax 16 lanes per row, four rows per wavefront: adds the partial scores, masks, keeps the running maximum and sum in float32.
//   values  every wavefront contracts the probabilities of all rows with its 32 columns of the value latents (read as two
//           columns of eight tokens per lane: the transposition that the matrix operand wants is a byte permute).
// One barrier per tile: in interval n are the keys of tile n, the softmax of n - 2 and the values of n - 3.  Latents,
// page-table entries and angles come by loads that write to LDS directly, n_stages - 1 tiles ahead, counted and
// never drained while tiles follow: 5.3 TB/s at 2 us latency take 40 KB in flight per compute unit.
// Partial results (unnormalised sums, maxima, row sums) are merged, normalised and multiplied by B_v in paged_merge_kernel.
//
// Rotation.  The angle of position t0 + i is that of t0 plus that of i: cos and sin of i < 16 stay in registers, those of
// each 16 tokens' first position are fetched from the table (512 bytes), instead of 512 bytes per token.  Products of
// numbers that are right to 1e-7.
// Rounding.  The matrix instructions take 16-bit operands.  A float16 layer's output is rounded to 2^-11 relative, so
// the rotated keys, the queries and the probabilities enter as pairs of float16 numbers hi + lo (2^-21).  A bfloat16
// layer's output is rounded to 2^-8: keys and queries enter as one float16 number each (2^-11), probabilities as a pair
// of bfloat16 numbers.  Keys are scaled by 1/8 and the queries by 8 (exact): magnitudes up to 524032 stay in range.

#include "paged_dev.h"

namespace palu {

template <typename T, int FQ, int KS, int VB, bool TURN>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_kernel(PagedArgs a) {
  constexpr bool PAIR = __is_same(T, F16);     // queries and keys as pairs hi + lo
  constexpr int NH = 8 / FQ;
  constexpr int FT = 8 / FQ;                   // tiles of 16 features per wavefront: low halves of the rotation pairs, then high halves
  constexpr int NP = 16 / FQ;                  // rotation pairs per lane
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  const PagedWork w(a);
  if (w.idle()) return;
  const int i0 = w.i0, i1 = w.i1, nr = w.nr, n_packed = w.n_packed;
  const int NB = a.n_stages;
  const PagedLds ld = paged_lds(w.un.n_groups(), KS, w.v_cols, n_packed, FQ, TURN, PAIR, NB);
  const uint32_t lds0 = lds_addr(lds);
  const bool works = wave % NH < w.nh;                       // else: the same instructions, results nowhere
  const int hh = works ? wave % NH : 0, fq = wave / NH;
  const int fbase = (64 / FQ) * fq;                          // first rotation pair of this wavefront
  const int hg = w.un.n_groups() > 1 ? hh / w.per_group : 0; // the head's group inside the unit
  const int E = 2 * NB - 1;                                  // entries are requested so many tiles ahead: early enough to be there when rows are made of them
  int* const entries = reinterpret_cast<int*>(lds + ld.entries);
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  // the lane, once more: where registers are short, what is made of it is made anew, not kept in registers of the loop, which spill
  auto fresh_lane = [&]() __attribute__((always_inline)) {
    int l = lane;
    if (KS * FT >= 24 || VB == 2) asm volatile("" : "+v"(l));
    return l;
  };
  auto make_row = [&](int i, int x) __attribute__((always_inline)) {
    rows[(i % kPagedRowSlots) * kPagedTile + x] = w.row_of(i, x, entries[(i % kPagedEntrySlots) * kPagedTile + x]);
  };

  // ---- requests of interval n: keys of tile n + NB - 1, values of n + NB - 4, entries of n + E; the rows of tile
  // n + NB.  An operation moves 64 16-byte pieces, lane i the i-th of them; a wavefront takes every eighth.
  const int id0 = wave * 64 + lane, x_k = id0 / ld.k_pieces, x_v = id0 / ld.v_pieces;
  const int p_k = (id0 % ld.k_pieces) ^ paged_key_swizzle(x_k);
  const unsigned char* const src_k0 = paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k);
  const unsigned char* const src_k1 = FQ == 4 ? paged_source(a.hk, a.meta.k_off[w.g], w.k_cols, p_k ^ 2) : src_k0;   // (64 pieces: eight tokens on)
  const unsigned char* const src_v = paged_source(a.hv, a.meta.v_off[w.g], w.v_cols, (id0 % ld.v_pieces) ^ paged_value_swizzle(x_v));
  const uint32_t k_pitch = (uint32_t)a.R_k * 2, v_pitch = (uint32_t)a.R_v * 2;
  // Half 0 or 1 of a tile's operations, the rows r of its tokens at hand: a wavefront waits while its operations are taken, one per 16 cycles
  // of all the wavefronts', so they come in fours through the interval.
  constexpr int KR = FQ == 4 ? 4 : 2, VR = VB == 2 ? 4 : 2;  // operations of a wavefront, at most
  auto rows_of = [&](int j, int x, auto count, uint32_t* r) __attribute__((always_inline)) {
    const int* from = rows + (j % kPagedRowSlots) * kPagedTile + x;
#pragma unroll
    for (int i = 0; i < decltype(count)::value; ++i) r[i] = from[i * (kPagedTile / decltype(count)::value)];
  };
  auto request_keys = [&](int half, const uint32_t* r, int stage) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (FQ == 4) {                                           // rows of 64 pieces
      load_to_lds(src_k0 + (uint64_t)r[2 * half] * k_pitch, dst + 16384 * half);
      load_to_lds(src_k1 + (uint64_t)r[2 * half + 1] * k_pitch, dst + 16384 * half + 8192);
    } else if (half == 0 ? ld.k_pieces >= 16 || wave < 4 : ld.k_pieces == 32) {
      load_to_lds(src_k0 + (uint64_t)r[half] * k_pitch, dst + 8192 * half);
    }
  };
  auto request_values = [&](int half, const uint32_t* r, int stage) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + stage + wave * 1024;
    if (VB == 2) {                                           // rows of 64 pieces
      load_to_lds(src_v + (uint64_t)r[2 * half] * v_pitch, dst + 16384 * half);
      load_to_lds(src_v + (uint64_t)r[2 * half + 1] * v_pitch, dst + 16384 * half + 8192);
    } else if (half == 0 || ld.v_pieces == 32) {
      load_to_lds(src_v + (uint64_t)r[half] * v_pitch, dst + 8192 * half);
    }
  };
  auto request_entries = [&](int n) __attribute__((always_inline)) {
    const int je = n + E;
    if (wave == 6 && je < i1 && lane < kPagedTile) load_to_lds4(w.entry_of(je, lane), lds0 + ld.entries + (je % kPagedEntrySlots) * (kPagedTile * 4));
    if (wave == 5 && n >= i0 && n + NB < i1 && lane < kPagedTile) make_row(n + NB, lane);
  };
  const int per_interval = (ld.k_pieces / 2 + 7 - wave) / 8 + (ld.v_pieces / 2 + 7 - wave) / 8;
  // Stages in use, as LDS offsets: keys of tile n and values of tile n - 3 (the stage before is requested into), angles of n and n - 1.
  const PagedRing ring_k{ld.k, ld.stage_k, NB}, ring_v{ld.v, ld.stage_v, NB}, ring_b{ld.base, (kPagedTile / 16) * kDHead * 4, kPagedBaseSlots};
  int k_at = ring_k.stage(i0), v_at = ring_v.stage(i0 + 3 * NB - 3), b_at = ring_b.stage(i0), b_old = ring_b.before(b_at);

  // ---- prologue
  for (int x = tid; x < kPagedTile * E; x += kPagedThreads) {   // entries of the first tiles, and rows of those that are requested at once
    const int i = i0 + x / kPagedTile;
    if (i < i1) {
      entries[(i % kPagedEntrySlots) * kPagedTile + x % kPagedTile] = *w.entry_of(i, x % kPagedTile);
      if (i < i0 + NB) make_row(i, x % kPagedTile);
    }
  }
  lds_barrier();
  uint32_t row_k[KR], row_v[VR];
  for (int j = i0; j < min(i0 + NB - 1, i1); ++j) {
    rows_of(j, x_k, IntC<KR>(), row_k);
    request_keys(0, row_k, ring_k.stage(j));
    request_keys(1, row_k, ring_k.stage(j));
  }
  for (int j = i0; j < min(i0 + NB - 4, i1); ++j) {
    rows_of(j, x_v, IntC<VR>(), row_v);
    request_values(0, row_v, ring_v.stage(j));
    request_values(1, row_v, ring_v.stage(j));
  }

  PagedAngles angles{w, lds, lds0, ld.base, ld.anchors, lane, 0.f, 0.f, 0.f, 0.f};
  if (wave == 3) {
    angles.begin(NB + (TURN ? 1 : 0));
    if (TURN && i0 + 1 < i1) angles.make(i0 + 1);
  }

  const int tok = paged_token(col);
  // angles of position tok, of this lane's rotation pairs fbase + NP kg ..; scaled
  float ang_c[NP], ang_s[NP];
  if (TURN) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      ang_c[p] = kKeyScale * a.rope[rope_f32_index(tok, fbase + NP * kg + p, 0, kRopeTableStride)];
      ang_s[p] = kKeyScale * a.rope[rope_f32_index(tok, fbase + NP * kg + p, 1, kRopeTableStride)];
    }
  } else {
    float* ang = reinterpret_cast<float*>(lds + ld.ang);
    for (int x = tid; x < 16 * kDHead; x += kPagedThreads)
      ang[(x & 15) * kPagedAngPitch + (x >> 4)] = kKeyScale * a.rope[rope_f32_index(x & 15, (x >> 4) & 63, x >> 10, kRopeTableStride)];
  }
  w.rotate_queries<T, TURN, 1>(lds + ld.q, ld.q_pitch);

  // weights.  FQ = 2: rotation pair fbase + 2 m + j is row m of tile j (low half) and 2 + j (high half); FQ = 4: pair fbase + m of tiles
  // 0 and 1.  A lane reads its features from eight rows of B_k and transposes them.  They stay in the accumulation registers, which the
  // matrix instructions read as they are.
  uint4v W[KS][FT];
  {
    const int width = w.per_group * kDHead;
    const uint16_t* B = a.Bk + w.weights_of(hh, hg) + fbase;
    constexpr int AHEAD = KS < 4 ? KS : 4;                   // steps whose rows are in flight
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
  float4v O[VB][2];
#pragma unroll
  for (int v = 0; v < VB; ++v) O[v][0] = O[v][1] = float4v{0, 0, 0, 0};

  // softmax state of the lanes of the last four wavefronts: row, two of its tokens; rows of the cache that the row may see
  const int srow = 4 * (wave & 3) + (lane >> 4);
  float run_max = -INFINITY, run_sum = 0.f;
  const int limit = srow < n_packed ? w.limit_of(srow % nr) : w.L;

  // The queries turned back to the first position of every sub-tile of tile j, [turned slot][packed row][hi | lo][feature]: with them, a
  // sub-tile's keys are rotated by the angles of 0 .. 15, which are the same for all.
  auto turned_slot = [&](int j, int sub) __attribute__((always_inline)) { return ld.turned + (sub == 0 ? j & 1 : 2 + (j + 3) % 3) * n_packed * ld.q_pitch; };
  auto turn_queries = [&](int j) __attribute__((always_inline)) {
    const int lane = fresh_lane();
    const float* base = reinterpret_cast<const float*>(lds + ld.base) + j % kPagedBaseSlots * (kPagedTile / 16) * kDHead + lane;
    for (int x = wave; x < 2 * n_packed; x += 8) {           // lane: rotation pair
      const int sub = x >= n_packed, r = x - sub * n_packed;
      const float* q = reinterpret_cast<const float*>(lds + ld.q) + r * kDHead + lane;
      const float c = base[sub * kDHead], s = base[sub * kDHead + kHalf], x0 = q[0], x1 = q[kHalf];
      paged_store_query<T>(lds + turned_slot(j, sub) + r * ld.q_pitch, lane, __builtin_fmaf(x0, c, x1 * s), __builtin_fmaf(x1, c, -(x0 * s)));
    }
  };
  if (TURN) {
    lds_barrier();
    turn_queries(i0);
  }
  wait_vm(0);
  lds_barrier();
  const int steady = (NB - 2) * per_interval;
  // (a wavefront that has softmax rows has more to do than the other of its SIMD: it goes first.  8 sequences, one latent per head: 242 -> 222 us)
  if (wave >= 4 && 4 * (wave & 3) < n_packed) __builtin_amdgcn_s_setprio(2);

  const int my_row = works && col < nr ? hh * nr + col : n_packed;       // where this lane's scores go; of no row: behind the last
  const int q_lane = (hh * nr + min(col, nr - 1)) * ld.q_pitch + 2 * (fbase + NP * kg);
  const int h_key = paged_key_swizzle(tok);
  const int h_lane = tok * ld.k_pieces * 16 + hg * KS * 64, off0 = h_lane + (kg ^ h_key) * 16, off1 = h_lane + ((4 + kg) ^ h_key) * 16;
  float minus_one = -1.f;                                    // (not a constant to the compiler, which would make a conversion and a subtraction of `less`)
  asm("" : "+s"(minus_one));

  float4v acc[2][FT];
#pragma unroll
  for (int j = 0; j < FT; ++j) acc[0][j] = acc[1][j] = float4v{0, 0, 0, 0};

  // Keys of sub-tile `sub` of the tile staged at k_stage into acc[sub]; between their matrix instructions the previous sub-tile's, of tile
  // `np` with its angles at b_stage, are rotated, split and multiplied by the queries.  The vector work is 8 steps of two or three
  // instructions for every two pairs (a matrix instruction takes the issue slots of four).
  auto keys = [&](auto sub_c, int k_stage, int np, int b_stage, auto&& halfway) __attribute__((always_inline)) {
    constexpr int sub = decltype(sub_c)::value, old = 1 - sub;
    constexpr int kSlots = KS * FT, kSteps = NP * 4;
    const unsigned char* h0p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off0;
    const unsigned char* h1p = lds + k_stage + 16 * sub * ld.k_pieces * 16 + off1;
    const float* bas = reinterpret_cast<const float*>(lds + b_stage) + old * kDHead + fbase + NP * kg;
    const float* ang = reinterpret_cast<const float*>(lds + ld.ang) + tok * kPagedAngPitch + fbase + NP * kg;
    const unsigned char* q_row = lds + (TURN ? turned_slot(np, old) : ld.q) + q_lane;
    uint4v af[3];
    af[0] = *reinterpret_cast<const uint4v*>(h0p);
    af[1] = *reinterpret_cast<const uint4v*>(h1p);
    uint32_t khi[4], klo[4];                                 // of a contraction step: low halves of four pairs, high halves
    float4v dot = {0, 0, 0, 0};
    uint2v ql[2], qh[2];
    float4v c4, s4;                                          // cos and sin of a step's pairs
    float t1, t2, lo[2], hi[2], l0, l1, l2, l3;
    uint32_t x, y;
    auto step = [&](int e) __attribute__((always_inline)) {
      const int pa = 2 * (e >> 3), pb = pa + 1, t = pa >> 2, at = (e >> 3) & 1;   // pairs pa and pb
      auto low = [&](int p) { return FQ == 2 ? acc[old][p & 1][p >> 1] : acc[old][0][p]; };
      auto high = [&](int p) { return FQ == 2 ? acc[old][FT / 2 + (p & 1)][p >> 1] : acc[old][1][p]; };
      auto cosine = [&](int p) { return TURN ? ang_c[p] : c4[p & 3]; };
      auto sine = [&](int p) { return TURN ? ang_s[p] : s4[p & 3]; };
      switch (e & 7) {
        case 0:
          if (at == 0) {                                     // the step's queries and angles
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              qh[u] = *reinterpret_cast<const uint2v*>(q_row + u * 128 + 8 * t);
              if (PAIR) ql[u] = *reinterpret_cast<const uint2v*>(q_row + 256 + u * 128 + 8 * t);
            }
            if (!TURN) {
              const float4v c0 = *reinterpret_cast<const float4v*>(bas + 4 * t), s0 = *reinterpret_cast<const float4v*>(bas + 4 * t + kHalf);
              const float4v c1 = *reinterpret_cast<const float4v*>(ang + 4 * t), s1 = *reinterpret_cast<const float4v*>(ang + 4 * t + kHalf);
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                c4[p] = __builtin_fmaf(c1[p], c0[p], -(s1[p] * s0[p]));
                s4[p] = __builtin_fmaf(s1[p], c0[p], c1[p] * s0[p]);
              }
            }
          }
          t1 = high(pa) * sine(pa);
          t2 = low(pa) * sine(pa);
          break;
        case 1:
          lo[0] = __builtin_fmaf(low(pa), cosine(pa), -t1);
          hi[0] = __builtin_fmaf(high(pa), cosine(pa), t2);
          break;
        case 2:
          t1 = high(pb) * sine(pb);
          t2 = low(pb) * sine(pb);
          break;
        case 3:
          lo[1] = __builtin_fmaf(low(pb), cosine(pb), -t1);
          hi[1] = __builtin_fmaf(high(pb), cosine(pb), t2);
          break;
        case 4:
          // (the empty statements: a product and its rounding stay two instructions.  As one, they would round the exact product to hi
          // where lo is measured from the float32 one, and take one instruction per number instead of one per two.)
          asm("" : "+v"(lo[0]), "+v"(lo[1]), "+v"(hi[0]), "+v"(hi[1]));
          x = pack2<F16>(lo[0], lo[1]);
          y = pack2<F16>(hi[0], hi[1]);
          if (PAIR) asm("" : "+v"(x), "+v"(y));
          khi[at] = x;
          khi[2 + at] = y;
          break;
        case 5:
          if (PAIR) {
            l0 = less<F16>(lo[0], x, minus_one);
            l1 = less<F16>(lo[1], x >> 16, minus_one);
          }
          break;
        case 6:
          if (PAIR) {
            l2 = less<F16>(hi[0], y, minus_one);
            l3 = less<F16>(hi[1], y >> 16, minus_one);
          }
          break;
        case 7:
          if (PAIR) {
            klo[at] = pack2<F16>(l0, l1);
            klo[2 + at] = pack2<F16>(l2, l3);
          }
          if (at == 1) {
            const uint4v h = {khi[0], khi[1], khi[2], khi[3]}, q = {qh[0].x, qh[0].y, qh[1].x, qh[1].y};
            dot = mma<F16>(h, q, dot);
            if (PAIR) {
              const uint4v l = {klo[0], klo[1], klo[2], klo[3]}, r = {ql[0].x, ql[0].y, ql[1].x, ql[1].y};
              dot = mma<F16>(h, r, dot);
              dot = mma<F16>(l, q, dot);
            }
          }
          break;
      }
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 2 < KS) af[(ks + 2) % 3] = *reinterpret_cast<const uint4v*>(((ks & 1) ? h1p : h0p) + ((ks + 2) >> 1) * 128);
#pragma unroll
      for (int j = 0; j < FT; ++j) {
        const int slot = ks * FT + j;
        if (slot == kSlots / 2) halfway();
        acc[sub][j] = mma<T>(W[ks][j], af[ks % 3], ks == 0 ? float4v{0, 0, 0, 0} : acc[sub][j]);
#pragma unroll
        for (int e = slot * kSteps / kSlots; e < (slot + 1) * kSteps / kSlots; ++e) step(e);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // lane: query row col, tokens kg + 4 i of sub-tile old
    float* score = reinterpret_cast<float*>(lds + ld.s) + ((np + kPagedScoreSlots) % kPagedScoreSlots * FQ + fq) * (n_packed + 1) * kPagedScorePitch;
    *reinterpret_cast<float4v*>(score + my_row * kPagedScorePitch + 16 * old + 4 * kg) = dot;
  };

  // ---- softmax of tile n: this lane has scores 2 col and 2 col + 1 of row srow, of tokens stok and stok + 4
  auto softmax = [&](int n) __attribute__((always_inline)) {
    const int l = fresh_lane(), col = l & 15, srow = 4 * (wave & 3) + (l >> 4), stok = 16 * (col >> 3) + 8 * (col & 1) + (col >> 1 & 3);
    const int buf = n & 1, t0 = w.tile_pos(n) + stok, r = min(srow, n_packed);
    const float* row = reinterpret_cast<const float*>(lds + ld.s) + (n % kPagedScoreSlots * FQ * (n_packed + 1) + r) * kPagedScorePitch + 2 * col;
    float s0 = row[0], s1 = row[1];
#pragma unroll
    for (int f = 1; f < FQ; ++f) {
      s0 += row[f * (n_packed + 1) * kPagedScorePitch];
      s1 += row[f * (n_packed + 1) * kPagedScorePitch + 1];
    }
    if (t0 >= limit || (t0 >= w.span.sink && t0 < w.span.lo)) s0 = -INFINITY;
    if (t0 + 4 >= limit || (t0 + 4 >= w.span.sink && t0 + 4 < w.span.lo)) s1 = -INFINITY;
    const float now = fmaxf(run_max, max_of_row(fmaxf(s0, s1)));
    const float zero = now == -INFINITY ? 0.f : now;         // no row seen yet: exp2(-inf) = 0 below
    const float alpha = __builtin_amdgcn_exp2f(run_max - zero);
    const float p0 = __builtin_amdgcn_exp2f(s0 - zero), p1 = __builtin_amdgcn_exp2f(s1 - zero);
    uint32_t hi, lo;
    split2<T>(p0, p1, &hi, &lo);
    run_max = now;
    run_sum = run_sum * alpha + (p0 + p1);
    // in the order of the value product's contraction: lane group kg', token kg' + 4 e
    unsigned char* P = lds + ld.p + (buf * 17 + min(srow, 16)) * kPagedProbPitch + 16 * (col >> 1 & 3) + 8 * (col >> 3) + 4 * (col & 1);
    *reinterpret_cast<uint32_t*>(P) = hi;
    *reinterpret_cast<uint32_t*>(P + 64) = lo;
    reinterpret_cast<float*>(lds + ld.alpha)[buf * 20 + srow] = alpha;
  };

  // ---- values of tile n, staged at v_stage
  auto values = [&](int n, int v_stage) __attribute__((always_inline)) {
    const int l = fresh_lane(), col = l & 15, kg = l >> 4, v_lane = kg * ld.v_pieces * 16 + (col & 3) * 4, v_pitch16 = 4 * ld.v_pieces * 16;
    const int buf = n & 1;
    const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (buf * 20 + 4 * kg) * 4);
    const unsigned char* P = lds + ld.p + (buf * 17 + col) * kPagedProbPitch + 16 * kg;
    const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 64);
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
      O[v][0] = mma<T>(hi, f0, O[v][0] * al);
      O[v][1] = mma<T>(hi, f1, O[v][1] * al);
      O[v][0] = mma<T>(lo, f0, O[v][0]);
      O[v][1] = mma<T>(lo, f1, O[v][1]);
    }
  };

  for (int n = i0; n < i1 + 3; ++n) {
    const bool more_k = n + NB - 1 < i1, more_v = n + NB - 4 >= i0 && n + NB - 4 < i1;
    const int to_k = ring_k.before(k_at), to_v = ring_v.before(v_at);
    if (more_k) rows_of(n + NB - 1, x_k, IntC<KR>(), row_k);
    if (more_v) rows_of(n + NB - 4, x_v, IntC<VR>(), row_v);
    request_entries(n);
    if (wave == 3) {
      angles.request(n + NB + (TURN ? 1 : 0), i0 + 1);
      if (n + 1 + (TURN ? 1 : 0) < i1) angles.make(n + 1 + (TURN ? 1 : 0));
    }
    // The first wavefronts of the SIMDs end with the keys, the others begin with them: the matrix instructions of one run beside the rest
    // of the other.
    const bool front = wave < 4;
    auto rest = [&]() __attribute__((always_inline)) {
      if (!front && 4 * (wave & 3) < n_packed && n >= i0 + 2 && n < i1 + 2) softmax(n - 2);
      if (n >= i0 + 3) values(n - 3, v_at);
      if (TURN && n + 1 < i1) turn_queries(n + 1);
    };
    auto request = [&](int part) __attribute__((always_inline)) {
      if (part < 2) {
        if (more_k) request_keys(part, row_k, to_k);
      } else {
        if (more_v) request_values(part - 2, row_v, to_v);
      }
    };
    if (front) {
      request(0);
      rest();
    }
    if (n <= i1)                                             // (behind the last tile, and of the one before the first: nothing that is used)
      keys(IntC<0>(), k_at, n - 1, b_old, [&]() __attribute__((always_inline)) { if (front) request(1); else request(0); });
    if (front) request(2);
    else request(1);
    if (n < i1) {
      keys(IntC<1>(), k_at, n, b_at, [&]() __attribute__((always_inline)) { if (front) request(3); else request(2); });
    } else {
      if (front) request(3);
      else request(2);
    }
    if (!front) {
      request(3);
      rest();
    }
    k_at = ring_k.behind(k_at);
    v_at = ring_v.behind(v_at);
    b_old = b_at;
    b_at = ring_b.behind(b_at);
    // what interval n + 1 reads was requested in n - NB + 2; the NB - 2 intervals since then may be outstanding where all of them
    // requested whole tiles
    if (n > i0 && n + NB - 1 < i1) wait_vm(steady);
    else wait_vm(0);
    lds_barrier();
  }

  // ---- partial results
#pragma unroll
  for (int d = 1; d < 16; d *= 2) run_sum += __shfl_xor(run_sum, d);
  if (wave >= 4 && srow < n_packed && col == 0) w.store_ml(srow / nr, srow % nr, run_max, run_sum);
#pragma unroll
  for (int v = 0; v < VB; ++v) {
    const int block = wave + 8 * v;
    if (block >= n_blocks) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * kg + e < n_packed) w.store_o(4 * kg + e, block * 32 + 2 * col, O[v][0][e], O[v][1][e]);
  }
}

namespace {
template <typename T, int FQ, int KS>
PagedFn pick(const PagedForm& f) {
  if (f.turned) return f.vb == 1 ? paged_kernel<T, FQ, KS, 1, true> : paged_kernel<T, FQ, KS, 2, true>;
  return f.vb == 1 ? paged_kernel<T, FQ, KS, 1, false> : paged_kernel<T, FQ, KS, 2, false>;
}
}  // namespace

template <typename T> PagedFn paged_form(const PagedForm& f) {
  switch (f.ks) {
    case 2: return pick<T, 2, 2>(f);
    case 4: return pick<T, 2, 4>(f);
    case 6: return pick<T, 2, 6>(f);
    case 8: return pick<T, 2, 8>(f);
    case 12: return pick<T, 4, 12>(f);
    default: return pick<T, 4, 16>(f);
  }
}
template PagedFn paged_form<PALU_PAGED_ACT>(const PagedForm&);

}  // namespace palu
