// Decode attention over a paged latent cache, for key ranks above 256 (paged.hip takes the others, and explains the arithmetic).
//
// The weights of a head do not fit one wavefront: eight wavefronts, two per SIMD, share two heads, each with 16 of a head's 64
// rotation pairs at all latent channels.  Per tile of 32 tokens: partial scores to LDS, barrier, softmax (four threads per row add
// the partial scores), barrier; a tile's values are contracted beside the next tile's keys.  Loads to LDS run n_stages - 1 tiles ahead.

#include "paged_dev.h"

namespace palu {

template <typename T, int VB>
__global__ __launch_bounds__(kPagedWideThreads, 2) void paged_wide_kernel(PagedArgs a) {
  constexpr bool PAIR = __is_same(T, F16);     // queries and keys as pairs hi + lo
  constexpr int HL = PAIR ? 2 : 1;
  constexpr int FQ = kPagedWideParts;          // a head's rotation pairs go to this many wavefronts, 16 to each
  constexpr int KSM = 16;                      // steps of 32 latent channels, at most
  constexpr int SUB = kPagedTile / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  // ---- what this workgroup does
  const int bid = blockIdx.x;
  const PagedUnit un = a.units[bid % a.n_units];
  int rest = bid / a.n_units;
  const int rb = rest % a.n_row_blocks;
  rest /= a.n_row_blocks;
  const bool shared = a.shared != 0;
  const int seq = shared ? 0 : rest / a.n_slots;
  const int chunk = rest - seq * a.n_slots;
  int L = shared || !a.seq_lens ? a.max_len : a.seq_lens[seq];
  L = __builtin_amdgcn_readfirstlane(max(0, min(L, a.max_len)));
  const PagedSpan span = paged_span(L, a.first, a.window, a.n_sink);
  const int n_chunks = (span.n_tiles + a.chunk_tiles - 1) / a.chunk_tiles;
  if (chunk >= n_chunks) return;
  const int i0 = (int)((long long)span.n_tiles * chunk / n_chunks), i1 = (int)((long long)span.n_tiles * (chunk + 1) / n_chunks);

  const PagedMeta& m = a.meta;
  const int g = un.group(), nh = un.nh(), h0 = un.h0();
  const int rk = m.k_off[g + 1] - m.k_off[g], rv = m.v_off[g + 1] - m.v_off[g];
  const int per_group = m.head_off[g + 1] - m.head_off[g];   // a unit of several groups takes whole ones
  const int k_cols = rk, v_cols = rv;                        // (units of one group)
  const int nks = rk / 32;
  const int row0 = rb * a.block_rows;
  const int nr = min(a.block_rows, a.rows - row0);           // rows per head, at most 8
  const int n_packed = nh * nr;
  const int NB = a.n_stages;
  const PagedWideLds ld = paged_wide_lds(k_cols, v_cols, n_packed, PAIR, NB);
  const uint32_t lds0 = lds_addr(lds);

  const int hh = wave & 1, fq = wave >> 1;
  const int fbase = 16 * fq;                                 // first rotation pair of this wavefront
  const bool works = hh < nh;

  // position of tile i, and the position whose row its token x reads (a masked token: the first attended one's)
  auto tile_pos = [&](int i) { return kPagedTile * (i < span.sink_tiles ? i : span.tile0 + i - span.sink_tiles); };
  auto token_of = [&](int t0, int x) __attribute__((always_inline)) {
    const int t = t0 + x, head = t0 < span.sink ? t0 : max(t0, span.lo);
    return t >= L || (t >= span.sink && t < span.lo) ? head : t;
  };
  const int32_t* pages = a.page_table + (size_t)seq * a.table_stride;
  const int page_mask = (1 << a.page_shift) - 1;
  auto row_of = [&](int t, int entry) __attribute__((always_inline)) {
    return ((size_t)max(0, min(entry, a.n_pages - 1)) << a.page_shift) + (t & page_mask);
  };
  const int E = 2 * NB - 2;                                  // entries are requested so many tiles ahead: early enough to be there when rows are

  // ---- requests of interval n: keys and angles of tile n + NB - 1, values of n + NB - 2, entries of n + E.
  // 16-byte piece p of a key row goes to piece p ^ (t % 8) (eight tokens' same pieces lie on all banks), of a value row to
  // p ^ 4 (t / 8) (the four tokens that a lane group reads at a time do).
  const uint32_t inv_k = ((1u << 20) + ld.k_pieces - 1) / ld.k_pieces, inv_v = ((1u << 20) + ld.v_pieces - 1) / ld.v_pieces;
  const int ops_k = ld.k_pieces / 2, ops_v = ld.v_pieces / 2;   // of 64 pieces, dealt out to the wavefronts
  const uint16_t* hk = a.hk + m.k_off[g];
  const uint16_t* hv = a.hv + m.v_off[g];
  const int* entries = reinterpret_cast<const int*>(lds + ld.entries);
  auto request = [&](int n) __attribute__((always_inline)) {
    const int jk = n + NB - 1, jv = n + NB - 2, je = n + E;
    if (jk < i1) {
      const int t0 = tile_pos(jk);
      const int slot = jk % NB;
      const int* ent = entries + (jk % kPagedEntrySlots) * kPagedTile;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int op = k * 8 + wave;
        if (op < ops_k) {
          const uint32_t id = (uint32_t)(op * 64 + lane), x = (id * inv_k) >> 20;
          const uint32_t p = (id - x * ld.k_pieces) ^ (x & 7);
          const size_t row = row_of(token_of(t0, x), ent[x]);
          if ((int)p * 8 < k_cols) load_to_lds(hk + row * a.R_k + p * 8, lds0 + ld.k + slot * ld.stage_k + op * 1024);
        }
      }
      if (wave < 2 * SUB) {                                  // angles: (sub-tile, cos | sin) of this wavefront, lane: pair
        const int p = min(t0 + 16 * (wave >> 1), a.rope_len - 1);
        load_to_lds4(a.rope + rope_f32_index(p, lane, wave & 1, kRopeTableStride), lds0 + ld.base + (slot * 2 * SUB + wave) * 256);
      }
    }
    if (jv >= i0 && jv < i1) {
      const int t0 = tile_pos(jv);
      const int* ent = entries + (jv % kPagedEntrySlots) * kPagedTile;
#pragma unroll
      for (int k = 0; k < 2 * VB; ++k) {
        const int op = k * 8 + wave;
        if (op < ops_v) {
          const uint32_t id = (uint32_t)(op * 64 + lane), x = (id * inv_v) >> 20;
          const uint32_t p = (id - x * ld.v_pieces) ^ (4 * (x >> 3));
          const size_t row = row_of(token_of(t0, x), ent[x]);
          if ((int)p * 8 < v_cols) load_to_lds(hv + row * a.R_v + p * 8, lds0 + ld.v + (jv % NB) * ld.stage_v + op * 1024);
        }
      }
    }
    if (je < i1 && wave == 7 && lane < kPagedTile)
      load_to_lds4(pages + (token_of(tile_pos(je), lane) >> a.page_shift), lds0 + ld.entries + (je % kPagedEntrySlots) * (kPagedTile * 4));
  };
  const int per_interval = (ops_k - wave + 7) / 8 + (ops_v - wave + 7) / 8 + (wave < 2 * SUB ? 1 : 0);

  // ---- prologue
  if (tid < 32 * E) {                                        // entries of the first tiles
    const int i = i0 + (tid >> 5);
    if (i < i1) reinterpret_cast<int*>(lds + ld.entries)[(i % kPagedEntrySlots) * kPagedTile + (tid & 31)] = pages[token_of(tile_pos(i), tid & 31) >> a.page_shift];
  }
  lds_barrier();
  for (int n = i0 - NB + 1; n < i0; ++n) request(n);

  // angles of the first 16 positions, scaled
  float* const angles = reinterpret_cast<float*>(lds + ld.ang);
  for (int x = tid; x < 16 * kDHead; x += kPagedWideThreads) {
    const int t = x & 15, c = x >> 4;
    angles[t * kPagedAngPitch + c] = kKeyScale * a.rope[rope_f32_index(t, c & 63, c >> 6, kRopeTableStride)];
  }
  // rotated queries: [packed row][feature part][hi | lo][lane group] x 16 bytes: four low halves, four high halves of pairs
  for (int x = tid; x < n_packed * kHalf; x += kPagedWideThreads) {
    const int f = x & 63, pr = x >> 6;
    const int h = pr / nr, r = pr - h * nr;
    int b = seq, qh = row0 + r;
    if (shared) { b = qh / m.qpk; qh -= b * m.qpk; }
    const uint16_t* qp = a.q + ((size_t)b * m.n_heads * m.qpk + (h0 + h) * m.qpk + qh) * kDHead;
    const float x0 = T::to_float(qp[f]), x1 = T::to_float(qp[f + kHalf]);
    int pos = a.q_pos ? a.q_pos[b] : (a.seq_lens ? a.seq_lens[b] : a.pos_len) - 1;
    pos = max(0, min(pos, a.rope_len - 1));
    const float k = a.scale / kKeyScale;
    const float c = a.rope[rope_f32_index(pos, f, 0, kRopeTableStride)] * k, s = a.rope[rope_f32_index(pos, f, 1, kRopeTableStride)] * k;
    const float y0 = x0 * c - x1 * s, y1 = x1 * c + x0 * s;
    uint32_t hi, lo;
    split2<F16>(y0, y1, &hi, &lo);
    uint16_t* q = reinterpret_cast<uint16_t*>(lds + ld.q + pr * ld.q_pitch + ((f >> 4) * HL * 4 + ((f >> 2) & 3)) * 16) + (f & 3);
    q[0] = (uint16_t)hi;
    q[4] = (uint16_t)(hi >> 16);
    if (PAIR) {
      q[32] = (uint16_t)lo;
      q[36] = (uint16_t)(lo >> 16);
    }
  }

  // weights: tile 0: pairs' low halves, feature fbase + m in row m, tile 1: high halves.  Eight consecutive latent channels per lane.
  uint4v W[KSM][2];
  {
    const int width = per_group * kDHead;
    const uint16_t* B = a.Bk + m.bk_off[g] + (size_t)((works ? hh : 0) + h0 - m.head_off[g]) * kDHead + fbase + col;
#pragma unroll
    for (int ks = 0; ks < KSM; ++ks) {
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        W[ks][side] = uint4v{0, 0, 0, 0};
        if (ks < nks) {
          const uint16_t* p = B + (size_t)(32 * ks + 8 * kg) * width + side * kHalf;
#pragma unroll
          for (int i = 0; i < 4; ++i) W[ks][side][i] = p[(size_t)(2 * i) * width] | ((uint32_t)p[(size_t)(2 * i + 1) * width] << 16);
        }
      }
    }
  }

  const int n_blocks = v_cols / 32;                          // of 32 value columns, one (VB) per wavefront
  float4v O[VB][2];
#pragma unroll
  for (int v = 0; v < VB; ++v) O[v][0] = O[v][1] = float4v{0, 0, 0, 0};

  // softmax state of thread (row, quarter); rows the row may see
  const int srow = tid >> 2, squart = tid & 3;
  float run_max = -INFINITY, run_sum = 0.f;
  int limit = L;
  if (shared && srow < n_packed) limit = min(L, a.seq_lens ? a.seq_lens[(row0 + srow % nr) / m.qpk] : L);

  wait_vm(0);
  lds_barrier();

  // ---- keys of tile n and their scores
  auto keys = [&](int n) __attribute__((always_inline)) {
    const int slot = n % NB;
    const int off0 = (kg ^ (lane & 7)) * 16, off1 = ((4 + kg) ^ (lane & 7)) * 16;
    const unsigned char* qf = lds + ld.q + (hh * nr + min(col, nr - 1)) * ld.q_pitch + (fq * HL * 4 + kg) * 16;
    float* Sc = reinterpret_cast<float*>(lds + ld.s) + fq * (16 * kPagedScorePitch);
#pragma unroll
    for (int x = 0; x < SUB; ++x) {
      const unsigned char* hrow = lds + ld.k + slot * ld.stage_k + (16 * x + col) * ld.k_pieces * 16;
      float4v acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
      for (int ks = 0; ks < KSM; ++ks) {
        if (ks < nks) {
          const uint4v h = *reinterpret_cast<const uint4v*>(hrow + (ks >> 1) * 128 + ((ks & 1) ? off1 : off0));
          acc[0] = mma<T>(W[ks][0], h, acc[0]);
          acc[1] = mma<T>(W[ks][1], h, acc[1]);
        }
      }
      // rotate; lane: token col, pairs fbase + 4 kg + i
      const float* bas = reinterpret_cast<const float*>(lds + ld.base) + (slot * SUB + x) * kDHead + fbase + 4 * kg;
      const float* ang = angles + col * kPagedAngPitch + fbase + 4 * kg;
      const float4v c0 = *reinterpret_cast<const float4v*>(bas), s0 = *reinterpret_cast<const float4v*>(bas + kHalf);
      const float4v c1 = *reinterpret_cast<const float4v*>(ang), s1 = *reinterpret_cast<const float4v*>(ang + kHalf);
      float lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float c = __builtin_fmaf(c1[i], c0[i], -(s1[i] * s0[i])), s = __builtin_fmaf(s1[i], c0[i], c1[i] * s0[i]);
        lo[i] = __builtin_fmaf(acc[0][i], c, -(acc[1][i] * s));
        hi[i] = __builtin_fmaf(acc[1][i], c, acc[0][i] * s);
      }
      uint32_t kh[4], kl[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (PAIR) {
          split2<F16>(lo[2 * e], lo[2 * e + 1], &kh[e], &kl[e]);
          split2<F16>(hi[2 * e], hi[2 * e + 1], &kh[2 + e], &kl[2 + e]);
        } else {
          kh[e] = pack2<F16>(lo[2 * e], lo[2 * e + 1]);
          kh[2 + e] = pack2<F16>(hi[2 * e], hi[2 * e + 1]);
        }
      }
      const uint4v qh = *reinterpret_cast<const uint4v*>(qf), k = {kh[0], kh[1], kh[2], kh[3]};
      float4v s = mma<F16>(k, qh, float4v{0, 0, 0, 0});
      if (PAIR) {
        const uint4v ql = *reinterpret_cast<const uint4v*>(qf + 64), l = {kl[0], kl[1], kl[2], kl[3]};
        s = mma<F16>(k, ql, s);
        s = mma<F16>(l, qh, s);
      }
      if (col < nr) *reinterpret_cast<float4v*>(&Sc[(hh * nr + col) * kPagedScorePitch + 16 * x + 4 * kg]) = s;   // lane: query row col, tokens 4 kg ..
    }
  };

  // ---- softmax of tile n
  auto softmax = [&](int n) __attribute__((always_inline)) {
    if (srow >= n_packed) return;
    const int t0 = tile_pos(n) + 8 * squart;
    const float* row = reinterpret_cast<const float*>(lds + ld.s) + srow * kPagedScorePitch + 8 * squart;
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = row[e];
#pragma unroll
    for (int f = 1; f < FQ; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += row[f * (16 * kPagedScorePitch) + e];
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = t0 + e;
      if (t >= limit || (t >= span.sink && t < span.lo)) s[e] = -INFINITY;
      top = fmaxf(top, s[e]);
    }
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
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
    unsigned char* P = lds + ld.p + srow * kPagedProbPitch + 16 * squart;
    *reinterpret_cast<uint4v*>(P) = uint4v{ph[0], ph[1], ph[2], ph[3]};
    *reinterpret_cast<uint4v*>(P + 64) = uint4v{pl[0], pl[1], pl[2], pl[3]};
    if (squart == 0) reinterpret_cast<float*>(lds + ld.alpha)[srow] = alpha;
  };

  // ---- values of tile n
  auto values = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < VB; ++v) {
      const int block = wave + 8 * v;
      if (block < n_blocks) {
        uint32_t x[8];
        const unsigned char* row = lds + ld.v + (n % NB) * ld.stage_v + 8 * kg * ld.v_pieces * 16 + ((block * 4 + (col >> 2)) ^ (4 * kg)) * 16 + (col & 3) * 4;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = *reinterpret_cast<const uint32_t*>(row + e * ld.v_pieces * 16);
        uint4v f0, f1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f0[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);
          f1[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);
        }
        const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + 4 * kg * 4);
        const unsigned char* P = lds + ld.p + col * kPagedProbPitch + 16 * kg;
        const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 64);
        O[v][0] = mma<T>(hi, f0, O[v][0] * al);
        O[v][1] = mma<T>(hi, f1, O[v][1] * al);
        O[v][0] = mma<T>(lo, f0, O[v][0]);
        O[v][1] = mma<T>(lo, f1, O[v][1]);
      }
    }
  };

  for (int n = i0; n < i1 + 1; ++n) {
    request(n);
    if (n - 1 >= i0) values(n - 1);
    if (n < i1 && works) keys(n);
    lds_barrier();
    if (n < i1) softmax(n);
    // what interval n + 1 reads was requested in n - NB + 2; the NB - 2 intervals since then may be outstanding where all of them
    // requested whole tiles
    if (n + NB - 1 < i1) wait_vm((NB - 2) * (per_interval + (wave == 7 && n + E < i1 ? 1 : 0)));
    else wait_vm(0);
    lds_barrier();
  }

  // ---- partial results
  run_sum += __shfl_xor(run_sum, 1);
  run_sum += __shfl_xor(run_sum, 2);
  const size_t slot = shared ? (size_t)chunk : (size_t)seq * a.n_slots + chunk;
  if (srow < n_packed && squart == 0) {
    const int h = srow / nr, r = srow - h * nr;
    float2* ml = reinterpret_cast<float2*>(a.ml_part) + slot * m.n_heads * a.rows + (size_t)(h0 + h) * a.rows + row0 + r;
    *ml = make_float2(run_max, run_sum);
  }
#pragma unroll
  for (int v = 0; v < VB; ++v) {
    const int block = wave + 8 * v;
    if (block >= n_blocks) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int pr = 4 * kg + e;
      if (pr < n_packed) {
        const int h = pr / nr, r = pr - h * nr;
        const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
        float* o = a.o_part + slot * a.o_stride + (size_t)a.rows * ohead + (size_t)(row0 + r) * rv + block * 32 + 2 * col;
        *reinterpret_cast<float2*>(o) = make_float2(O[v][0][e], O[v][1][e]);
      }
    }
  }
}

template <typename T> PagedFn paged_wide_form(int vb) { return vb == 1 ? paged_wide_kernel<T, 1> : paged_wide_kernel<T, 2>; }
template PagedFn paged_wide_form<F16>(int);
template PagedFn paged_wide_form<BF16>(int);

}  // namespace palu
