// Decode attention over a paged 4-bit latent cache on the matrix cores, part of the query folded into the weights.
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v,   H[t, r] = (code - zero) * scale
//
// With q' the query rotated to its own position, a key's pair (k, k') of features (f, f + 64) adds  k a_f(t) + k' b_f(t)  to the score,
//   a_f(t) = cos(w_f t) q'_f + sin(w_f t) q'_{f+64},   b_f(t) = cos(w_f t) q'_{f+64} - sin(w_f t) q'_f,   w_f = theta^(-f/64).
// Pairs 0 .. 31 turn fast: their keys are rebuilt, 64 features a head.  Pairs 32 .. 63 turn by 1.3 radians at most in 128 positions:
// over a span of up to 256 positions their a_f and b_f are polynomials of degree 7 in t to 2e-6 of the fastest, and far less of the others, so
//   sum_{f >= 32} = sum_{i < 8} L_i(t)  h_t . g_i,   g_i[r] = sum_f B_k[r, f] a_f(t_i) + B_k[r, f + 64] b_f(t_i),
// with t_i the Chebyshev nodes of the span and L_i their Lagrange polynomials: 16 rows of weights (g_i as a pair of float16
// numbers) instead of 64, made anew once per span by a sixteenth of the work that they save.

#include "paged_dev.h"
#include "pagedq.h"

namespace palu {

namespace {

constexpr int kSteps = kPagedQStep;
constexpr float kWeightScale = 16384.f;        // of the values' weights in float16 pairs: 2^-39 of the largest is left of the others

// a and b with the upper half of a and the lower half of b exchanged; the same of odd and even rows of 16 lanes
struct Swapped {
  float a, b;
};
__device__ __forceinline__ Swapped swap32(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const uint32_t r0 = r[0], r1 = r[1];                       // (a bit cast of r[1] itself takes r[0])
  return Swapped{__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)};
}
__device__ __forceinline__ Swapped swap16(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const uint32_t r0 = r[0], r1 = r[1];
  return Swapped{__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1)};
}
__device__ __forceinline__ float max_of_wave(float x) {
  x = max_with<0x140>(max_of_8(x));            // mirrored in 16 lanes
  const Swapped r = swap16(x, x);
  x = fmaxf(r.a, r.b);
  const Swapped h = swap32(x, x);
  return fmaxf(h.a, h.b);
}
__device__ __forceinline__ float sum_of_wave(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float add_swapped32(float a, float b) {
  const Swapped r = swap32(a, b);
  return r.a + r.b;
}
__device__ __forceinline__ float add_swapped16(float a, float b) {
  const Swapped r = swap16(a, b);
  return r.a + r.b;
}
// x plus that of the lane 8 on among 16
__device__ __forceinline__ float add_8_on(float x) {
  const int u = __builtin_bit_cast(int, x);
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, 0x128, 0xf, 0xf, false));
}
__device__ __forceinline__ bool small_integer(float z) { return fabsf(z) <= 1000.f && z == rintf(z); }

// 16-bit weights as float16 numbers: as they are, or bfloat16 ones times 2^shift (exact down to 2^-31 of the largest, right to 2^-39 of it below)
template <typename T> __device__ __forceinline__ uint32_t to_f16(uint32_t w, int shift);
template <> __device__ __forceinline__ uint32_t to_f16<F16>(uint32_t w, int) { return w; }
template <> __device__ __forceinline__ uint32_t to_f16<BF16>(uint32_t w, int shift) {
  const float x = __builtin_amdgcn_ldexpf(BF16::to_float((uint16_t)w), shift), y = __builtin_amdgcn_ldexpf(BF16::to_float((uint16_t)(w >> 16)), shift);
  return pack2<F16>(x, y);
}

}  // namespace

// KS steps of 32 key channels per wavefront; SL wavefronts share a head's channels; NQ query rows of a head
template <typename T, int KS, int SL, int NQ>
__global__ __launch_bounds__(kPagedQThreads, 1) void pagedq_kernel(PagedQArgs a) {
  constexpr int HEADS = 4 / SL;                // of a unit
  constexpr int NB = KS / 4;                   // blocks of 128 channels
  constexpr int LG = NQ == 1 ? 1 : NQ / 2;     // folded query rows, 16 (row, node) a group
  constexpr int NG = NQ == 1 ? 1 : NQ;         // tiles of folded weights: of one row hi and lo in one tile, else apart
  constexpr int MAXCB = 4;
  constexpr int kLoRows = NQ == 1 ? 4 : (SL == 1 ? 16 : 8);  // rows of probabilities before those that the rounding left
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const PagedMeta& m = a.meta;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  // ---- what this workgroup does
  const PagedUnit un = a.units[blockIdx.x % a.n_units];
  int rest = blockIdx.x / a.n_units;
  const int rb = rest % a.n_row_blocks;
  rest /= a.n_row_blocks;
  const int seq = rest / a.n_slots, chunk = rest - seq * a.n_slots;
  const int L = __builtin_amdgcn_readfirstlane(max(0, min(a.seq_lens ? a.seq_lens[seq] : a.max_len, a.max_len)));
  const PagedSpan span = paged_span(L, 0, a.window, a.n_sink);
  const int n_chunks = (span.n_tiles + a.chunk_tiles - 1) / a.chunk_tiles;
  if (chunk >= n_chunks) return;
  const int i0 = (int)((long long)span.n_tiles * chunk / n_chunks), i1 = (int)((long long)span.n_tiles * (chunk + 1) / n_chunks);
  const int g = un.group(), nh = un.nh(), h0 = un.h0();
  const int rk = m.k_off[g + 1] - m.k_off[g], rv = m.v_off[g + 1] - m.v_off[g], per_group = m.head_off[g + 1] - m.head_off[g];
  const int k_cols = un.n_groups() * rk, v_cols = un.n_groups() * rv, CB = v_cols / 128;
  const int row0 = rb * NQ, nr = min(NQ, m.qpk - row0);      // query rows of a head
  const PagedQLds ld = pagedq_lds(k_cols, v_cols, SL, NQ);
  const uint32_t lds0 = lds_addr(lds);

  const int hw = wave % HEADS, slice = wave / HEADS;
  const int hh = min(hw, nh - 1);                            // (a wavefront without a head does another one's work, results nowhere)
  const int hg = un.n_groups() > 1 ? hh / per_group : 0;     // the head's group in the unit
  const int width = per_group * kDHead;
  const uint16_t* const B = a.Bk + m.bk_off[g] + (size_t)hg * rk * width + (size_t)(hh + h0 - m.head_off[g] - hg * per_group) * kDHead;
  const int ks_here = min(KS, (rk - slice * KS * 32) / 32);  // steps of this slice

  // ---- steps of 64 positions: those of the sinks' tiles first
  const int mid = max(i0, min(i1, span.sink_tiles));
  const int steps_s = (mid - i0 + 1) / 2, n_steps = steps_s + (i1 - mid + 1) / 2;
  const int pos_w = kPagedTile * (span.tile0 + mid - span.sink_tiles);     // (where mid < i1)
  auto pos_of = [&](int n) __attribute__((always_inline)) { return n < steps_s ? kPagedTile * i0 + kSteps * n : pos_w + kSteps * (n - steps_s); };
  auto end_of = [&](int n) __attribute__((always_inline)) { return min(L, n < steps_s ? kPagedTile * mid : pos_w + kPagedTile * (i1 - mid)); };
  auto attended = [&](int n, int t) __attribute__((always_inline)) { return t < end_of(n) && (t < span.sink || t >= span.lo); };
  auto folds = [&](int n) __attribute__((always_inline)) { return (n < steps_s ? n : n - steps_s) % a.span_steps == 0; };

  // ---- requests.  In interval n: keys, scales and angles of step n + 2, values of n + 1, page-table entries of n + 4.
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  const int k_pieces = k_cols / 32, v_pieces = v_cols / 32;  // 16-byte pieces of a raw row
  const int k_block0 = m.k_off[g] / 128, v_block0 = m.v_off[g] / 128;
  uint16_t zraw[4], tok_raw[8];
  int entry = 0;
  float anchor_c = 0.f, anchor_s = 0.f;
  auto token_of = [&](int n, int x) __attribute__((always_inline)) {       // the position whose row token x reads (a masked token: the first attended one's)
    const int t0 = pos_of(n), t = t0 + x;
    return attended(n, t) ? t : (t0 < span.sink ? t0 : max(t0, span.lo));
  };
  auto entry_of = [&](int n) __attribute__((always_inline)) {
    return a.page_table[(size_t)seq * a.table_stride + (token_of(n, lane) >> a.page_shift)];
  };
  auto put_rows = [&](int n, int e) __attribute__((always_inline)) {
    rows[(n & 3) * kSteps + lane] = (max(0, min(e, a.n_pages - 1)) << a.page_shift) + (token_of(n, lane) & ((1 << a.page_shift) - 1));
  };
  auto request_keys = [&](int n) __attribute__((always_inline)) {
    const int* const r = rows + (n & 3) * kSteps;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i * 128 >= k_cols) break;
      const int id = i * kPagedQThreads + tid, x = id / k_pieces, pc = id - x * k_pieces;
      const size_t row = r[x];
      load_to_lds(a.k.codes + row * a.k.row_bytes + m.k_off[g] / 2 + pc * 16, lds0 + ld.raw + (SL == 1 ? (n & 1) * ld.raw_size : 0) + (i * kPagedQThreads + wave * 64) * 16);
      zraw[i] = a.k.zero[row * a.k.n_blocks + k_block0 + (pc >> 2)];
    }
    if (wave < 2) {                            // scales and zero-points by token
      const PagedQSide& s = wave == 0 ? a.k : a.v;
      const int blocks = wave == 0 ? k_cols / 128 : CB;
      const size_t at = (size_t)r[lane] * s.n_blocks + (wave == 0 ? k_block0 : v_block0);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b >= blocks) break;
        tok_raw[b] = s.scale[at + b];
        tok_raw[4 + b] = s.zero[at + b];
      }
    }
    if (wave == 2 && folds(n)) {
      anchor_c = a.rope[rope_f32_index(pos_of(n), lane, 0, kRopeTableStride)];
      anchor_s = a.rope[rope_f32_index(pos_of(n), lane, 1, kRopeTableStride)];
    }
  };
  constexpr int VBUFS = SL == 1 ? 3 : 2;
  auto request_values = [&](int n) __attribute__((always_inline)) {
    const int* const r = rows + (n & 3) * kSteps;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i * 128 >= v_cols) break;
      const int id = i * kPagedQThreads + tid, x = id / v_pieces, pc = id - x * v_pieces;
      load_to_lds(a.v.codes + (size_t)r[x] * a.v.row_bytes + m.v_off[g] / 2 + pc * 16, lds0 + ld.v + (n % VBUFS) * ld.v_size + (i * kPagedQThreads + wave * 64) * 16);
    }
  };
  // ---- what came of them: scales by token; keys as float16 numbers, code - zero where the zero-point is a small integer (else the code)
  float2* const k_tok = reinterpret_cast<float2*>(lds + ld.k_tok);
  float* const k_left = reinterpret_cast<float*>(lds + ld.k_tok + 2 * kSteps * 2 * 8);
  float2* const v_tok = reinterpret_cast<float2*>(lds + ld.v_tok);
  float* const anchors = reinterpret_cast<float*>(lds + ld.anchors);
  int* const flags = reinterpret_cast<int*>(lds + ld.flags);
  auto put_tokens = [&](int n) __attribute__((always_inline)) {
    if (wave == 0) {
      bool any = false;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b * 128 >= k_cols) break;
        const float z = F16::to_float(tok_raw[4 + b]);
        const float left = small_integer(z) ? 0.f : z;
        any = any || !(left == 0.f);
        k_left[((n & 1) * 4 + b) * kSteps + lane] = left;
      }
      const int some = __any(any) ? 1 : 0;
      if (lane == 0) flags[n & 1] = some;
#pragma unroll
      for (int s = 0; s < 2; ++s) {            // blocks of a slice, or of a group: (first * ratio + second) * scale.  (A second scale of zero: so
        if (s * NB * 128 >= k_cols) break;     // small a number that nothing of the second block is left.)
        const float s0 = F16::to_float(tok_raw[NB * s]);
        float s1 = s0, ratio = 1.f;
        if (NB == 2 && (2 * s + 1) * 128 < k_cols) {
          s1 = F16::to_float(tok_raw[2 * s + 1]);
          if (s1 == 0.f) s1 = 0x1p-60f;
          ratio = s0 / s1;
        }
        k_tok[((n & 1) * 2 + s) * kSteps + lane] = make_float2(ratio, s1);
      }
    }
    if (wave == 1) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b >= CB) break;
        v_tok[((n & 1) * CB + b) * kSteps + lane] = make_float2(F16::to_float(tok_raw[b]), F16::to_float(tok_raw[4 + b]));
      }
    }
    if (wave == 2 && folds(n)) {
      anchors[(n & 1) * kDHead + lane] = anchor_c;
      anchors[(n & 1) * kDHead + kHalf + lane] = anchor_s;
    }
  };
  const uint32_t k1024 = per_lane_constant(0x64006400u);
  // piece i of this thread
  auto convert = [&](int n, int i, uint16_t z16) __attribute__((always_inline)) {
    const int id = i * kPagedQThreads + tid, x = id / k_pieces, pc = id - x * k_pieces;
    const uint4v w = *reinterpret_cast<const uint4v*>(lds + ld.raw + (SL == 1 ? (n & 1) * ld.raw_size : 0) + id * 16);
    const float z = F16::to_float(z16);
    const half2v off = {(_Float16)(-1024.f - (small_integer(z) ? z : 0.f)), (_Float16)(-1024.f - (small_integer(z) ? z : 0.f))};
    unsigned char* const row = lds + ld.k + (SL == 1 ? (n & 1) * ld.k_size : 0) + x * ld.k_pitch;
#pragma unroll
    for (int c = 0; c < 4; ++c) {              // lane group c's channels: 4 c + u and 16 + 4 c + u of the step
      const uint32_t both = __builtin_amdgcn_perm(w[2 + (c >> 1)], w[c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
      uint4v out;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        out[u] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, ((both >> (4 * u)) & 0x000f000fu) | k1024) + off);
      const int p = 4 * pc + c;
      *reinterpret_cast<uint4v*>(row + ((p & ~15) | ((p ^ x) & 15)) * 16) = out;
    }
  };

  // ---- prologue: rows of the first four steps
  if (wave < min(4, n_steps)) put_rows(wave, entry_of(wave));
  // queries, rotated to their position and scaled, [wave][row][feature]
  float* const qs = reinterpret_cast<float*>(lds + ld.p) + wave * NQ * kDHead;
  float q_max[NQ], q_sum[NQ];                  // of the folded pairs
  {
    const int pos = max(0, min(a.q_pos ? a.q_pos[seq] : L - 1, a.rope_len - 1));
    const float c = a.rope[rope_f32_index(pos, lane, 0, kRopeTableStride)], s = a.rope[rope_f32_index(pos, lane, 1, kRopeTableStride)];
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const uint16_t* q = a.q + ((size_t)seq * m.n_heads * m.qpk + (h0 + hh) * m.qpk + row0 + min(r, nr - 1)) * kDHead;
      const float x0 = T::to_float(q[lane]), x1 = T::to_float(q[lane + kHalf]);
      const float y0 = (x0 * c - x1 * s) * a.scale, y1 = (x1 * c + x0 * s) * a.scale;
      qs[r * kDHead + lane] = y0;
      qs[r * kDHead + kHalf + lane] = y1;
      const float size = lane >= kPagedQLow ? fabsf(y0) + fabsf(y1) : 0.f;
      q_max[r] = max_of_wave(size);
      q_sum[r] = sum_of_wave(size);
    }
  }
  {                                            // Lagrange polynomials of the span's Chebyshev nodes (barycentric form), per position
    const double T2 = 0.5 * kSteps * a.span_steps, x = (tid - (T2 - 0.5)) / T2;
    // cos((2 i + 1) pi / 16) and the barycentric weights (-1)^i sin((2 i + 1) pi / 16)
    constexpr double kNode[4] = {0.98078528040323044913, 0.83146961230254523708, 0.55557023301960222474, 0.19509032201612826785};
    double w[8], sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double node = i < 4 ? kNode[i] : -kNode[7 - i], weight = (i & 1 ? -1.0 : 1.0) * kNode[i < 4 ? 3 - i : i - 4];
      w[i] = weight / (x - node);
      sum += w[i];
    }
    float* const basis = reinterpret_cast<float*>(lds + ld.basis) + tid * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) basis[i] = (float)(w[i] / sum);
  }
  lds_barrier();
  request_keys(0);
  request_values(0);

  // ---- weights, as operand rows.  W: tile j's row 2 x (+ 1) is feature 4 x + j (+ 64), x < 8; it stays in the accumulation registers, which
  // the matrix instructions read as they are.  Those to be folded: a channel's features 32 + 8 kg .. and 96 + 8 kg .., read for every span.
  uint4v W[KS][4];
  const uint16_t* const BF = B + kPagedQLow + 8 * kg;
  auto fold_weights = [&](int ks, uint4v (&f)[2][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int ch = min(slice * KS * 32 + 32 * ks + 16 * v + col, rk - 1);
      f[v][0] = *reinterpret_cast<const uint4v*>(BF + (size_t)ch * width);
      f[v][1] = *reinterpret_cast<const uint4v*>(BF + (size_t)ch * width + kHalf);
    }
  };
  int shift = 0;                               // they are held times 2^shift
  float b_max = 0.f;                           // of those to be folded
  {
    uint32_t top = 0, top_f = 0;               // the largest, without its sign
    auto larger = [](uint32_t t, uint32_t w) __attribute__((always_inline)) { return max(t, max(w & 0x7fffu, (w >> 16) & 0x7fffu)); };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4v f[2][2];
      fold_weights(ks, f);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint2v x[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const int ch = min(slice * KS * 32 + 32 * ks + 16 * v + 4 * kg + u, rk - 1);
          x[v] = *reinterpret_cast<const uint2v*>(B + (size_t)ch * width + (col & 1) * kHalf + 4 * (col >> 1));
        }
        const uint32_t keep = ks < ks_here ? 0xffffffffu : 0u;           // channels behind the rank: zero
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          W[ks][j][u] = keep & __builtin_amdgcn_perm(x[1][j >> 1], x[0][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
          if (!__is_same(T, F16)) top = larger(top, W[ks][j][u]);
        }
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 2; ++e) top_f = larger(top_f, f[v][e][u]);
      }
      if (__is_same(T, F16))
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+a"(W[ks][j]));
    }
    b_max = max_of_wave(T::to_float((uint16_t)top_f));
    if (!__is_same(T, F16)) {
      const float all = max_of_wave(T::to_float((uint16_t)max(top, top_f)));
      shift = __builtin_amdgcn_readfirstlane(15 - __builtin_amdgcn_frexp_expf(all));
      b_max = __builtin_amdgcn_ldexpf(b_max, shift);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int i = 0; i < 4; ++i) W[ks][j][i] = to_f16<T>(W[ks][j][i], shift);
          asm volatile("" : "+a"(W[ks][j]));
        }
      }
    }
  }

  // ---- angles and queries of this lane.  Rebuilt pairs 8 kg + p at token col of 16; folded pairs 32 + 8 kg + p at node col % 8 of a span.
  float tc[8], ts[8];                          // cos and sin of 16 positions
  float hc[8], hs[8];                          // of col positions; with one query row its a and b there
  float nc[LG][8], ns[LG][8];                  // a and b at the node, times 2^e of its row
  float qa[NQ == 1 ? 1 : NQ][8], qb[NQ == 1 ? 1 : NQ][8];    // several rows: the queries
  float low_unit[NQ];                          // what a folded row's sums are worth
  float g_scale[LG];                           // ... and what its weights are multiplied by, by this lane's row
  {
    const float unit = __builtin_amdgcn_ldexpf(1.f, -shift);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int f = 8 * kg + p, at16 = min(16, a.rope_len - 1), at = min(col, a.rope_len - 1);
      tc[p] = a.rope[rope_f32_index(at16, f, 0, kRopeTableStride)];
      ts[p] = a.rope[rope_f32_index(at16, f, 1, kRopeTableStride)];
      const float c = a.rope[rope_f32_index(at, f, 0, kRopeTableStride)], s = a.rope[rope_f32_index(at, f, 1, kRopeTableStride)];
      if (NQ == 1) {
        const float x = qs[f] * unit, y = qs[kHalf + f] * unit;
        hc[p] = c * x + s * y;
        hs[p] = c * y - s * x;
      } else {
        hc[p] = c;
        hs[p] = s;
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          qa[r][p] = qs[r * kDHead + f] * unit;
          qb[r][p] = qs[r * kDHead + kHalf + f] * unit;
        }
      }
    }
    int ea[NQ], eg[NQ];
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      ea[r] = 8 - __builtin_amdgcn_frexp_expf(q_max[r]);
      eg[r] = 15 - __builtin_amdgcn_frexp_expf(__builtin_amdgcn_ldexpf(1.4143f * b_max * q_sum[r], ea[r]));
      low_unit[r] = __builtin_amdgcn_ldexpf(1.f, -ea[r] - eg[r] - shift);
    }
    const double T2 = 0.5 * kSteps * a.span_steps;
    constexpr float kNode[4] = {0.98078528040323044913f, 0.83146961230254523708f, 0.55557023301960222474f, 0.19509032201612826785f};
    const int node = col & 7;
    const float shape = node == 0 || node == 7 ? kNode[0] : (node == 1 || node == 6 ? kNode[1] : (node == 2 || node == 5 ? kNode[2] : kNode[3]));
    const float at = (float)(T2 - 0.5) + (float)T2 * (node < 4 ? shape : -shape);
    const int upper = NQ == 1 ? 0 : col >> 3;                // which of a group's two rows
#pragma unroll
    for (int l = 0; l < LG; ++l) {
      const float scale = __builtin_amdgcn_ldexpf(1.f, NQ == 1 ? ea[0] : (upper ? ea[(2 * l + 1) % NQ] : ea[2 * l]));
      g_scale[l] = __builtin_amdgcn_ldexpf(1.f, NQ == 1 ? eg[0] : (upper ? eg[(2 * l + 1) % NQ] : eg[2 * l]));
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const int f = kPagedQLow + 8 * kg + p;
        float s, c;
        sincosf(a.w_low[8 * kg + p] * at, &s, &c);
        const float x = qs[(2 * l + upper) * kDHead + f] * scale, y = qs[(2 * l + upper) * kDHead + kHalf + f] * scale;
        nc[l][p] = c * x + s * y;
        ns[l][p] = c * y - s * x;
      }
    }
  }

  // ---- the first step's keys
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_barrier();                               // (with several query rows the queries reach into what follows)
  put_tokens(0);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i * 128 < k_cols) convert(0, i, zraw[i]);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the raw codes have been read)
  if (n_steps > 1) request_keys(1);
  if (3 < n_steps && wave == 3) entry = entry_of(3);         // (its rows are there: the same again)
  lds_barrier();

  float sc[8], ss[8];                          // cos and sin (one query row: a and b) of the next 16 tokens
  uint4v G[KS][NG];
  // Folded weights from step n on
  auto fold = [&](int n) __attribute__((always_inline)) {
    const float* at = anchors + (n & 1) * kDHead;
    auto four = [&](int f) __attribute__((always_inline)) { return *reinterpret_cast<const float4v*>(at + f); };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float4v c = four(8 * kg + 4 * half), s = four(kHalf + 8 * kg + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int p = 4 * half + e;
        if (NQ == 1) {
          sc[p] = __builtin_fmaf(c[e], hc[p], s[e] * hs[p]);
          ss[p] = __builtin_fmaf(c[e], hs[p], -(s[e] * hc[p]));
        } else {
          sc[p] = __builtin_fmaf(c[e], hc[p], -(s[e] * hs[p]));
          ss[p] = __builtin_fmaf(c[e], hs[p], s[e] * hc[p]);
        }
      }
    }
    uint4v va[LG][2], vb[LG][2];               // a and b of the folded pairs at the nodes, hi and lo (one row: by lanes)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float4v c = four(kPagedQLow + 8 * kg + 4 * half), s = four(kHalf + kPagedQLow + 8 * kg + 4 * half);
#pragma unroll
      for (int l = 0; l < LG; ++l)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float x[2], y[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int p = 4 * half + e + i;
            x[i] = __builtin_fmaf(c[e + i], nc[l][p], s[e + i] * ns[l][p]);
            y[i] = __builtin_fmaf(c[e + i], ns[l][p], -(s[e + i] * nc[l][p]));
          }
          uint32_t h, lo;
          split2<F16>(x[0], x[1], &h, &lo);
          va[l][0][2 * half + e / 2] = NQ == 1 && col >= 8 ? lo : h;
          va[l][1][2 * half + e / 2] = lo;
          split2<F16>(y[0], y[1], &h, &lo);
          vb[l][0][2 * half + e / 2] = NQ == 1 && col >= 8 ? lo : h;
          vb[l][1][2 * half + e / 2] = lo;
        }
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (SL == 2 && ks >= ks_here) {          // channels behind the rank
#pragma unroll
        for (int l = 0; l < NG; ++l) G[ks][l] = uint4v{0, 0, 0, 0};
        continue;
      }
      uint4v F[2][2];
      fold_weights(ks, F);
      if (!__is_same(T, F16))
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int e = 0; e < 2; ++e) F[v][e][i] = to_f16<T>(F[v][e][i], shift);
#pragma unroll
      for (int l = 0; l < LG; ++l) {
        float4v d[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          d[v] = mma<F16>(F[v][0], va[l][0], float4v{0, 0, 0, 0});
          d[v] = mma<F16>(F[v][1], vb[l][0], d[v]);
          if (NQ > 1) {
            d[v] = mma<F16>(F[v][0], va[l][1], d[v]);
            d[v] = mma<F16>(F[v][1], vb[l][1], d[v]);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float x = d[0][u], y = d[1][u];
          if (NQ == 1) {
            x = add_8_on(x);
            y = add_8_on(y);
          }
          uint32_t h, lo;
          split2<F16>(x * g_scale[l], y * g_scale[l], &h, &lo);
          if (NQ == 1) {
            G[ks][0][u] = col >= 8 ? lo : h;
          } else {
            G[ks][2 * l][u] = h;
            G[ks][(2 * l + 1) % NG][u] = lo;
          }
        }
      }
    }
  };

  // ---- keys of sub-tile `sub` of step n: every query row's partial score of token col, by lane group
  const int k_at = (SL == 1 ? hg * KS * 64 : slice * 512) + col * ld.k_pitch;
  int k_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_off[i] = k_at + (((4 * i + kg) ^ col) & 15) * 16;
  const int b_last = ks_here / 4 - 1;          // last block of this slice
  auto keys = [&](int n, int sub, float (&part)[NQ]) __attribute__((always_inline)) {
    const unsigned char* const k = lds + ld.k + (SL == 1 ? (n & 1) * ld.k_size : 0) + 16 * sub * ld.k_pitch;
    float4v acc[4], low[LG];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = float4v{0, 0, 0, 0};
#pragma unroll
    for (int l = 0; l < LG; ++l) low[l] = float4v{0, 0, 0, 0};
    auto product = [&](int ks, uint4v h) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = mma<F16>(W[ks][j], h, acc[j]);
#pragma unroll
      for (int l = 0; l < NG; ++l) low[NQ == 1 ? 0 : l / 2] = mma<F16>(G[ks][l], h, low[NQ == 1 ? 0 : l / 2]);
    };
    const float2 tok = k_tok[((n & 1) * 2 + (SL == 1 ? hg : slice)) * kSteps + 16 * sub + col];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) product(4 * b + i, *reinterpret_cast<const uint4v*>(k + k_off[i] + (SL == 1 ? b : min(b, b_last)) * 256));
      if (flags[n & 1]) {                      // zero-points that are no small integers: as operands of their own, the same for all channels
        const int block = SL == 1 ? hg * NB + b : min(2 * slice + b, k_cols / 128 - 1);
        const float left = k_left[((n & 1) * 4 + block) * kSteps + 16 * sub + col];
        const uint32_t w = pack2<F16>(-left, -left);
#pragma unroll
        for (int i = 0; i < 4; ++i) product(4 * b + i, uint4v{w, w, w, w});
      }
      if (b + 1 < NB) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] *= tok.x;
#pragma unroll
        for (int l = 0; l < LG; ++l) low[l] *= tok.x;
      }
    }
    const int t = pos_of(n) + 16 * sub + col;
    const int first = n < steps_s ? kPagedTile * i0 : pos_w;
    const float4v basis = *reinterpret_cast<const float4v*>(lds + ld.basis + (((t - first) & (kSteps * a.span_steps - 1)) * 8 + 4 * (kg & 1)) * 4);
#pragma unroll
    for (int r = 0; r < NQ; ++r) part[r] = 0.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const float lo = acc[p & 3][2 * (p >> 2)], hi = acc[p & 3][2 * (p >> 2) + 1], c = sc[p], s = ss[p];
      if (NQ == 1) {
        part[0] = __builtin_fmaf(lo, c, part[0]);
        part[0] = __builtin_fmaf(hi, s, part[0]);
        sc[p] = __builtin_fmaf(c, tc[p], s * ts[p]);         // a and b, 16 positions on
        ss[p] = __builtin_fmaf(s, tc[p], -(c * ts[p]));
      } else {
        const float x = __builtin_fmaf(lo, c, -(hi * s)), y = __builtin_fmaf(hi, c, lo * s);
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          part[r] = __builtin_fmaf(x, qa[r][p], part[r]);
          part[r] = __builtin_fmaf(y, qb[r][p], part[r]);
        }
        sc[p] = __builtin_fmaf(c, tc[p], -(s * ts[p]));
        ss[p] = __builtin_fmaf(s, tc[p], c * ts[p]);
      }
    }
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const float4v x = low[NQ == 1 ? 0 : r / 2];
      const float sum = __builtin_fmaf(x[0], basis[0], __builtin_fmaf(x[1], basis[1], __builtin_fmaf(x[2], basis[2], x[3] * basis[3])));
      const bool mine = NQ == 1 || (kg >> 1) == (r & 1);
      part[r] = mine ? __builtin_fmaf(sum, low_unit[r], part[r]) : part[r];
      part[r] *= tok.y;
    }
  };

  // ---- softmax of step n, a token per lane
  float run_max[NQ], run_sum[NQ], blk_max[NQ][MAXCB], z_sum[NQ][MAXCB];
#pragma unroll
  for (int r = 0; r < NQ; ++r) {
    run_max[r] = -INFINITY;
    run_sum[r] = 0.f;
#pragma unroll
    for (int b = 0; b < MAXCB; ++b) {
      blk_max[r][b] = -INFINITY;
      z_sum[r][b] = 0.f;
    }
  }
  float* const scores = reinterpret_cast<float*>(lds + ld.scores);
  auto softmax = [&](int n, const float (&x_in)[NQ]) __attribute__((always_inline)) {
    const bool seen = attended(n, pos_of(n) + lane);
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const float x = seen ? x_in[r] : -INFINITY;
      const float now = fmaxf(run_max[r], max_of_wave(x)), zero = now == -INFINITY ? 0.f : now;
      run_sum[r] = run_sum[r] * __builtin_amdgcn_exp2f(run_max[r] - zero) + __builtin_amdgcn_exp2f(x - zero);
      run_max[r] = now;
      const int row = hw * NQ + r;
#pragma unroll
      for (int b = 0; b < MAXCB; ++b) {
        if (b >= CB) break;
        const float2 tok = v_tok[((n & 1) * CB + b) * kSteps + lane];
        const float u = x + (float)__builtin_amdgcn_frexp_expf(tok.x);
        const float top = fmaxf(blk_max[r][b], max_of_wave(u)), base = top == -INFINITY ? 0.f : top;
        const float alpha = __builtin_amdgcn_exp2f(blk_max[r][b] - base);
        const float w = seen ? __builtin_amdgcn_frexp_mantf(tok.x) * __builtin_amdgcn_exp2f(u - base) : 0.f;
        blk_max[r][b] = top;
        z_sum[r][b] = z_sum[r][b] * alpha + (seen ? w * (tok.y - 8.f) : 0.f);
        uint32_t hi, lo;
        split2<F16>(w * kWeightScale, 0.f, &hi, &lo);
        uint16_t* P = reinterpret_cast<uint16_t*>(lds + ld.p + (n & 1) * ld.p_size + b * ld.p_cb + row * kPagedQProbPitch) + lane;
        P[0] = (uint16_t)hi;
        P[kLoRows * (kPagedQProbPitch / 2)] = (uint16_t)lo;
        if (lane == 0) reinterpret_cast<float*>(lds + ld.alpha)[((n & 1) * CB + b) * 16 + row] = alpha;
      }
    }
  };

  // ---- values of step n.  A wavefront has a block of 128 columns, and half of the tokens where there are one or two blocks.
  float4v O[8];                                // column 8 col + u of rows 4 kg + e; odd columns in units of 2^-20, even ones of 2^-24
#pragma unroll
  for (int u = 0; u < 8; ++u) O[u] = float4v{0, 0, 0, 0};
  const int vb = CB <= 2 ? wave % CB : wave;
  const int half0 = CB <= 2 ? wave / CB : 0, half1 = CB <= 2 ? min(half0 + 1, 2) : 2;
  const bool has_values = CB <= 2 ? half0 < 2 : wave < CB;
  // Codes enter as code - 8: most zero-points are near 8, and sums of codes and of zero-points, which all but cancel over many tokens, would leave their
  // rounding (4e-5 of the largest output at 3000 tokens, against 4e-6).
  const half2v minus8_even = __builtin_bit_cast(half2v, 0x80088008u), minus8_odd = __builtin_bit_cast(half2v, 0x80808080u);
  auto values = [&](int n) __attribute__((always_inline)) {
    if (!has_values) return;
    const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (((n & 1) * CB + vb) * 16 + (NQ == 1 ? 0 : 4 * kg)) * 4);
    if (__any(!(al[0] == 1.f && al[1] == 1.f && al[2] == 1.f && al[3] == 1.f)))
#pragma unroll
      for (int u = 0; u < 8; ++u) O[u] *= al;
    for (int half = half0; half < half1; ++half) {
      uint32_t d[8];
      const unsigned char* const v = lds + ld.v + (n % VBUFS) * ld.v_size + (32 * half + 8 * kg) * (v_cols / 2) + vb * 64 + col * 4;
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = *reinterpret_cast<const uint32_t*>(v + e * (v_cols / 2));
      const unsigned char* const P = lds + ld.p + (n & 1) * ld.p_size + vb * ld.p_cb + (NQ == 1 || SL == 2 ? col & 7 : col) * kPagedQProbPitch + (32 * half + 8 * kg) * 2;
      const uint4v hi = *reinterpret_cast<const uint4v*>(P);
      uint4v lo = hi;
      if (NQ > 1) lo = *reinterpret_cast<const uint4v*>(P + kLoRows * kPagedQProbPitch);
#pragma unroll
      for (int j = 0; j < 4; ++j) {            // byte j: channels 2 j and 2 j + 1
        uint4v even, odd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = __builtin_amdgcn_perm(d[2 * i + 1], d[2 * i], 0x0c040c00u + 0x00010001u * j);
          even[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, x & 0x000f000fu) + minus8_even);
          odd[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, x & 0x00f000f0u) + minus8_odd);
        }
        O[2 * j] = mma<F16>(hi, even, O[2 * j]);
        O[2 * j + 1] = mma<F16>(hi, odd, O[2 * j + 1]);
        if (NQ > 1) {
          O[2 * j] = mma<F16>(lo, even, O[2 * j]);
          O[2 * j + 1] = mma<F16>(lo, odd, O[2 * j + 1]);
        }
      }
    }
  };

  for (int n = 0; n <= n_steps; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what interval n - 1 requested
    uint16_t z_now[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z_now[i] = zraw[i];
    if (n + 1 < n_steps) put_tokens(n + 1);
    if (wave == 3 && n + 3 < n_steps) put_rows(n + 3, entry);
    if (SL == 1 && n + 2 < n_steps) request_keys(n + 2);
    if (SL == 1 && n + 1 < n_steps) request_values(n + 1);
    if (wave == 3 && n + 4 < n_steps) entry = entry_of(n + 4);
    if (n > 0) values(n - 1);
    if (n == n_steps) break;
    if (folds(n)) fold(n);
    float part[4][NQ], x[NQ];
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
      keys(n, sub, part[sub]);
      if (SL == 1 && sub < 4 && n + 1 < n_steps && sub * 128 < k_cols) convert(n + 1, sub, z_now[sub]);
    }
#pragma unroll
    for (int r = 0; r < NQ; ++r) x[r] = add_swapped16(add_swapped32(part[0][r], part[2][r]), add_swapped32(part[1][r], part[3][r]));
    if (SL == 2) {
      if (slice == 1)
#pragma unroll
        for (int r = 0; r < NQ; ++r) scores[(hw * NQ + r) * kSteps + lane] = x[r];
      lds_barrier();
      if (n + 1 < n_steps) request_values(n + 1);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + 1 < n_steps && i * 128 < k_cols) convert(n + 1, i, z_now[i]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the raw codes have been read)
      if (n + 2 < n_steps) request_keys(n + 2);
#pragma unroll
      for (int r = 0; r < NQ; ++r) x[r] += scores[(hw * NQ + r) * kSteps + lane];
    }
    if (slice == 0) softmax(n, x);
    lds_barrier();
  }

  // ---- partial results
  lds_barrier();
  float* const halves = reinterpret_cast<float*>(lds + ld.k);              // O of the second halves of the tokens
  float2* const fin = reinterpret_cast<float2*>(lds + ld.p);               // [16 rows][4 blocks]: what the zero-points take off, what a sum is worth
  const size_t slot = (size_t)seq * a.n_slots + chunk;
  if (has_values && half0 == 1)
#pragma unroll
    for (int u = 0; u < 8; ++u) *reinterpret_cast<float4v*>(halves + ((vb * 8 + u) * 64 + lane) * 4) = O[u];
  if (slice == 0)
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const float sum = sum_of_wave(run_sum[r]);
#pragma unroll
      for (int b = 0; b < MAXCB; ++b) {
        if (b >= CB) break;
        const float z = sum_of_wave(z_sum[r][b]);
        if (lane == 0) fin[(hw * NQ + r) * MAXCB + b] = make_float2(z, run_max[r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(blk_max[r][b] - run_max[r]));
      }
      if (lane == 0 && hw < nh && r < nr)
        reinterpret_cast<float2*>(a.ml_part)[(slot * m.n_heads + h0 + hw) * m.qpk + row0 + r] = make_float2(run_max[r], sum);
    }
  lds_barrier();
  if (has_values && half0 == 0) {
    if (CB <= 2)
#pragma unroll
      for (int u = 0; u < 8; ++u) O[u] += *reinterpret_cast<const float4v*>(halves + ((vb * 8 + u) * 64 + lane) * 4);
    const int vg = 128 * vb / rv;              // the columns' group in the unit
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        y[u] = O[u][e];
        if (NQ == 1) y[u] += __shfl_xor(y[u], 16);
      }
      const int row = NQ == 1 ? e : 4 * kg + e, h = row / NQ, r = row % NQ;
      if (h >= nh || h >= HEADS || r >= nr || (NQ == 1 && kg != 0) || (un.n_groups() > 1 && h / per_group != vg)) continue;
      const float2 f = fin[row * MAXCB + vb];
#pragma unroll
      for (int u = 0; u < 8; ++u) y[u] = (y[u] * ((u & 1 ? 1048576.f : 16777216.f) / kWeightScale) - f.x) * f.y;
      const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
      float* const o = a.o_part + slot * a.o_stride + (size_t)m.qpk * ohead + (size_t)(row0 + r) * rv + 128 * vb - vg * rv + 8 * col;
      *reinterpret_cast<float4v*>(o) = float4v{y[0], y[1], y[2], y[3]};
      *reinterpret_cast<float4v*>(o + 4) = float4v{y[4], y[5], y[6], y[7]};
    }
  }
}

namespace {
template <typename T, int KS, int SL> PagedQFn pick(int rows) {
  return rows == 1 ? pagedq_kernel<T, KS, SL, 1> : (rows == 2 ? pagedq_kernel<T, KS, SL, 2> : pagedq_kernel<T, KS, SL, 4>);
}
template <typename T> PagedQFn pick(const PagedQForm& f) {
  return f.slices == 2 ? pick<T, 8, 2>(f.rows) : (f.ks == 4 ? pick<T, 4, 1>(f.rows) : pick<T, 8, 1>(f.rows));
}
}  // namespace

PagedQFn pagedq_form(int act, const PagedQForm& f) { return act == PALU_F16 ? pick<F16>(f) : pick<BF16>(f); }

}  // namespace palu
