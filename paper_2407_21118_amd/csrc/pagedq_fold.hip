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
constexpr float kSlack = 4.f;                  // a running maximum rises when a score exceeds it by so much (base-2 logarithms)
constexpr float kWeightScale = 2048.f;         // of the values' weights, up to 2^4, in float16 pairs: those of the others are right to 2^-36 of the largest

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

// KS steps of 32 key channels per wavefront; SL wavefronts share a head's channels; NQ query rows of a head; PIPED: see the loop, for units of KB and
// VB blocks of key and value columns
template <typename T, int KS, int SL, int NQ, bool PIPED, int KB = 0, int VB = 0>
__global__ __launch_bounds__(kPagedQThreads, 1) void pagedq_kernel(PagedQArgs a) {
  constexpr int HEADS = 4 / SL;                // of a unit
  constexpr int NB = KS / 4;                   // blocks of 128 channels
  constexpr int LG = NQ == 1 ? 1 : NQ / 2;     // folded query rows, 16 (row, node) a group
  constexpr int NG = NQ == 1 ? 1 : NQ;         // tiles of folded weights: of one row hi and lo in one tile, else apart
  constexpr int MAXCB = PIPED ? VB : 4;
  constexpr PagedQLds ld = pagedq_lds(KS, SL, NQ, KB, VB, PIPED);
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
  const int k_cols = PIPED ? 128 * KB : un.n_groups() * rk, v_cols = PIPED ? 128 * VB : un.n_groups() * rv, CB = v_cols / 128;
  const int row0 = rb * NQ, nr = min(NQ, m.qpk - row0);      // query rows of a head
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
  // spans: the first steps of either part, and every span_steps-th
  const int span_log = __builtin_ctz(a.span_steps), spans_s = (steps_s + a.span_steps - 1) >> span_log;
  auto folds = [&](int n) __attribute__((always_inline)) { return ((n < steps_s ? n : n - steps_s) & (a.span_steps - 1)) == 0; };
  auto span_of = [&](int n) __attribute__((always_inline)) { return n < steps_s ? n >> span_log : spans_s + ((n - steps_s) >> span_log); };
  auto span_step = [&](int k) __attribute__((always_inline)) { return k < spans_s ? k << span_log : steps_s + ((k - spans_s) << span_log); };

  // ---- requests.  In interval n: scales and zero-points of step n + 3, keys of n + 2, values (PIPED: of n, else n + 1), page-table entries of n + 5,
  // the angles of the third span after one that begins.
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  const int k_pieces = k_cols / 32, v_pieces = v_cols / 32;  // 16-byte pieces of a raw row
  const int k_block0 = m.k_off[g] / 128, v_block0 = m.v_off[g] / 128;
  uint16_t tok_raw[8];
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
    rows[(n & 7) * kSteps + lane] = (max(0, min(e, a.n_pages - 1)) << a.page_shift) + (token_of(n, lane) & ((1 << a.page_shift) - 1));
  };
  const unsigned char* const k_src = a.k.codes + m.k_off[g] / 2 + (tid % k_pieces) * 16;
  const int k_x = tid / k_pieces;              // (PIPED: row of the first piece; the second lies 32 on)
  auto request_keys = [&](int n) __attribute__((always_inline)) {
    const int* const r = rows + (n & 7) * kSteps;
    const uint32_t dst = lds0 + ld.raw + (PIPED ? (n & 1) * ld.raw_size : 0) + wave * 1024;
    if (PIPED) {
      const uint32_t r0 = r[k_x], r1 = r[(k_x + 32) & 63];
      load_to_lds(k_src + (uint64_t)r0 * (uint32_t)a.k.row_bytes, dst);
      if (k_cols > 128) load_to_lds(k_src + (uint64_t)r1 * (uint32_t)a.k.row_bytes, dst + kPagedQThreads * 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i * 128 >= k_cols) break;
        const int id = i * kPagedQThreads + tid, x = id / k_pieces, pc = id - x * k_pieces;
        load_to_lds(a.k.codes + (size_t)r[x] * a.k.row_bytes + m.k_off[g] / 2 + pc * 16, dst + i * kPagedQThreads * 16);
      }
    }
  };
  // role 0: keys', 1: values'; an even and an odd wavefront's, which keeps to its role
  const PagedQSide& tok_side = wave & 1 ? a.v : a.k;
  const uint16_t* const tok_scale = tok_side.scale + (wave & 1 ? v_block0 : k_block0);
  const uint16_t* const tok_zero = tok_side.zero + (wave & 1 ? v_block0 : k_block0);
  const uint32_t tok_blocks = tok_side.n_blocks;
  auto request_tokens = [&](int n, int role) __attribute__((always_inline)) {
    const int blocks = role == 0 ? k_cols / 128 : CB;
    const uint64_t at = (uint64_t)(uint32_t)rows[(n & 7) * kSteps + lane] * tok_blocks;
    const uint16_t *scale = tok_scale + at, *zero = tok_zero + at;
    tok_raw[0] = scale[0];
    tok_raw[4] = zero[0];
    if (blocks > 1) {
      tok_raw[1] = scale[1];
      tok_raw[5] = zero[1];
    }
    if (blocks > 2) {
#pragma unroll
      for (int b = 2; b < 4; ++b) {
        tok_raw[b] = scale[min(b, blocks - 1)];
        tok_raw[4 + b] = zero[min(b, blocks - 1)];
      }
    }
  };
  auto request_anchors = [&](int k) __attribute__((always_inline)) {
    anchor_c = a.rope[rope_f32_index(pos_of(span_step(k)), lane, 0, kRopeTableStride)];
    anchor_s = a.rope[rope_f32_index(pos_of(span_step(k)), lane, 1, kRopeTableStride)];
  };
  constexpr int VBUFS = PIPED ? 3 : 2;
  int v_at[4];                                 // pieces of the values: column << 8 | row
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int id = i * kPagedQThreads + tid, x = (id / v_pieces) & 63;
    v_at[i] = (id % v_pieces) << 12 | x;
  }
  const unsigned char* const v_src = a.v.codes + m.v_off[g] / 2;
  auto request_values = [&](int n) __attribute__((always_inline)) {
    const int* const r = rows + (n & 7) * kSteps;
    const uint32_t dst = lds0 + ld.v + (n % VBUFS) * ld.v_size + wave * 1024;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i * 128 >= v_cols) break;
      load_to_lds(v_src + ((uint64_t)(uint32_t)r[v_at[i] & 63] * (uint32_t)a.v.row_bytes + (v_at[i] >> 8)), dst + i * kPagedQThreads * 16);
    }
  };
  // ---- what came of them
  float2* const k_tok = reinterpret_cast<float2*>(lds + ld.k_tok);
  uint32_t* const k_zero = reinterpret_cast<uint32_t*>(lds + ld.k_zero);
  uint32_t* const v_tok = reinterpret_cast<uint32_t*>(lds + ld.v_tok);
  float* const anchors = reinterpret_cast<float*>(lds + ld.anchors);
  int* const flags = reinterpret_cast<int*>(lds + ld.flags);
  auto put_tokens = [&](int n, int role) __attribute__((always_inline)) {
    if (role == 0) {
      bool any = false;
#pragma unroll
      for (int b = 0; b < 4; ++b) {            // codes take their zero-point where it is a small integer; what is left of it (with the other sign): see zero_points
        if (b * 128 >= k_cols) break;
        const float z = F16::to_float(tok_raw[4 + b]);
        const bool small = small_integer(z);
        any = any || !small;
        k_zero[((n & 3) * 4 + b) * kSteps + lane] = (uint32_t)F16::from_float(-1024.f - (small ? z : 0.f)) | (small ? 0u : (uint32_t)(tok_raw[4 + b] ^ 0x8000u) << 16);
      }
      const int some = __any(any) ? 1 : 0;
      if (lane == 0) flags[n & 3] = some;
#pragma unroll
      for (int s = 0; s < 2; ++s) {            // blocks of a slice, or of a group: (first * ratio + second) * scale.  (A second scale of zero: so
        if (s * NB * 128 >= k_cols) break;     // small a number that nothing of the second block is left.)
        const float s0 = F16::to_float(tok_raw[NB * s]);
        float s1 = s0, ratio = 1.f;
        if (NB == 2 && (2 * s + 1) * 128 < k_cols) {
          s1 = F16::to_float(tok_raw[2 * s + 1]);
          if (s1 == 0.f) s1 = 0x1p-60f;
          ratio = s0 * __builtin_amdgcn_rcpf(s1);            // (right to 2^-22)
        }
        k_tok[((n & 3) * 2 + s) * kSteps + lane] = make_float2(ratio, s1);
      }
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b >= CB) break;
        v_tok[((n & 3) * CB + b) * kSteps + lane] = (uint32_t)tok_raw[b] | (uint32_t)tok_raw[4 + b] << 16;
      }
    }
  };
  auto put_anchors = [&](int k) __attribute__((always_inline)) {
    anchors[(k & 3) * kDHead + lane] = anchor_c;
    anchors[(k & 3) * kDHead + kHalf + lane] = anchor_s;
  };
  const uint32_t k1024 = per_lane_constant(0x64006400u);
  // piece i of this thread: its codes; what is added to 1024 + code; quarter c of it, lane group c's channels, 4 c + u and 16 + 4 c + u of the step
  auto zero_of = [&](int n, int x, int pc) __attribute__((always_inline)) {
    const uint32_t z = k_zero[((n & 3) * 4 + (pc >> 2)) * kSteps + x];
    return __builtin_bit_cast(half2v, __builtin_amdgcn_perm(z, z, 0x01000100u));
  };
  auto raw_codes = [&](int n, int i) __attribute__((always_inline)) {
    return *reinterpret_cast<const uint4v*>(lds + ld.raw + (PIPED ? (n & 1) * ld.raw_size : 0) + (i * kPagedQThreads + tid) * 16);
  };
  auto quarter_codes = [&](uint4v w, int c) __attribute__((always_inline)) {
    return __builtin_amdgcn_perm(w[2 + (c >> 1)], w[c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
  };
  auto spread = [&](uint32_t both, half2v off, int u) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, ((both >> (4 * u)) & 0x000f000fu) | k1024) + off);
  };
  auto quarter = [&](uint4v w, half2v off, int c, unsigned char* to) __attribute__((always_inline)) {
    const uint32_t both = quarter_codes(w, c);
    uint4v out;
#pragma unroll
    for (int u = 0; u < 4; ++u) out[u] = spread(both, off, u);
    *reinterpret_cast<uint4v*>(to) = out;
  };
  auto convert = [&](int n, int i) __attribute__((always_inline)) {
    const int id = i * kPagedQThreads + tid, x = id / k_pieces, pc = id - x * k_pieces;
    const uint4v w = raw_codes(n, i);
    const half2v off = zero_of(n, x, pc);
    unsigned char* const row = lds + ld.k + (PIPED ? (n & 1) * ld.k_size : 0) + x * ld.k_pitch;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int p = 4 * pc + c;
      quarter(w, off, c, row + ((p & ~15) | ((p ^ x) & 15)) * 16);
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
  if (!PIPED) request_values(0);
  const int token_step = min(wave >> 1, n_steps - 1);        // waves 0 and 1: of the first step, 2 and 3: of the second
  request_tokens(token_step, wave & 1);
  if (wave < 3 && span_step(wave) < n_steps) request_anchors(wave);

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
    int ea[NQ];
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      // a folded weight is at most b_max * sqrt(2) * q_sum, an a or b at most q_max: both times 2^e are float16 numbers
      ea[r] = min(15 - __builtin_amdgcn_frexp_expf(1.4143f * b_max * q_sum[r]), 15 - __builtin_amdgcn_frexp_expf(q_max[r]));
      low_unit[r] = __builtin_amdgcn_ldexpf(1.f, -ea[r] - shift);
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
  if (PIPED) {                                 // the weights of values before the first step
    for (int x = tid; x < 2 * ld.p_size / 16; x += kPagedQThreads) *reinterpret_cast<uint4v*>(lds + ld.p + x * 16) = uint4v{0, 0, 0, 0};
    for (int x = tid; x < 2 * CB * 16; x += kPagedQThreads) reinterpret_cast<float*>(lds + ld.alpha)[x] = 1.f;
  }
  put_tokens(token_step, wave & 1);
  if (wave < 3 && span_step(wave) < n_steps) put_anchors(wave);
  lds_barrier();
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i * 128 < k_cols) convert(0, i);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // (the raw codes have been read)
  if (n_steps > 1) request_keys(1);
  if (n_steps > 2 && wave < 2) request_tokens(2, wave);
  if (4 < n_steps && wave == 3) entry = entry_of(4);
  lds_barrier();

  // What interval n - 1 requested goes to LDS, before anything is requested: the compiler waits for all loads that it does not know of, too
  auto put = [&](int n) __attribute__((always_inline)) {
    if (wave < 2) {
      if (n + 2 < n_steps) put_tokens(n + 2, wave);
    } else if (wave == 2) {
      if (n > 0 && folds(n - 1) && span_step(span_of(n - 1) + 3) < n_steps) put_anchors(span_of(n - 1) + 3);
    } else {
      if (n + 4 < n_steps) put_rows(n + 4, entry);
    }
  };
  auto request = [&](int n) __attribute__((always_inline)) {
    if (wave < 2) {
      if (n + 3 < n_steps) request_tokens(n + 3, wave);
    } else if (wave == 2) {
      if (folds(n) && span_step(span_of(n) + 3) < n_steps) request_anchors(span_of(n) + 3);
    } else {
      if (n + 5 < n_steps) entry = entry_of(n + 5);
    }
  };
  float sc[8] = {}, ss[8] = {};                // cos and sin (one query row: a and b) of the next 16 tokens
  uint4v G[KS][NG];
  // angles of the first 16 tokens of step n
  auto start = [&](int n) __attribute__((always_inline)) {
    const float* at = anchors + (span_of(n) & 3) * kDHead + 8 * kg;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float4v c = *reinterpret_cast<const float4v*>(at + 4 * half), s = *reinterpret_cast<const float4v*>(at + kHalf + 4 * half);
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
  };
  // a and b of the folded pairs at the nodes of span k, hi and lo (one row: by lanes)
  struct Nodes {
    uint4v a[LG][NQ == 1 ? 1 : 2], b[LG][NQ == 1 ? 1 : 2];
  };
  auto nodes_of = [&](int k, Nodes& v) __attribute__((always_inline)) {
    const float* at = anchors + (k & 3) * kDHead + kPagedQLow + 8 * kg;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float4v c = *reinterpret_cast<const float4v*>(at + 4 * half), s = *reinterpret_cast<const float4v*>(at + kHalf + 4 * half);
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
          v.a[l][0][2 * half + e / 2] = NQ == 1 && col >= 8 ? lo : h;
          if (NQ > 1) v.a[l][NQ > 1][2 * half + e / 2] = lo;
          split2<F16>(y[0], y[1], &h, &lo);
          v.b[l][0][2 * half + e / 2] = NQ == 1 && col >= 8 ? lo : h;
          if (NQ > 1) v.b[l][NQ > 1][2 * half + e / 2] = lo;
        }
    }
  };
  // Folded weights of channel step ks, from its weights f
  const float lo_part = NQ == 1 && col >= 8 ? -1.f : 0.f;    // one row: these lanes hold what the rounding leaves
  auto fold_tile = [&](const uint4v (&f)[2], const Nodes& v, int l) __attribute__((always_inline)) {
    float4v d = mma<F16>(f[0], v.a[l][0], float4v{0, 0, 0, 0});
    d = mma<F16>(f[1], v.b[l][0], d);
    if (NQ > 1) {
      d = mma<F16>(f[0], v.a[l][NQ > 1], d);
      d = mma<F16>(f[1], v.b[l][NQ > 1], d);
    }
    return d;
  };
  auto fold_pack = [&](float x, float y, uint32_t* hi, uint32_t* lo) __attribute__((always_inline)) {
    if (NQ == 1) {
      x = add_8_on(x);
      y = add_8_on(y);
      uint32_t h = pack2<F16>(x, y);
      asm("" : "+v"(h));
      *hi = pack2<F16>(less<F16>(x, h, lo_part), less<F16>(y, h >> 16, lo_part));
    } else {
      split2<F16>(x, y, hi, lo);
    }
  };
  auto prepare_weights = [&](uint4v (&f)[2][2]) __attribute__((always_inline)) {
    if (!__is_same(T, F16))
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 2; ++e) f[v][e][i] = to_f16<T>(f[v][e][i], shift);
  };
  auto fold = [&](int n) __attribute__((always_inline)) {
    Nodes v;
    nodes_of(span_of(n), v);
    uint4v f[2][2][2];
    fold_weights(0, f[0]);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 1 < KS && (SL == 1 || ks + 1 < ks_here)) fold_weights(ks + 1, f[(ks + 1) & 1]);
      if (SL == 2 && ks >= ks_here) {          // channels behind the rank
#pragma unroll
        for (int l = 0; l < NG; ++l) G[ks][l] = uint4v{0, 0, 0, 0};
        continue;
      }
      prepare_weights(f[ks & 1]);
#pragma unroll
      for (int l = 0; l < LG; ++l) {
        const float4v d0 = fold_tile(f[ks & 1][0], v, l), d1 = fold_tile(f[ks & 1][1], v, l);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          uint32_t hi, lo = 0;
          fold_pack(d0[u], d1[u], &hi, &lo);
          G[ks][NQ == 1 ? 0 : 2 * l][u] = hi;
          if (NQ > 1) G[ks][(2 * l + 1) % NG][u] = lo;
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
  struct Sums {
    float4v acc[4], low[LG];
  };
  auto clear = [&](Sums& a) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a.acc[j] = float4v{0, 0, 0, 0};
#pragma unroll
    for (int l = 0; l < LG; ++l) a.low[l] = float4v{0, 0, 0, 0};
  };
  auto product = [&](Sums& a, int ks, uint4v h) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a.acc[j] = mma<F16>(W[ks][j], h, a.acc[j]);
#pragma unroll
    for (int l = 0; l < NG; ++l) a.low[NQ == 1 ? 0 : l / 2] = mma<F16>(G[ks][l], h, a.low[NQ == 1 ? 0 : l / 2]);
  };
  auto scale_sums = [&](Sums& a, float x) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a.acc[j] *= x;
#pragma unroll
    for (int l = 0; l < LG; ++l) a.low[l] *= x;
  };
  auto tok_of = [&](int n, int sub) __attribute__((always_inline)) {
    return k_tok[((n & 3) * 2 + (SL == 1 ? hg : slice)) * kSteps + 16 * sub + col];
  };
  auto operand = [&](int n, int sub, int ks) __attribute__((always_inline)) {
    const unsigned char* const k = lds + ld.k + (PIPED ? (n & 1) * ld.k_size : 0) + 16 * sub * ld.k_pitch;
    return *reinterpret_cast<const uint4v*>(k + k_off[ks & 3] + (SL == 1 ? ks >> 2 : min(ks >> 2, b_last)) * 256);
  };
  // zero-points that are no small integers: as operands of their own, the same for all channels of block b, times x
  auto zero_points = [&](Sums& a, int n, int sub, int b, float x) __attribute__((always_inline)) {
    const int block = SL == 1 ? hg * NB + b : min(2 * slice + b, k_cols / 128 - 1);
    const uint32_t z = k_zero[((n & 3) * 4 + block) * kSteps + 16 * sub + col], w = __builtin_amdgcn_perm(z, z, 0x03020302u);
    Sums more;
    clear(more);
#pragma unroll
    for (int i = 0; i < 4; ++i) product(more, 4 * b + i, uint4v{w, w, w, w});
#pragma unroll
    for (int j = 0; j < 4; ++j) a.acc[j] += more.acc[j] * x;
#pragma unroll
    for (int l = 0; l < LG; ++l) a.low[l] += more.low[l] * x;
  };
  // What pair p of this lane adds to the scores; its angle (one query row: a and b) 16 tokens on.  (The empty statements keep both where they are.)
  auto pair_adds = [&](const Sums& a, int p, float (&part)[NQ]) __attribute__((always_inline)) {
    const float lo = a.acc[p & 3][2 * (p >> 2)], hi = a.acc[p & 3][2 * (p >> 2) + 1], c = sc[p], s = ss[p];
    if (NQ == 1) {
      part[0] = __builtin_fmaf(lo, c, part[0]);
      part[0] = __builtin_fmaf(hi, s, part[0]);
      asm volatile("" : "+v"(part[0]));
    } else {
      const float x = __builtin_fmaf(lo, c, -(hi * s)), y = __builtin_fmaf(hi, c, lo * s);
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        part[r] = __builtin_fmaf(x, qa[r][p], part[r]);
        part[r] = __builtin_fmaf(y, qb[r][p], part[r]);
        asm volatile("" : "+v"(part[r]));
      }
    }
  };
  auto pair_turns = [&](int p) __attribute__((always_inline)) {
    const float c = sc[p], s = ss[p];
    if (NQ == 1) {
      sc[p] = __builtin_fmaf(c, tc[p], s * ts[p]);
      ss[p] = __builtin_fmaf(s, tc[p], -(c * ts[p]));
    } else {
      sc[p] = __builtin_fmaf(c, tc[p], -(s * ts[p]));
      ss[p] = __builtin_fmaf(s, tc[p], c * ts[p]);
    }
    asm volatile("" : "+v"(sc[p]), "+v"(ss[p]));
  };
  auto pair = [&](const Sums& a, int p, float (&part)[NQ]) __attribute__((always_inline)) {
    pair_adds(a, p, part);
    pair_turns(p);
  };
  const int my_basis = ld.basis + (col * 8 + 4 * (kg & 1)) * 4;
  auto basis_of = [&](int n, int sub) __attribute__((always_inline)) {
    const int step = (n < steps_s ? n : n - steps_s) & (a.span_steps - 1);
    return *reinterpret_cast<const float4v*>(lds + my_basis + (step * kSteps + 16 * sub) * 32);
  };
  auto folded = [&](const Sums& a, float4v basis, float scale, float (&part)[NQ]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const float4v x = a.low[NQ == 1 ? 0 : r / 2];
      const float sum = __builtin_fmaf(x[0], basis[0], __builtin_fmaf(x[1], basis[1], __builtin_fmaf(x[2], basis[2], x[3] * basis[3])));
      const bool mine = NQ == 1 || (kg >> 1) == (r & 1);
      part[r] = mine ? __builtin_fmaf(sum, low_unit[r], part[r]) : part[r];
      part[r] *= scale;
    }
  };
  auto keys = [&](int n, int sub, float (&part)[NQ]) __attribute__((always_inline)) {
    Sums a;
    clear(a);
    const float2 tok = tok_of(n, sub);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) product(a, 4 * b + i, operand(n, sub, 4 * b + i));
      if (flags[n & 3]) zero_points(a, n, sub, b, 1.f);
      if (b + 1 < NB) scale_sums(a, tok.x);
    }
#pragma unroll
    for (int r = 0; r < NQ; ++r) part[r] = 0.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) pair(a, p, part);
    folded(a, basis_of(n, sub), tok.y, part);
  };
  // every query row's scores of step n, a token per lane, from the lane groups' parts of its sub-tiles
  auto whole_scores = [&](const float (&part)[4][NQ], float (&x)[NQ]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < NQ; ++r) x[r] = add_swapped16(add_swapped32(part[0][r], part[2][r]), add_swapped32(part[1][r], part[3][r]));
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
  struct Weights {                             // of step n's rows, on the way to LDS
    float x[NQ], u[NQ][MAXCB];
    uint32_t tok[MAXCB];                       // scale, zero-point
    bool seen;
  };
  // Scores and what of them the blocks' values weigh, masked; running maxima
  auto weigh = [&](int n, const float (&x)[NQ], Weights& w) __attribute__((always_inline)) {
    w.seen = attended(n, pos_of(n) + lane);
#pragma unroll
    for (int b = 0; b < MAXCB; ++b)
      if (b < CB) w.tok[b] = v_tok[((n & 3) * CB + b) * kSteps + lane];
    bool rises = false;
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      w.x[r] = w.seen ? x[r] : -INFINITY;
      rises = rises || w.x[r] > run_max[r] + kSlack;
#pragma unroll
      for (int b = 0; b < MAXCB; ++b)
        if (b < CB) {
          w.u[r][b] = w.x[r] + (float)__builtin_amdgcn_frexp_expf(F16::to_float((uint16_t)w.tok[b]));
          rises = rises || w.u[r][b] > blk_max[r][b] + kSlack;
        }
    }
    float* const alphas = reinterpret_cast<float*>(lds + ld.alpha) + (n & 1) * CB * 16 + hw * NQ;
    if (__any(rises)) {                        // seldom behind the first steps
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        const float now = fmaxf(run_max[r], max_of_wave(w.x[r]));
        run_sum[r] *= __builtin_amdgcn_exp2f(run_max[r] - (now == -INFINITY ? 0.f : now));
        run_max[r] = now;
#pragma unroll
        for (int b = 0; b < MAXCB; ++b)
          if (b < CB) {
            const float top = fmaxf(blk_max[r][b], max_of_wave(w.u[r][b]));
            const float alpha = __builtin_amdgcn_exp2f(blk_max[r][b] - (top == -INFINITY ? 0.f : top));
            z_sum[r][b] *= alpha;
            blk_max[r][b] = top;
            if (lane == 0) alphas[b * 16 + r] = alpha;
          }
      }
    } else if (lane < CB) {
#pragma unroll
      for (int r = 0; r < NQ; ++r) alphas[lane * 16 + r] = 1.f;
    }
  };
  auto add_sum = [&](const Weights& w, int r) __attribute__((always_inline)) {
    run_sum[r] += __builtin_amdgcn_exp2f(w.x[r] - (run_max[r] == -INFINITY ? 0.f : run_max[r]));
    asm volatile("" : "+v"(run_sum[r]));
  };
  auto weight = [&](const Weights& w, int r, int b) __attribute__((always_inline)) {
    const float y = __builtin_amdgcn_frexp_mantf(F16::to_float((uint16_t)w.tok[b])) * kWeightScale * __builtin_amdgcn_exp2f(w.u[r][b] - (blk_max[r][b] == -INFINITY ? 0.f : blk_max[r][b]));
    return w.seen ? y : 0.f;
  };
  auto put_weight = [&](int n, const Weights& w, int r, int b, float y) __attribute__((always_inline)) {
    z_sum[r][b] += w.seen ? y * (F16::to_float((uint16_t)(w.tok[b] >> 16)) - 8.f) : 0.f;
    asm volatile("" : "+v"(z_sum[r][b]));
    uint32_t hi, lo;
    split2<F16>(y, 0.f, &hi, &lo);
    uint16_t* P = reinterpret_cast<uint16_t*>(lds + ld.p + (n & 1) * ld.p_size + b * ld.p_cb + (hw * NQ + r) * kPagedQProbPitch) + lane;
    P[0] = (uint16_t)hi;
    P[kLoRows * (kPagedQProbPitch / 2)] = (uint16_t)lo;
  };
  auto softmax = [&](int n, const float (&x)[NQ]) __attribute__((always_inline)) {
    Weights w;
    weigh(n, x, w);
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      add_sum(w, r);
#pragma unroll
      for (int b = 0; b < MAXCB; ++b)
        if (b < CB) put_weight(n, w, r, b, weight(w, r, b));
    }
  };

  // ---- values of step n.  A wavefront has a block of 128 columns, and half of the tokens where there are one or two blocks.
  float4v O[8];                                // column 8 col + u of rows 4 kg + e; odd columns in units of 2^-20, even ones of 2^-24
#pragma unroll
  for (int u = 0; u < 8; ++u) O[u] = float4v{0, 0, 0, 0};
  const int vb = CB <= 2 ? wave % CB : min(wave, CB - 1);
  const int half0 = CB <= 2 ? wave / CB : 0;
  const bool has_values = CB <= 2 ? half0 < 2 : wave < CB;   // (the others do a part that another one does, results nowhere)
  // Codes enter as code - 8: most zero-points are near 8, and sums of codes and of zero-points, which all but cancel over many tokens, would leave their
  // rounding (4e-5 of the largest output at 3000 tokens, against 4e-6).
  const half2v minus8_even = __builtin_bit_cast(half2v, 0x80088008u), minus8_odd = __builtin_bit_cast(half2v, 0x80808080u);
  struct Values {
    uint32_t d[8];
    uint4v hi, lo, even, odd;
  };
  auto rescale = [&](int n) __attribute__((always_inline)) {
    const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (((n & 1) * CB + vb) * 16 + (NQ == 1 ? 0 : 4 * kg)) * 4);
    if (__any(!(al[0] == 1.f && al[1] == 1.f && al[2] == 1.f && al[3] == 1.f)))
#pragma unroll
      for (int u = 0; u < 8; ++u) O[u] *= al;
  };
  auto fetch_values = [&](int n, int half, Values& v) __attribute__((always_inline)) {
    const unsigned char* const at = lds + ld.v + ((n + VBUFS) % VBUFS) * ld.v_size + (32 * half + 8 * kg) * (v_cols / 2) + vb * 64 + col * 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) v.d[e] = *reinterpret_cast<const uint32_t*>(at + e * (v_cols / 2));
    const unsigned char* const P = lds + ld.p + (n & 1) * ld.p_size + vb * ld.p_cb + (NQ == 1 || SL == 2 ? col & 7 : col) * kPagedQProbPitch + (32 * half + 8 * kg) * 2;
    v.hi = *reinterpret_cast<const uint4v*>(P);
    if (NQ > 1) v.lo = *reinterpret_cast<const uint4v*>(P + kLoRows * kPagedQProbPitch);
  };
  // byte j of the codes, channels 2 j and 2 j + 1: of tokens 2 i and 2 i + 1; its products
  auto value_codes = [&](Values& v, int j, int i) __attribute__((always_inline)) {
    const uint32_t x = __builtin_amdgcn_perm(v.d[2 * i + 1], v.d[2 * i], 0x0c040c00u + 0x00010001u * j);
    v.even[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, x & 0x000f000fu) + minus8_even);
    v.odd[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, x & 0x00f000f0u) + minus8_odd);
  };
  auto value_products = [&](const Values& v, int j) __attribute__((always_inline)) {
    O[2 * j] = mma<F16>(v.hi, v.even, O[2 * j]);
    O[2 * j + 1] = mma<F16>(v.hi, v.odd, O[2 * j + 1]);
    if (NQ > 1) {
      O[2 * j] = mma<F16>(v.lo, v.even, O[2 * j]);
      O[2 * j + 1] = mma<F16>(v.lo, v.odd, O[2 * j + 1]);
    }
  };
  auto value_half = [&](int n, int half) __attribute__((always_inline)) {
    Values v;
    fetch_values(n, half, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) value_codes(v, j, i);
      value_products(v, j);
    }
  };
  auto values = [&](int n) __attribute__((always_inline)) {
    rescale(n);
    value_half(n, half0 & 1);
    if (CB > 2) value_half(n, 1);
  };

  if constexpr (PIPED) {
    // Interval n: the matrix instructions of step n's four sub-tiles; between them, dealt out a few at a time, the scores of the sub-tile before (of
    // step n - 1's last, of n's first three), the codes of step n + 1, the weights of n - 1, the values of n - 2.  One barrier.
    const int x0 = tid / k_pieces, pc = tid - x0 * k_pieces; // first piece of this thread; the second (of 256 columns) lies 32 rows on
    unsigned char* to[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) to[c] = lds + ld.k + x0 * ld.k_pitch + (((4 * pc) & ~15) | (((4 * pc + c) ^ x0) & 15)) * 16;
    const bool two = k_cols > 128;
    Sums sums[2];
    clear(sums[0]);
    clear(sums[1]);
    float part[4][NQ];
    constexpr int kPer = 4 + NG, kSlots = KS * kPer;         // matrix instructions of a step of channels, of a sub-tile
    // What a sub-tile begins with: its first operands, its tokens' scales, the basis of the one before it; requested in the middle of that one
    uint4v h[3];
    float2 tok_now = {}, tok_before = {};
    float4v basis = {};
    auto first_operands = [&](int n) __attribute__((always_inline)) {
      h[0] = operand(n, 0, 0);
      h[1] = operand(n, 0, 1);
      tok_now = tok_of(n, 0);
      basis = basis_of(n - 1, 3);
    };
    float early[NQ];                           // the scores of the last sub-tile of step n - 1
    // products of sub-tile SUB of step n, the scores of the sub-tile before it and MORE pieces of something else between them
    auto sub_tile = [&](auto sub_c, int n, bool left, auto more_c, auto&& more) __attribute__((always_inline)) {
      constexpr int SUB = decltype(sub_c)::value, MORE = decltype(more_c)::value;
      uint4v h_next[2] = {};
      Sums& now = sums[SUB & 1];
      const Sums& before = sums[(SUB + 1) & 1];
      float (&scores_before)[NQ] = *(SUB == 0 ? &early : &part[(SUB + 3) & 3]);
      const float ratio = NB == 2 ? tok_now.x : 1.f, scale_before = tok_before.y;
      const float4v basis_before = basis;
      tok_before = tok_now;
      clear(now);
#pragma unroll
      for (int r = 0; r < NQ; ++r) scores_before[r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks + 2 < KS) h[(ks + 2) % 3] = operand(n, SUB, ks + 2);
        if (SUB < 3 && ks + 2 >= KS) h_next[ks + 2 - KS] = operand(n, SUB < 3 ? SUB + 1 : SUB, ks + 2 - KS);
        if (SUB < 3 && ks == KS / 2) {
          tok_now = tok_of(n, SUB < 3 ? SUB + 1 : SUB);
          basis = basis_of(n, SUB);
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          float4v& sum = j < 4 ? now.acc[j] : now.low[NQ == 1 ? 0 : (j - 4) / 2];
          if (NB == 2 && ks == 4 && (j < 4 || NQ == 1 || j % 2 == 0)) sum *= ratio;
          sum = mma<F16>(j < 4 ? W[ks][j] : G[ks][j - 4], h[ks % 3], sum);
          const int slot = ks * kPer + j;
#pragma unroll
          for (int q = slot * 16 / kSlots; q < (slot + 1) * 16 / kSlots; ++q) {
            if (q & 1) pair_turns(q >> 1);
            else pair_adds(before, q >> 1, scores_before);
          }
#pragma unroll
          for (int q = slot * MORE / kSlots; q < (slot + 1) * MORE / kSlots; ++q) more(q);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      folded(before, basis_before, scale_before, scores_before);
#pragma unroll
      for (int r = 0; r < NQ; ++r) asm volatile("" : "+v"(scores_before[r]));
      h[0] = h_next[0];
      h[1] = h_next[1];
      if (left) {
        zero_points(now, n, SUB, 0, ratio);
        if (NB == 2) zero_points(now, n, SUB, NB - 1, 1.f);
      }
    };
    // the codes w of one piece, in sixteen pieces
    uint32_t both = 0;
    uint4v out;
    auto conversion = [&](int q, uint4v w, half2v off, int shift_bytes) __attribute__((always_inline)) {
      const int c = q >> 2, u = q & 3;
      if (u == 0) both = quarter_codes(w, c);
      out[u] = spread(both, off, u);
      asm volatile("" : "+v"(out[u]));
      if (u == 3) *reinterpret_cast<uint4v*>(to[c] + shift_bytes) = out;
    };
    // One query row: a quarter of the next span's folded weights in every step of a span of four
    constexpr bool AHEAD = NQ == 1;
    constexpr int kAhead = KS / 4;             // steps of channels
    uint4v H[AHEAD ? KS : 1];
    Nodes nodes;
    int ready = 0;                             // steps of channels that are folded
    for (int n = 0; n < n_steps; ++n) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // what interval n - 1 requested
      first_operands(n);
      const bool left = __builtin_amdgcn_readfirstlane(flags[n & 3]) != 0;
      // (behind the last step: codes of the one before it, converted into a buffer that nobody reads)
      const uint4v raw0 = raw_codes(n + 1, 0), raw1 = raw_codes(n + 1, two ? 1 : 0);
      const half2v off0 = zero_of(n + 1, x0, pc), off1 = zero_of(n + 1, two ? x0 + 32 : x0, pc);
      put(n);
      if (n + 2 < n_steps) request_keys(n + 2);
      request_values(n);
      request(n);
      const int k = span_of(n);
      const bool begins = folds(n), ahead = AHEAD && a.span_steps == 4 && span_step(k + 1) < n_steps;
      const int quarter_of_span = (n < steps_s ? n : n - steps_s) & 3;
      if (begins) {
        if (AHEAD && ready == KS) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) G[ks][0] = H[ks % (AHEAD ? KS : 1)];
        } else {
          fold(n);
        }
        ready = 0;
        if (ahead) nodes_of(k + 1, nodes);
      }
      const int next = ((n + 1) & 1) * ld.k_size, next1 = two ? next + 32 * ld.k_pitch : next;
      sub_tile(IntC<0>(), n, left, IntC<16>(), [&](int q) __attribute__((always_inline)) { conversion(q, raw0, off0, next); });
      if (begins) start(n);
      Weights w;
      float x[NQ], half_sums[NQ][2], first[NQ];
#pragma unroll
      for (int r = 0; r < NQ; ++r) first[r] = part[0][r];    // (sub-tile 1 makes another one)
      constexpr int kScores = NQ * 3;          // a row: halves of its scores by lane groups, wholes
      sub_tile(IntC<1>(), n, left, IntC<kScores + 16>(), [&](int q) __attribute__((always_inline)) {
        if (q >= kScores) {
          conversion(q - kScores, raw1, off1, next1);
        } else {
          const int r = q / 3;
          if (q % 3 < 2) half_sums[r][q % 3 & 1] = q % 3 == 0 ? add_swapped32(first[r], part[2][r]) : add_swapped32(part[1][r], early[r]);
          else x[r] = add_swapped16(half_sums[r][0], half_sums[r][1]);
          if (q % 3 < 2) asm volatile("" : "+v"(half_sums[r][q % 3 & 1]));
        }
      });
      if (n > 0) {
        weigh(n - 1, x, w);
      } else {                                 // no step before: weights of zero
        w.seen = false;
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          w.x[r] = -INFINITY;
#pragma unroll
          for (int b = 0; b < MAXCB; ++b) w.u[r][b] = -INFINITY;
        }
#pragma unroll
        for (int b = 0; b < MAXCB; ++b) w.tok[b] = 0;
      }
      uint4v f[kAhead][2][2];
      if (ahead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fold_weights(quarter_of_span * kAhead + i, f[i]);
      }
      Values v;
      fetch_values(n - 2, half0 & 1, v);
      float y = 0.f;
      constexpr int kRow = 1 + 2 * MAXCB, kWeights = NQ * kRow;          // a row: its sum, the blocks' weights and their way to LDS
      sub_tile(IntC<2>(), n, left, IntC<kWeights>(), [&](int q) __attribute__((always_inline)) {
        const int r = q / kRow, k = q % kRow;
        if (k == 0) {
          add_sum(w, r);
        } else if (k & 1) {
          y = weight(w, r, k >> 1);
          asm volatile("" : "+v"(y));
        } else {
          put_weight(n - 1, w, r, (k >> 1) - 1, y);
        }
      });
      rescale(n);                              // (of n - 2; in the first two intervals there are no weights and nothing to rescale)
      sub_tile(IntC<3>(), n, left, IntC<20>(), [&](int q) __attribute__((always_inline)) {
        if (q % 5 < 4) {
          value_codes(v, q / 5, q % 5);
          asm volatile("" : "+v"(v.even[q % 5 & 3]), "+v"(v.odd[q % 5 & 3]));
        } else {
          value_products(v, q / 5);
        }
      });
      if (CB > 2) value_half(n - 2, 1);
      if (ahead) {
        uint4v hi[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          prepare_weights(f[i]);
          const float4v d0 = fold_tile(f[i][0], nodes, 0), d1 = fold_tile(f[i][1], nodes, 0);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            uint32_t h, lo = 0;
            fold_pack(d0[u], d1[u], &h, &lo);
            hi[i][u] = h;
          }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (quarter_of_span == c)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) H[(c * kAhead + i) % (AHEAD ? KS : 1)] = hi[i];
        ready += kAhead;
      }
      lds_barrier();
    }
    {                                          // the last step's scores and values, and those of the one before it
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int r = 0; r < NQ; ++r) part[3][r] = 0.f;
#pragma unroll
      for (int p = 0; p < 8; ++p) pair(sums[1], p, part[3]);
      folded(sums[1], basis_of(n_steps - 1, 3), tok_of(n_steps - 1, 3).y, part[3]);
      float x[NQ];
      whole_scores(part, x);
      softmax(n_steps - 1, x);
      values(n_steps - 2);
      lds_barrier();
      values(n_steps - 1);
    }
  } else {
  for (int n = 0; n <= n_steps; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what interval n - 1 requested
    put(n);
    request(n);
    if (n > 0) values(n - 1);
    if (n == n_steps) break;
    if (folds(n)) {
      fold(n);
      start(n);
    }
    float part[4][NQ], x[NQ];
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) keys(n, sub, part[sub]);
    whole_scores(part, x);
    if (SL == 2 && slice == 1)
#pragma unroll
      for (int r = 0; r < NQ; ++r) scores[(hw * NQ + r) * kSteps + lane] = x[r];
    lds_barrier();
    if (n + 1 < n_steps) request_values(n + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + 1 < n_steps && i * 128 < k_cols) convert(n + 1, i);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the raw codes have been read)
    if (n + 2 < n_steps) request_keys(n + 2);
    if (SL == 2)
#pragma unroll
      for (int r = 0; r < NQ; ++r) x[r] += scores[(hw * NQ + r) * kSteps + lane];
    if (slice == 0) softmax(n, x);
    lds_barrier();
  }
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
      for (int u = 0; u < 8; ++u) y[u] = (y[u] * ((u & 1 ? 1048576.f : 16777216.f)) - f.x) * (f.y / kWeightScale);
      const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
      float* const o = a.o_part + slot * a.o_stride + (size_t)m.qpk * ohead + (size_t)(row0 + r) * rv + 128 * vb - vg * rv + 8 * col;
      *reinterpret_cast<float4v*>(o) = float4v{y[0], y[1], y[2], y[3]};
      *reinterpret_cast<float4v*>(o + 4) = float4v{y[4], y[5], y[6], y[7]};
    }
  }
}

namespace {
template <typename T, int NQ, int KS, int KB> PagedQFn pick_piped(int v_blocks) {
  if constexpr (NQ <= kPagedQPipedRows)
    return v_blocks == 1 ? pagedq_kernel<T, KS, 1, NQ, true, KB, 1> : (v_blocks == 2 ? pagedq_kernel<T, KS, 1, NQ, true, KB, 2> : pagedq_kernel<T, KS, 1, NQ, true, KB, 3>);
  return nullptr;
}
template <typename T, int NQ> PagedQFn pick(const PagedQForm& f) {
  if (f.slices == 2) return pagedq_kernel<T, 8, 2, NQ, false>;
  if (f.piped) return f.ks == 8 ? pick_piped<T, NQ, 8, 2>(f.v_blocks) : (f.k_blocks == 2 ? pick_piped<T, NQ, 4, 2>(f.v_blocks) : pick_piped<T, NQ, 4, 1>(f.v_blocks));
  return f.ks == 4 ? pagedq_kernel<T, 4, 1, NQ, false> : pagedq_kernel<T, 8, 1, NQ, false>;
}
}  // namespace

// (every number of rows is a translation unit of its own)
template <> PagedQFn pagedq_rows_form<PALU_PAGEDQ_ROWS>(int act, const PagedQForm& f) {
  return act == PALU_F16 ? pick<F16, PALU_PAGEDQ_ROWS>(f) : pick<BF16, PALU_PAGEDQ_ROWS>(f);
}

}  // namespace palu
