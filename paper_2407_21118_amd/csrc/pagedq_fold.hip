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
//
// A workgroup takes up to four heads of a group (or of groups side by side; two heads, in halves of their channels, for key ranks above 256) and a run of
// steps of 64 tokens.  Eight wavefronts, two to a SIMD: a head's rebuilt pairs half each, weights in registers for the whole run.  Codes are staged in LDS
// as exact float16 integers; a token's scales multiply sums, not codes.  In an interval one of the two wavefronts makes the scores of step n while the
// other weighs step n - 1, adds up the values of n - 2 and converts the codes of n + 1, and then the other way round: matrix and vector instructions go
// together without being mixed by hand.  (One wavefront per SIMD with 512 registers, its scores, weights, values and codes dealt out between the matrix
// instructions, as graph replays: 312 us for 16 x 8192 rows of 32 heads of rank 256 against 282, 177 against 157 for one sequence of 65536, and 193 against
// 106 for 4 x 16384 rows with four query rows a head, two of which are taken at a time here.  Calls among others take 278, 154 and 100.)
//
// Bound by the instructions of two wavefronts a SIMD and their latencies: 8700 cycles an interval, of which the matrix pipe is busy 2800 and the vector
// unit 5200; the start of a run takes 34000 (weights of 256 KB a workgroup from L2) and its end 4000.  One query row takes 64 + 16 operand rows a head
// where rebuilding takes 128; two rows 64 + 32, for which four rows rebuild every key twice: 4 x 16384 rows from 16-bit pages, rebuilt once for all, take
// 61 us.  Seven of the 32 forms spill 4 to 36 registers (20 to 92 bytes a lane), all with eight steps of channels: bfloat16 ones, and two rows with four
// value blocks.

#include "paged_dev.h"
#include "pagedq.h"

namespace palu {

namespace {

constexpr int kSteps = kPagedQStep, kThreads = kPagedQFoldThreads;
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
// as load_to_lds4, of 2 bytes per lane to the lower half of the lane's 4
__device__ __forceinline__ void load16_to_lds(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ushort %0, off" ::"v"(p), "s"(lds) : "memory");
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

// KS steps of 32 key channels per wavefront, SL slices of a head's channels, NQ query rows of a head, KB and VB blocks of 128 key and value columns of a
// unit, at most.  Eight wavefronts, two to a SIMD: of a head's rebuilt pairs (and of a slice of its channels) half each.
template <typename T, int KS, int SL, int NQ, int KB, int VB>
__global__ __launch_bounds__(kThreads, 2) void pagedq_kernel(PagedQArgs a) {
  constexpr int HEADS = 4 / SL;                // of a unit
  constexpr int NB = KS / 4;                   // blocks of 128 channels
  constexpr int NG = NQ;                       // operands of the folded query rows, 16 (row, node): with two rows hi and lo
  constexpr int PARTS = 2 * SL;                // wavefronts whose scores of a head are added up
  constexpr int kLoRows = 4 * NQ;              // rows of probabilities before those that the rounding left
  constexpr bool TWO = pagedq_two_phases(SL, NQ, VB);        // see below
  constexpr int KG = pagedq_key_scales(KS, KB);              // groups, or slices, with scales of their own
  constexpr int MB = VB < PARTS ? 1 : VB / PARTS;            // blocks of values whose weights a wavefront makes
  constexpr int NO = VB == 2 ? 4 : 8;          // columns of values of a lane
  constexpr PagedQLds ld = pagedq_lds(PagedQForm{KS, SL, NQ, KB, VB});
  static_assert(ld.total <= kPagedLdsBytes, "LDS");
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const PagedMeta& m = a.meta;
  const int tid = threadIdx.x;
  int lane = tid & 63;
  int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int col = lane & 15, kg = lane >> 4;
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
  const int share = span.n_tiles / n_chunks, longer = span.n_tiles - share * n_chunks;   // the first runs are a tile longer
  const int i0 = chunk * share + min(chunk, longer), i1 = i0 + share + (chunk < longer ? 1 : 0);
  const int g = un.group(), nh = un.nh(), h0 = un.h0();
  const int rk = m.k_off[g + 1] - m.k_off[g], rv = m.v_off[g + 1] - m.v_off[g], per_group = m.head_off[g + 1] - m.head_off[g];
  int k_cols = un.n_groups() * rk, v_cols = un.n_groups() * rv, CB = v_cols / 128;
  const int row0 = rb * NQ, nr = min(NQ, m.qpk - row0);      // query rows of a head
  const uint32_t lds0 = lds_addr(lds);

  int hw = wave % HEADS;
  const int half = (wave / HEADS) & 1, slice = wave / (2 * HEADS);
  int member = wave / HEADS;                           // among a head's wavefronts
  const int hh = min(hw, nh - 1);                            // (a wavefront without a head does another one's work, results nowhere)
  const int hg = un.n_groups() > 1 ? hh / per_group : 0;     // the head's group in the unit
  const int width = per_group * kDHead;
  const uint16_t* const B = a.Bk + m.bk_off[g] + (size_t)hg * rk * width + (size_t)(hh + h0 - m.head_off[g] - hg * per_group) * kDHead;
  const int ks_here = min(KS, (rk - slice * KS * 32) / 32);  // steps of this slice

  // ---- steps of 64 positions: those of the sinks' tiles first
  const int mid = max(i0, min(i1, span.sink_tiles));
  int steps_s = (mid - i0 + 1) / 2, n_steps = steps_s + (i1 - mid + 1) / 2;
  const int pos_w = kPagedTile * (span.tile0 + mid - span.sink_tiles);     // (where mid < i1)
  auto pos_of = [&](int n) __attribute__((always_inline)) { return n < steps_s ? kPagedTile * i0 + kSteps * n : pos_w + kSteps * (n - steps_s); };
  auto end_of = [&](int n) __attribute__((always_inline)) { return min(L, n < steps_s ? kPagedTile * mid : pos_w + kPagedTile * (i1 - mid)); };
  auto attended = [&](int n, int t) __attribute__((always_inline)) { return t < end_of(n) && (t < span.sink || t >= span.lo); };
  // spans: the first steps of either part, and every span_steps-th
  const int span_log = __builtin_ctz(a.span_steps), spans_s = (steps_s + a.span_steps - 1) >> span_log;
  auto folds = [&](int n) __attribute__((always_inline)) { return ((n < steps_s ? n : n - steps_s) & (a.span_steps - 1)) == 0; };
  auto span_of = [&](int n) __attribute__((always_inline)) { return n < steps_s ? n >> span_log : spans_s + ((n - steps_s) >> span_log); };
  auto span_step = [&](int k) __attribute__((always_inline)) { return k < spans_s ? k << span_log : steps_s + ((k - spans_s) << span_log); };

  // ---- requests.  In interval n: scales and zero-points of step n + 3, keys of n + 2, values of n, page-table entries of n + 5, the angles of the
  // third span after one that begins.
  constexpr int kMasked = 1 << 31;             // a masked token's row, with the number of an attended one's
  int* const rows = reinterpret_cast<int*>(lds + ld.rows);
  int k_pieces = k_cols / 32, v_pieces = v_cols / 32;  // 16-byte pieces of a raw row
  const int k_block0 = m.k_off[g] / 128, v_block0 = m.v_off[g] / 128;
  // (What a wavefront requests for itself waits in LDS, not in registers, for which the compiler would wait where paths join.)
  auto stage = [&](int i) __attribute__((always_inline)) { return reinterpret_cast<uint32_t*>(lds + ld.stage) + i * kSteps; };
  constexpr int kStageEntry = 2 * KB + 2 * VB;
  auto token_of = [&](int n, int x) __attribute__((always_inline)) {       // the position whose row token x reads (a masked token: the first attended one's)
    const int t0 = pos_of(n), t = t0 + x;
    return attended(n, t) ? t : (t0 < span.sink ? t0 : max(t0, span.lo));
  };
  auto entry_of = [&](int n) __attribute__((always_inline)) { return a.page_table + ((size_t)seq * a.table_stride + (token_of(n, lane) >> a.page_shift)); };
  auto put_rows = [&](int n, int e) __attribute__((always_inline)) {
    const int row = (max(0, min(e, a.n_pages - 1)) << a.page_shift) + (token_of(n, lane) & ((1 << a.page_shift) - 1));
    rows[(n & 7) * kSteps + lane] = row | (attended(n, pos_of(n) + lane) ? 0 : kMasked);
  };
  auto row_at = [&](int n, int x) __attribute__((always_inline)) { return (uint32_t)(rows[(n & 7) * kSteps + x] & ~kMasked); };
  // pieces of this thread: row, and piece of the row (of idle threads: those of others, results nowhere)
  constexpr int VBUFS = TWO ? 2 : 3;
  constexpr int KP = (KB + 1) / 2, VP = (VB + 1) / 2;        // pieces of keys and values per thread
  int k_x[KP], k_pc[KP], v_x[VP], v_pc[VP];
#pragma unroll
  for (int i = 0; i < KP; ++i) {
    const int id = (i * kThreads + tid) % (kSteps * k_pieces);
    k_x[i] = id / k_pieces;
    k_pc[i] = id - k_x[i] * k_pieces;
  }
#pragma unroll
  for (int i = 0; i < VP; ++i) {
    const int id = (i * kThreads + tid) % (kSteps * v_pieces);
    v_x[i] = id / v_pieces;
    v_pc[i] = id - v_x[i] * v_pieces;
  }
  const unsigned char *const k_src = a.k.codes + m.k_off[g] / 2, *const v_src = a.v.codes + m.v_off[g] / 2;
  uint4v raw[KP];
  auto request_keys = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KP; ++i)
      raw[i] = *reinterpret_cast<const uint4v*>(k_src + ((uint64_t)row_at(n, k_x[i]) * (uint32_t)a.k.row_bytes + k_pc[i] * 16));
  };
  auto request_values = [&](int n) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VP; ++i)
      if (i * kThreads + wave * 64 < kSteps * v_pieces)
        load_to_lds(v_src + ((uint64_t)row_at(n, v_x[i]) * (uint32_t)a.v.row_bytes + v_pc[i] * 16), lds0 + ld.v + n % VBUFS * ld.v_size + (i * kThreads + wave * 64) * 16);
  };
  // role 0: keys', 1: values'; an even and an odd wavefront's, which keeps to its role
  const PagedQSide& tok_side = wave & 1 ? a.v : a.k;
  const uint16_t* const tok_scale = tok_side.scale + (wave & 1 ? v_block0 : k_block0);
  const uint16_t* const tok_zero = tok_side.zero + (wave & 1 ? v_block0 : k_block0);
  const uint32_t tok_blocks = tok_side.n_blocks;
  auto request_tokens = [&](int n, int role) __attribute__((always_inline)) {
    const int blocks = role == 0 ? k_cols / 128 : CB;
    const uint64_t at = (uint64_t)row_at(n, lane) * tok_blocks;
    const uint16_t *scale = tok_scale + at, *zero = tok_zero + at;
    const uint32_t to = lds0 + ld.stage + (role == 0 ? 0 : 2 * KB) * kSteps * 4;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (b >= blocks) break;
      load16_to_lds(scale + b, to + 2 * b * kSteps * 4);
      load16_to_lds(zero + b, to + (2 * b + 1) * kSteps * 4);
    }
  };
  auto request_anchors = [&](int k) __attribute__((always_inline)) {
    const int pos = pos_of(span_step(k));
    load_to_lds4(a.rope + rope_f32_index(pos, lane, 0, kRopeTableStride), lds0 + ld.anchors + (k & 3) * kDHead * 4);
    load_to_lds4(a.rope + rope_f32_index(pos, lane, 1, kRopeTableStride), lds0 + ld.anchors + ((k & 3) * kDHead + kHalf) * 4);
  };
  auto request_entry = [&](int n) __attribute__((always_inline)) { load_to_lds4(entry_of(n), lds0 + ld.stage + kStageEntry * kSteps * 4); };
  // ---- what came of them
  float2* const k_tok = reinterpret_cast<float2*>(lds + ld.k_tok);
  uint32_t* const k_zero = reinterpret_cast<uint32_t*>(lds + ld.k_zero);
  uint32_t* const v_tok = reinterpret_cast<uint32_t*>(lds + ld.v_tok);
  float* const anchors = reinterpret_cast<float*>(lds + ld.anchors);
  int* const flags = reinterpret_cast<int*>(lds + ld.flags);
  auto put_tokens = [&](int n, int role) __attribute__((always_inline)) {
    // (all blocks that there may be: loads and conversions side by side; those behind the last are never read)
    if (role == 0) {
      uint32_t scale[KB], zero[KB];
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        scale[b] = stage(2 * b)[lane];
        zero[b] = stage(2 * b + 1)[lane] & 0xffffu;
      }
      bool any = false;
#pragma unroll
      for (int b = 0; b < KB; ++b) {           // codes take their zero-point where it is a small integer; what is left of it (with the other sign): see zero_points
        const float z = F16::to_float((uint16_t)zero[b]);
        const bool small = small_integer(z);
        any = any || (!small && b * 128 < k_cols);
        k_zero[((n & 3) * KB + b) * kSteps + lane] = (uint32_t)F16::from_float(-1024.f - (small ? z : 0.f)) | (small ? 0u : (zero[b] ^ 0x8000u) << 16);
      }
      flags[n & 3] = __any(any) ? 1 : 0;
#pragma unroll
      for (int s = 0; s < KG; ++s) {           // blocks of a slice, or of a group: (first * ratio + second) * scale.  (A second scale of zero: so
        const float s0 = F16::to_float((uint16_t)scale[NB * s]);         // small a number that nothing of the second block is left.)
        float s1 = s0, ratio = 1.f;
        if (NB == 2 && (SL == 1 || (2 * s + 1) * 128 < k_cols)) {
          s1 = F16::to_float((uint16_t)scale[(NB * s + 1) % KB]);
          if (s1 == 0.f) s1 = 0x1p-60f;
          ratio = s0 * __builtin_amdgcn_rcpf(s1);            // (right to 2^-22)
        }
        k_tok[((n & 3) * KG + s) * kSteps + lane] = make_float2(ratio, s1);
      }
    } else {
      uint32_t raw_tok[2 * VB];
#pragma unroll
      for (int b = 0; b < 2 * VB; ++b) raw_tok[b] = stage(2 * KB + b)[lane];
#pragma unroll
      for (int b = 0; b < VB; ++b) v_tok[((n & 3) * VB + b) * kSteps + lane] = (raw_tok[2 * b] & 0xffffu) | raw_tok[2 * b + 1] << 16;
    }
  };
  const uint32_t k1024 = per_lane_constant(0x64006400u);
  // piece i of this thread: its codes; what is added to 1024 + code; quarter c of it, lane group c's channels, 4 c + u and 16 + 4 c + u of the step
  auto zero_of = [&](int n, int x, int pc) __attribute__((always_inline)) {
    const uint32_t z = k_zero[((n & 3) * KB + (pc >> 2)) * kSteps + x];
    return __builtin_bit_cast(half2v, __builtin_amdgcn_perm(z, z, 0x01000100u));
  };
  auto convert = [&](int n, const uint4v (&w)[KP]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      if (i * kThreads + wave * 64 >= kSteps * k_pieces) break;
      const int x = k_x[i], pc = k_pc[i];
      const half2v off = zero_of(n, x, pc);
      unsigned char* const row = lds + ld.k + (TWO ? 0 : (n & 1) * ld.k_size) + x * ld.k_pitch + (4 * pc & ~15) * 16;
#pragma unroll
      for (int c = 0; c < 4; ++c) {            // lane group c's channels
        const uint32_t both = __builtin_amdgcn_perm(w[i][2 + (c >> 1)], w[i][c >> 1], c & 1 ? 0x07060302u : 0x05040100u);
        uint4v out;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          out[u] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, ((both >> (4 * u)) & 0x000f000fu) | k1024) + off);
        *reinterpret_cast<uint4v*>(row + (((4 * pc + c) ^ x) & 15) * 16) = out;
      }
    }
  };

  // ---- prologue: everything that memory has to give is requested first: page-table entries of the first four steps, queries, angles, weights
  const int first_entry = wave < min(4, n_steps) ? *entry_of(wave) : 0;
  float* const qs = reinterpret_cast<float*>(lds + ld.q) + hw * NQ * kDHead;         // queries, rotated to their position and scaled, [row][feature]
  const int q_pos = max(0, min(a.q_pos ? a.q_pos[seq] : L - 1, a.rope_len - 1));
  const float q_cos = a.rope[rope_f32_index(q_pos, lane, 0, kRopeTableStride)], q_sin = a.rope[rope_f32_index(q_pos, lane, 1, kRopeTableStride)];
  uint16_t q_raw[NQ][2];
#pragma unroll
  for (int r = 0; r < NQ; ++r) {
    const uint16_t* q = a.q + ((size_t)seq * m.n_heads * m.qpk + (h0 + hh) * m.qpk + row0 + min(r, nr - 1)) * kDHead;
    q_raw[r][0] = q[lane];
    q_raw[r][1] = q[lane + kHalf];
  }
  // rebuilt pairs: of a token of 16; 16 tokens on, pairs 16 half + 4 kg + p
  const float turn_cos = a.rope[rope_f32_index(min(tid >> 5, a.rope_len - 1), tid & 31, 0, kRopeTableStride)];
  const float turn_sin = a.rope[rope_f32_index(min(tid >> 5, a.rope_len - 1), tid & 31, 1, kRopeTableStride)];
  float tc[4], ts[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int f = 16 * half + 4 * kg + p, at16 = min(16, a.rope_len - 1);
    tc[p] = a.rope[rope_f32_index(at16, f, 0, kRopeTableStride)];
    ts[p] = a.rope[rope_f32_index(at16, f, 1, kRopeTableStride)];
  }
  // Weights, as operand rows.  W: tile j's row 2 x (+ 1) is feature 16 half + 2 x + j (+ 64), x < 8.  Those to be folded: a channel's features
  // 32 + 8 kg .. and 96 + 8 kg .., read for every span.  The halves take neighbouring steps of channels in the other order, and fold every second one.
  auto step_of = [&](int i) __attribute__((always_inline)) { return i ^ half; };
  const uint32_t b_pitch = width * 2;
  auto row_of = [&](int i, int x) __attribute__((always_inline)) {         // channel x of the step; steps behind the rank: the last, and zero instead
    const int ks = SL == 1 ? step_of(i) : min(step_of(i), ks_here - 1);
    return reinterpret_cast<const unsigned char*>(B) + (uint32_t)(slice * KS * 32 + 32 * ks + x) * b_pitch;
  };
  auto keep_of = [&](int i) __attribute__((always_inline)) { return SL == 1 || step_of(i) < ks_here ? 0xffffffffu : 0u; };
  uint4v W[KS][2];
  auto fold_weights = [&](int i, uint4v (&f)[2][2]) __attribute__((always_inline)) {
    const uint32_t at = col * b_pitch + (kPagedQLow + 8 * kg) * 2;
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
      for (int e = 0; e < 2; ++e) f[v][e] = *reinterpret_cast<const uint4v*>(row_of(2 * i, 16 * v) + (at + e * kHalf * 2));
    if (SL == 2)
#pragma unroll
      for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int e = 0; e < 2; ++e) f[v][e] &= keep_of(2 * i);
  };
  // W comes by LDS, half of the steps at a time, where keys and values will be: a step's 32 channels x 16 features twice in 2 KiB, the channels in an
  // order that spreads a lane group's over the banks.  (Loaded as operands, 4 bytes a lane, the weights took half of a prologue of 49000 cycles.)
  constexpr int kBatch = KS / 2;
  static_assert(ld.total - ld.p >= kBatch * 2048 * (kThreads / 64), "LDS");
  const int w_stage = ld.p + wave * (kBatch * 2048);
  auto request_weights = [&](int first) __attribute__((always_inline)) {
    const uint32_t at = (uint32_t)(16 * (lane >> 5) + 4 * ((lane >> 1) & 3) + ((lane >> 3) & 3)) * b_pitch + (16 * half + 8 * (lane & 1)) * 2;
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) load_to_lds(row_of(first + i, 0) + (at + e * kHalf * 2), lds0 + w_stage + i * 2048 + e * 1024);
  };
  uint32_t top = 0;                            // the largest, without its sign
  auto larger = [](uint32_t t, uint32_t w) __attribute__((always_inline)) { return max(t, max(w & 0x7fffu, (w >> 16) & 0x7fffu)); };
  auto take_weights = [&](int first) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t x[2];
#pragma unroll
        for (int v = 0; v < 2; ++v)
          x[v] = keep_of(first + i) & *reinterpret_cast<const uint32_t*>(lds + w_stage + i * 2048 + (col & 1) * 1024 + ((4 * v + u) * 8 + 2 * kg) * 16 + (col >> 1) * 4);
        W[first + i][0][u] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
        W[first + i][1][u] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
        if (!__is_same(T, F16)) top = larger(larger(top, x[0]), x[1]);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  request_weights(0);
  uint4v F[KS / 2][2][2];
#pragma unroll
  for (int i = 0; i < KS / 2; ++i) fold_weights(i, F[i]);
  __builtin_amdgcn_sched_barrier(0);

  if (wave < min(4, n_steps)) put_rows(wave, first_entry);
  float q_max[NQ], q_sum[NQ];                  // of the folded pairs
#pragma unroll
  for (int r = 0; r < NQ; ++r) {
    const float x0 = T::to_float(q_raw[r][0]), x1 = T::to_float(q_raw[r][1]);
    const float y0 = (x0 * q_cos - x1 * q_sin) * a.scale, y1 = (x1 * q_cos + x0 * q_sin) * a.scale;
    qs[r * kDHead + lane] = y0;
    qs[r * kDHead + kHalf + lane] = y1;
    const float size = lane >= kPagedQLow ? fabsf(y0) + fabsf(y1) : 0.f;
    q_max[r] = max_of_wave(size);
    q_sum[r] = sum_of_wave(size);
  }
  if (tid < kPagedQSpan) {
    // Lagrange polynomials of the span's Chebyshev nodes, per position, in their barycentric form.  (x is exact and so, but for one rounding, is its
    // distance to a node; that rounding moves an interpolated angle by 1e-7 of the span.)
    const float T2 = 0.5f * kSteps * a.span_steps, x = (tid - (T2 - 0.5f)) / T2;
    // cos((2 i + 1) pi / 16) and the barycentric weights (-1)^i sin((2 i + 1) pi / 16)
    constexpr float kNode[4] = {0.98078528040323044913f, 0.83146961230254523708f, 0.55557023301960222474f, 0.19509032201612826785f};
    float w[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float node = i < 4 ? kNode[i] : -kNode[7 - i], weight = (i & 1 ? -1.f : 1.f) * kNode[i < 4 ? 3 - i : i - 4];
      w[i] = weight / (x - node);
      sum += w[i];
    }
    float* const basis = reinterpret_cast<float*>(lds + ld.basis) + tid * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) basis[i] = w[i] / sum;
    const int i = tid >> 5, f = tid & 31;      // a node, a folded pair
    const float node = (T2 - 0.5f) + T2 * (i < 4 ? kNode[i & 3] : -kNode[7 - i & 3]);
    float* const at = reinterpret_cast<float*>(lds + ld.nodes + i * kPagedQTurnPitch) + f;
    sincosf(a.w_low[f] * node, at + kPagedQLow, at);
  }
  {
    float* const at = reinterpret_cast<float*>(lds + ld.turns + (tid >> 5) * kPagedQTurnPitch) + (tid & 31);
    at[0] = turn_cos;
    at[kPagedQLow] = turn_sin;
  }
  lds_barrier();
  request_keys(0);
  if (wave < 2) request_tokens(0, wave);
  if (wave == 3) request_entry(min(4, n_steps - 1));
  if (wave >= 4 && wave < 7 && span_step(wave - 4) < n_steps) request_anchors(wave - 4);

  int shift = 0;                               // weights are held times 2^shift
  float b_max = 0.f;                           // of those to be folded
  auto prepare_weights = [&](uint4v (&f)[2][2]) __attribute__((always_inline)) {
    if (!__is_same(T, F16))
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 2; ++e) f[v][e][i] = to_f16<T>(f[v][e][i], shift);
  };
  {
    uint32_t top_f = 0;
    take_weights(0);
    request_weights(kBatch);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
          for (int e = 0; e < 2; ++e) top_f = larger(top_f, F[i][v][e][u]);
    b_max = max_of_wave(T::to_float((uint16_t)top_f));
    take_weights(kBatch);
    if (!__is_same(T, F16)) {
      const float all = max_of_wave(T::to_float((uint16_t)max(top, top_f)));
      shift = __builtin_amdgcn_readfirstlane(15 - __builtin_amdgcn_frexp_expf(all));
      b_max = __builtin_amdgcn_ldexpf(b_max, shift);
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int u = 0; u < 4; ++u) W[i][j][u] = to_f16<T>(W[i][j][u], shift);
    }
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) asm volatile("" : "+v"(W[i][j]));
  }

  const float unit = __builtin_amdgcn_ldexpf(1.f, -shift);
  int ea[NQ];
#pragma unroll
  for (int r = 0; r < NQ; ++r)
    // a folded weight is at most b_max * sqrt(2) * q_sum, an a or b at most q_max: both times 2^e are float16 numbers
    ea[r] = __builtin_amdgcn_readfirstlane(min(15 - __builtin_amdgcn_frexp_expf(1.4143f * b_max * q_sum[r]), 15 - __builtin_amdgcn_frexp_expf(q_max[r])));

  // ---- the first step's keys
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  lds_barrier();
  for (int x = tid; x < 2 * ld.p_size / 16; x += kThreads) *reinterpret_cast<uint4v*>(lds + ld.p + x * 16) = uint4v{0, 0, 0, 0};   // weights of values before the first step
  for (int x = tid; x < 2 * VB * 16; x += kThreads) reinterpret_cast<float*>(lds + ld.alpha)[x] = 1.f;
  if (wave < 2) {
    put_tokens(0, wave);
    if (n_steps > 1) request_tokens(1, wave);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (n_steps > 1) put_tokens(1, wave);
  }
  lds_barrier();
  convert(0, raw);
  if (n_steps > 1) request_keys(1);
  if (n_steps > 2 && wave < 2) request_tokens(2, wave);
  lds_barrier();

  // What interval n - 1 requested goes to LDS, before anything is requested: the compiler waits for all loads that it does not know of, too
  auto put = [&](int n) __attribute__((always_inline)) {
    if (wave < 2) {
      if (n + 2 < n_steps) put_tokens(n + 2, wave);
    } else if (wave == 3) {
      if (n + 4 < n_steps) put_rows(n + 4, (int)stage(kStageEntry)[lane]);
    }
  };
  auto request = [&](int n) __attribute__((always_inline)) {
    if (wave < 2) {
      request_tokens(min(n + 3, n_steps - 1), wave);
    } else if (wave == 2) {
      if (folds(n) && span_step(span_of(n) + 3) < n_steps) request_anchors(span_of(n) + 3);
    } else if (wave == 3) {
      if (n + 5 < n_steps) request_entry(n + 5);
    }
  };
  float sc[4] = {}, ss[4] = {};                // cos and sin (one query row: a and b) of the next 16 tokens
  // angles of the first 16 tokens of step n
  auto start = [&](int n) __attribute__((always_inline)) {
    const float* const at = anchors + (span_of(n) & 3) * kDHead + 16 * half + 4 * kg;
    const float* const on = reinterpret_cast<const float*>(lds + ld.turns + col * kPagedQTurnPitch) + 16 * half + 4 * kg;
    const float4v c0 = *reinterpret_cast<const float4v*>(at), s0 = *reinterpret_cast<const float4v*>(at + kHalf);
    const float4v c1 = *reinterpret_cast<const float4v*>(on), s1 = *reinterpret_cast<const float4v*>(on + kPagedQLow);
    const float4v x = *reinterpret_cast<const float4v*>(qs + 16 * half + 4 * kg), y = *reinterpret_cast<const float4v*>(qs + kHalf + 16 * half + 4 * kg);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const float c = __builtin_fmaf(c0[p], c1[p], -(s0[p] * s1[p])), s = __builtin_fmaf(c0[p], s1[p], s0[p] * c1[p]);
      sc[p] = NQ == 1 ? __builtin_fmaf(c, x[p], s * y[p]) : c;
      ss[p] = NQ == 1 ? __builtin_fmaf(c, y[p], -(s * x[p])) : s;
    }
  };
  // a and b of the folded pairs at the nodes of span k, hi and lo (one row: by lanes)
  struct Nodes {
    uint4v a[NG], b[NG];
  };
  uint4v G[KS / 2][NG];                        // the folded weights
  auto nodes_of = [&](int k, Nodes& v) __attribute__((always_inline)) {
    const int f = 8 * kg, upper = NQ == 1 ? 0 : col >> 3;    // which of a group's two rows
    const float* const at = anchors + (k & 3) * kDHead + kPagedQLow + f;
    const float* const on = reinterpret_cast<const float*>(lds + ld.nodes + (col & 7) * kPagedQTurnPitch) + f;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float4v c0 = *reinterpret_cast<const float4v*>(at + 4 * q), s0 = *reinterpret_cast<const float4v*>(at + kHalf + 4 * q);
      const float4v c1 = *reinterpret_cast<const float4v*>(on + 4 * q), s1 = *reinterpret_cast<const float4v*>(on + kPagedQLow + 4 * q);
      const float* const row = qs + upper * kDHead + kPagedQLow + f + 4 * q;
      const float4v x = *reinterpret_cast<const float4v*>(row), y = *reinterpret_cast<const float4v*>(row + kHalf);
      const int e = upper ? ea[NQ - 1] : ea[0];
      float u[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float c = __builtin_fmaf(c0[i], c1[i], -(s0[i] * s1[i])), s = __builtin_fmaf(c0[i], s1[i], s0[i] * c1[i]);
        u[i] = __builtin_amdgcn_ldexpf(__builtin_fmaf(c, x[i], s * y[i]), e);
        w[i] = __builtin_amdgcn_ldexpf(__builtin_fmaf(c, y[i], -(s * x[i])), e);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t h, lo;
        split2<F16>(u[2 * i], u[2 * i + 1], &h, &lo);
        v.a[0][2 * q + i] = NQ == 1 && col >= 8 ? lo : h;
        if (NQ > 1) v.a[NG - 1][2 * q + i] = lo;
        split2<F16>(w[2 * i], w[2 * i + 1], &h, &lo);
        v.b[0][2 * q + i] = NQ == 1 && col >= 8 ? lo : h;
        if (NQ > 1) v.b[NG - 1][2 * q + i] = lo;
      }
    }
  };
  // Folded weights of channel step ks, from its weights f
  const float lo_part = NQ == 1 && col >= 8 ? -1.f : 0.f;    // one row: these lanes hold what the rounding leaves
  auto fold_tile = [&](const uint4v (&f)[2], const Nodes& v) __attribute__((always_inline)) {
    float4v d = {0, 0, 0, 0};
#pragma unroll
    for (int l = 0; l < NG; ++l) {
      d = mma<F16>(f[0], v.a[l], d);
      d = mma<F16>(f[1], v.b[l], d);
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
  auto fold_one = [&](const uint4v (&f)[2][2], const Nodes& v, uint4v (&g)[NG]) __attribute__((always_inline)) {
    const float4v d0 = fold_tile(f[0], v), d1 = fold_tile(f[1], v);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t hi, lo = 0;
      fold_pack(d0[u], d1[u], &hi, &lo);
      g[0][u] = hi;
      if (NQ > 1) g[NG - 1][u] = lo;
    }
  };
  auto fold = [&](int n) __attribute__((always_inline)) {
    Nodes v;
    constexpr int kAhead = 2;             // weights in registers at a time
    uint4v f[kAhead][2][2];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fold_weights(i, f[i]);
    nodes_of(span_of(n), v);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      prepare_weights(f[i % kAhead]);
      fold_one(f[i % kAhead], v, G[i]);
      if (i + kAhead < KS / 2) fold_weights(i + kAhead, f[i % kAhead]);
    }
  };

  // ---- keys of sub-tile `sub` of step n: every query row's partial score of token col, by lane group
  int k_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_off[i] = (SL == 1 ? hg * KS * 64 : slice * 512) + col * ld.k_pitch + (((4 * step_of(i) + kg) ^ col) & 15) * 16;
  const int b_last = ks_here / 4 - 1;          // last block of this slice
  struct Sums {
    float4v acc[2], low;
  };
  auto clear = [&](Sums& a) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) a.acc[j] = float4v{0, 0, 0, 0};
    a.low = float4v{0, 0, 0, 0};
  };
  auto product = [&](Sums& a, int i, uint4v h) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) a.acc[j] = mma<F16>(W[i][j], h, a.acc[j]);
    if (i % 2 == 0)
#pragma unroll
      for (int l = 0; l < NG; ++l) a.low = mma<F16>(G[i / 2][l], h, a.low);
  };
  auto scale_sums = [&](Sums& a, float x) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) a.acc[j] *= x;
    a.low *= x;
  };
  // zero-points that are no small integers: as operands of their own, the same for all channels of block b, times x
  auto zero_points = [&](Sums& a, int n, int sub, int b, float x) __attribute__((always_inline)) {
    const int block = SL == 1 ? hg * NB + b : min(2 * slice + b, k_cols / 128 - 1);
    const uint32_t z = k_zero[((n & 3) * KB + block) * kSteps + 16 * sub + col], w = __builtin_amdgcn_perm(z, z, 0x03020302u);
    Sums more;
    clear(more);
#pragma unroll
    for (int i = 0; i < 4; ++i) product(more, 4 * b + i, uint4v{w, w, w, w});
#pragma unroll
    for (int j = 0; j < 2; ++j) a.acc[j] += more.acc[j] * x;
    a.low += more.low * x;
  };
  // What pair p of this lane adds to the scores; its angle (one query row: a and b) 16 tokens on
  auto pair = [&](const Sums& a, int p, const float4v (&qa)[NQ], const float4v (&qb)[NQ], float (&part)[NQ]) __attribute__((always_inline)) {
    const float lo = a.acc[p & 1][2 * (p >> 1)], hi = a.acc[p & 1][2 * (p >> 1) + 1], c = sc[p], s = ss[p];
    if (NQ == 1) {
      part[0] = __builtin_fmaf(lo, c, part[0]);
      part[0] = __builtin_fmaf(hi, s, part[0]);
      sc[p] = __builtin_fmaf(c, tc[p], s * ts[p]);
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
  };
  const int my_basis = ld.basis + (col * 8 + 4 * (kg & 1)) * 4;
  auto scores_from = [&](const Sums& z, float4v basis, float scale, float (&part)[NQ]) __attribute__((always_inline)) {
    float4v qa[NQ] = {}, qb[NQ] = {};          // several rows: the queries
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      part[r] = 0.f;
      if (NQ == 1) continue;
      qa[r] = *reinterpret_cast<const float4v*>(qs + r * kDHead + 16 * half + 4 * kg);
      qb[r] = *reinterpret_cast<const float4v*>(qs + r * kDHead + kHalf + 16 * half + 4 * kg);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) pair(z, p, qa, qb, part);
    // (lanes of the folded pairs' rows 0 and 1: what is not a number stays in its row)
    const float sum = __builtin_fmaf(z.low[0], basis[0], __builtin_fmaf(z.low[1], basis[1], __builtin_fmaf(z.low[2], basis[2], z.low[3] * basis[3])));
    if (NQ == 1) {
      part[0] = __builtin_fmaf(sum, __builtin_amdgcn_ldexpf(1.f, -ea[0]), part[0]) * (unit * scale);
    } else {
      const float low = __builtin_amdgcn_ldexpf(sum, -(kg < 2 ? ea[0] : ea[NQ - 1]));
#pragma unroll
      for (int r = 0; r < NQ; ++r) part[r] = (part[r] + (kg >> 1 == r ? low : 0.f)) * (unit * scale);
    }
  };
  auto keys = [&](int n, int sub, float (&part)[NQ]) __attribute__((always_inline)) {
    Sums z;
    clear(z);
    const float2 tok = k_tok[((n & 3) * KG + (SL == 1 ? hg : slice)) * kSteps + 16 * sub + col];
    const unsigned char* const k = lds + ld.k + (TWO ? 0 : (n & 1) * ld.k_size) + 16 * sub * ld.k_pitch;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) product(z, 4 * b + i, *reinterpret_cast<const uint4v*>(k + k_off[i] + (SL == 1 ? b : min(b, b_last)) * 256));
      __builtin_amdgcn_sched_barrier(0);
      zero_points(z, n, sub, b, 1.f);
      if (b + 1 < NB) scale_sums(z, tok.x);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int step = (n < steps_s ? n : n - steps_s) & (a.span_steps - 1);
    scores_from(z, *reinterpret_cast<const float4v*>(lds + my_basis + (step * kSteps + 16 * sub) * 32), tok.y, part);
  };
  // All four sub-tiles of step n, without such zero-points: operands are read four steps of channels ahead, a
  // sub-tile's scores are made among the products of the next
  auto quick_keys = [&](int n, float (&part)[4][NQ]) __attribute__((always_inline)) {
    constexpr int kDeep = 4;
    const unsigned char* const k = lds + ld.k + (TWO ? 0 : (n & 1) * ld.k_size);
    auto operand = [&](int x) __attribute__((always_inline)) {
      const int sub = x / KS, i = x % KS;
      return *reinterpret_cast<const uint4v*>(k + 16 * sub * ld.k_pitch + k_off[i & 3] + (SL == 1 ? i >> 2 : min(i >> 2, b_last)) * 256);
    };
    const int step = (n < steps_s ? n : n - steps_s) & (a.span_steps - 1);
    const unsigned char* const basis_at = lds + my_basis + step * kSteps * 32;
    const float2* const tok_at = k_tok + ((n & 3) * KG + (SL == 1 ? hg : slice)) * kSteps + col;
    uint4v h[kDeep];
    Sums z[2];
    float2 tok = {}, tok_before = {};
    float4v basis = {};
#pragma unroll
    for (int x = 0; x < kDeep; ++x) h[x] = operand(x);
#pragma unroll
    for (int x = 0; x < 4 * KS; ++x) {
      const int sub = x / KS, i = x % KS;
      Sums& now = z[sub & 1];
      if (i == 0) {
        clear(now);
        tok_before = tok;
        tok = tok_at[16 * sub];
      }
      if (NB == 2 && i == 4) scale_sums(now, tok.x);
      product(now, i, h[x % kDeep]);
      if (x + kDeep < 4 * KS) h[x % kDeep] = operand(x + kDeep);
      if (sub > 0 && i == 2) scores_from(z[(sub - 1) & 1], basis, tok_before.y, part[sub > 0 ? sub - 1 : 0]);
      if (i == KS - 1) basis = *reinterpret_cast<const float4v*>(basis_at + 16 * sub * 32);
      __builtin_amdgcn_sched_barrier(0);
    }
    scores_from(z[1], basis, tok.y, part[3]);
  };
  float* const scores = reinterpret_cast<float*>(lds + ld.scores);
  auto scores_of = [&](int n, int r) __attribute__((always_inline)) {     // of this head's row r: PARTS parts
    return scores + (((TWO ? 0 : n & 1) * HEADS + hw) * NQ + r) * PARTS * kSteps + lane;
  };
  constexpr bool AHEAD = NQ == 1 && VB == 2 && SL == 1;
  uint4v H[AHEAD ? KS / 2 : 1][NG];
  Nodes nodes;
  int ready = 0;                               // steps of channels of the next span that are folded
  // One query row: of the next span's folded weights, one step of channels in every step of a span of four
  auto quarter_of = [&](int n) __attribute__((always_inline)) { return (n < steps_s ? n : n - steps_s) & 3; };
  auto ahead = [&](int n) __attribute__((always_inline)) { return AHEAD && a.span_steps == 4 && quarter_of(n) < KS / 2 && n < n_steps && span_step(span_of(n) + 1) < n_steps; };
  auto fold_ahead = [&](int n, uint4v (&f)[2][2]) __attribute__((always_inline)) {
    uint4v g[NG];
    prepare_weights(f);
    fold_one(f, nodes, g);
#pragma unroll
    for (int i = 0; i < (AHEAD ? KS / 2 : 0); ++i)
      if (quarter_of(n) == i) H[i][0] = g[0];
    ++ready;
  };
  auto begin_span = [&](int n) __attribute__((always_inline)) {
    if (ready == KS / 2) {                     // (or in G already)
#pragma unroll
      for (int i = 0; i < (AHEAD ? KS / 2 : 0); ++i) G[i][0] = H[AHEAD ? i : 0][0];
    } else {
      fold(n);
    }
    ready = 0;
    start(n);
    if (AHEAD) nodes_of(span_of(n) + 1, nodes);
  };
  // this wavefront's part of step n's scores, a token per lane
  auto all_keys = [&](int n) __attribute__((always_inline)) {
    if (__builtin_amdgcn_readfirstlane(flags[n & 3]) != 0) {
#pragma unroll 1
      for (int sub = 0; sub < 4; ++sub) {
        float part[NQ];
        keys(n, sub, part);
#pragma unroll
        for (int r = 0; r < NQ; ++r) {
          const float two = add_swapped32(part[r], part[r]), sum = add_swapped16(two, two);
          if (kg == 0) scores_of(n, r)[member * kSteps - lane + 16 * sub + col] = sum;
        }
      }
    } else {
      float part[4][NQ];
      quick_keys(n, part);
#pragma unroll
      for (int r = 0; r < NQ; ++r)
        scores_of(n, r)[member * kSteps] = add_swapped16(add_swapped32(part[0][r], part[2][r]), add_swapped32(part[1][r], part[3][r]));
    }
  };

  // ---- softmax of step n, a token per lane: weights of the values' blocks member, member + PARTS, ..
  float run_max[NQ], run_sum[NQ], blk_max[NQ][MB], z_sum[NQ][MB];
#pragma unroll
  for (int r = 0; r < NQ; ++r) {
    run_max[r] = -INFINITY;
    run_sum[r] = 0.f;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      blk_max[r][i] = -INFINITY;
      z_sum[r][i] = 0.f;
    }
  }
  auto softmax = [&](int n) __attribute__((always_inline)) {
    const bool seen = rows[(n & 7) * kSteps + lane] >= 0;
    float x[NQ], u[NQ][MB];
    uint32_t tok[MB];                          // scale, zero-point
#pragma unroll
    for (int i = 0; i < MB; ++i) tok[i] = v_tok[((n & 3) * VB + min(member + PARTS * i, CB - 1)) * kSteps + lane];
    bool rises = false;
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      const float* const at = scores_of(n, r);
      float sum = at[0];
#pragma unroll
      for (int i = 1; i < PARTS; ++i) sum += at[i * kSteps];
      x[r] = seen ? sum + (sum - sum) : -INFINITY;             // (of an infinite score nothing is known: not a number)
      rises = rises || x[r] > run_max[r] + kSlack;
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        u[r][i] = x[r] + (float)__builtin_amdgcn_frexp_expf(F16::to_float((uint16_t)tok[i]));
        rises = rises || u[r][i] > blk_max[r][i] + kSlack;
      }
    }
    float* const alphas = reinterpret_cast<float*>(lds + ld.alpha) + ((n & 1) * VB + member) * 16 + hw * NQ;
    if (__any(rises)) {                        // seldom behind the first steps
#pragma unroll
      for (int r = 0; r < NQ; ++r) {
        const float now = fmaxf(run_max[r], max_of_wave(x[r]));
        run_sum[r] *= __builtin_amdgcn_exp2f(run_max[r] - (now == -INFINITY ? 0.f : now));
        run_max[r] = now;
#pragma unroll
        for (int i = 0; i < MB; ++i) {
          const float top = fmaxf(blk_max[r][i], max_of_wave(u[r][i]));
          const float alpha = __builtin_amdgcn_exp2f(blk_max[r][i] - (top == -INFINITY ? 0.f : top));
          z_sum[r][i] *= alpha;
          blk_max[r][i] = top;
          if (lane == 0 && member + PARTS * i < CB) alphas[PARTS * 16 * i + r] = alpha;
        }
      }
    } else if (lane < NQ) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
        if (member + PARTS * i < CB) alphas[PARTS * 16 * i + lane] = 1.f;
    }
#pragma unroll
    for (int r = 0; r < NQ; ++r) {
      run_sum[r] += __builtin_amdgcn_exp2f(x[r] - (run_max[r] == -INFINITY ? 0.f : run_max[r]));
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        if (member + PARTS * i >= CB) break;
        float y = __builtin_amdgcn_frexp_mantf(F16::to_float((uint16_t)tok[i])) * kWeightScale * __builtin_amdgcn_exp2f(u[r][i] - (blk_max[r][i] == -INFINITY ? 0.f : blk_max[r][i]));
        y = seen ? y : 0.f;
        z_sum[r][i] += seen ? y * (F16::to_float((uint16_t)(tok[i] >> 16)) - 8.f) : 0.f;
        uint32_t hi, lo;
        split2<F16>(y, 0.f, &hi, &lo);
        uint16_t* P = reinterpret_cast<uint16_t*>(lds + ld.p + (n & 1) * ld.p_size + (member + PARTS * i) * ld.p_cb + (hw * NQ + r) * kPagedQProbPitch) + lane;
        P[0] = (uint16_t)hi;
        P[kLoRows * (kPagedQProbPitch / 2)] = (uint16_t)lo;
      }
    }
  };

  // ---- values of step n.  A wavefront has half of the tokens of a block of 128 columns, where there are one or two blocks of every second four.
  float4v O[NO];                               // column 8 col + (4 quarter +) u of rows 4 kg + e (behind the weights' rows those of what their rounding left); odd columns in units of 1/16
#pragma unroll
  for (int u = 0; u < NO; ++u) O[u] = float4v{0, 0, 0, 0};
  int vb0 = wave & (VB - 1), half0 = VB == 2 ? (wave >> 1) & 1 : wave >> 2, quarter = VB == 2 ? wave >> 2 : 0;
  // Codes enter as code - 8: most zero-points are near 8, and sums of codes and of zero-points, which all but cancel over many tokens, would leave their
  // rounding (4e-5 of the largest output at 3000 tokens, against 4e-6).  As normal numbers, by way of 1024 + code or 1024 + 16 code: the matrix cores keep 24
  // bits below the largest exponent of an instruction's products and take a subnormal operand's for 2^-14 (codes in units of 2^-24 and 2^-20 added an error of
  // 5.4e-5 of the output, 2-norm, to 65536 rows).
  const half2v minus8_even = __builtin_bit_cast(half2v, 0xe408e408u), minus8_odd = __builtin_bit_cast(half2v, 0xe480e480u);   // -1032, -1152
  auto values = [&](int n) __attribute__((always_inline)) {
    const int vb = vb0;
    if (vb >= CB) return;
    const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (((n & 1) * VB + vb) * 16 + 4 * (kg & (NQ - 1))) * 4);
    const unsigned char* const at = lds + ld.v + n % VBUFS * ld.v_size + (32 * half0 + 8 * kg) * (v_cols / 2) + vb * 64 + col * 4;
    uint32_t d[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = *reinterpret_cast<const uint32_t*>(at + e * (v_cols / 2));
    const unsigned char* const P = lds + ld.p + (n & 1) * ld.p_size + vb * ld.p_cb + (col & (2 * kLoRows - 1)) * kPagedQProbPitch + (32 * half0 + 8 * kg) * 2;
    const uint4v p = *reinterpret_cast<const uint4v*>(P);
    if (__any(!(al[0] == 1.f && al[1] == 1.f && al[2] == 1.f && al[3] == 1.f)))
#pragma unroll
      for (int u = 0; u < NO; ++u) O[u] *= al;
#pragma unroll
    for (int j = 0; j < NO / 2; ++j) {         // byte j (+ 2) of the codes
      const uint32_t pick = 0x0c040c00u + 0x00010001u * (j + 2 * quarter);
      uint4v even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {            // tokens 2 i, 2 i + 1
        const uint32_t x = __builtin_amdgcn_perm(d[2 * i + 1], d[2 * i], pick);
        even[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, (x & 0x000f000fu) | k1024) + minus8_even);
        odd[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, (x & 0x00f000f0u) | k1024) + minus8_odd);
      }
      O[2 * j] = mma<F16>(p, even, O[2 * j]);
      O[2 * j + 1] = mma<F16>(p, odd, O[2 * j + 1]);
    }
  };

  // ---- Interval n: the scores of step n, the weights of n - 1, the values of n - 2, the codes of n + 1, and one barrier.  Of a head's two wavefronts,
  // which share a SIMD, one begins with the scores and one with the rest: the matrix instructions of either go with the vector instructions of the other.
  // Where LDS cannot hold two steps' keys (TWO): the scores, a barrier, the weights of the same step, the values of n - 1, the codes, a barrier.
  uint4v now[KP];
  auto here = [&]() __attribute__((always_inline)) {         // addresses are made where they are used: kept over the loop they fill the registers
    asm volatile("" : "+v"(lane), "+v"(col), "+v"(kg));
    asm volatile("" : "+s"(wave), "+s"(member), "+s"(hw), "+s"(k_cols), "+s"(v_cols), "+s"(CB), "+s"(k_pieces), "+s"(v_pieces), "+s"(steps_s), "+s"(n_steps), "+s"(vb0), "+s"(half0), "+s"(quarter));
#pragma unroll
    for (int i = 0; i < KP; ++i) asm volatile("" : "+v"(k_x[i]), "+v"(k_pc[i]), "+v"(now[i]));
#pragma unroll
    for (int i = 0; i < VP; ++i) asm volatile("" : "+v"(v_x[i]), "+v"(v_pc[i]));
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(k_off[i]));
  };
  const int n_end = n_steps + (TWO ? 1 : 2);
  if (NQ == 1) {                               // the first span's.  (With two rows the weights' registers are wanted, and it reads them again.)
    nodes_of(0, nodes);
#pragma unroll
    for (int i = 0; i < KS / 2; ++i) {
      prepare_weights(F[i]);
      if (AHEAD) fold_one(F[i], nodes, H[AHEAD ? i : 0]);
      else fold_one(F[i], nodes, G[i]);
    }
    ready = KS / 2;
  }
  for (int n = 0; n < n_end; ++n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what interval n - 1 requested
#pragma unroll
    for (int i = 0; i < KP; ++i) now[i] = raw[i];
    here();
    put(n);
    if (n + 2 < n_steps) request_keys(n + 2);
    if (n < n_steps) request_values(n);
    request(n);
    constexpr bool kAtTop = AHEAD || TWO;      // (else one wavefront of a SIMD folds while the other does the rest)
    if (kAtTop && n < n_steps && folds(n)) begin_span(n);
    if constexpr (TWO) {
      here();
      if (n < n_steps) all_keys(n);
      lds_barrier();
      here();
      if (n < n_steps) softmax(n);
      if (n > 0) values(n - 1);
      if (n + 1 < n_steps) convert(n + 1, now);
    } else {
#pragma unroll 1
      for (int turn = 0; turn < 2; ++turn) {
        here();
        if (turn == half) {
          if (!kAtTop && n < n_steps && folds(n)) begin_span(n);
          if (n < n_steps) all_keys(n);
        } else {
          const bool more = ahead(n);
          if (n > 0 && n <= n_steps) softmax(n - 1);
          if (n > 1) values(n - 2);
          uint4v f[2][2];
          if (more) fold_weights(quarter_of(n), f);
          if (n + 1 < n_steps) convert(n + 1, now);
          if (more) fold_ahead(n, f);
        }
      }
    }
    lds_barrier();
  }

  // ---- partial results
  float* const halves = reinterpret_cast<float*>(lds + ld.v) + (VB == 2 ? 2 * vb0 + quarter : vb0) * NO * 256;  // O of the second halves of the tokens
  float2* const fin = reinterpret_cast<float2*>(lds + ld.p);               // [16 rows][blocks]: what the zero-points take off, the weights' maximum
  float* const tops = reinterpret_cast<float*>(lds + ld.p) + 2 * 16 * VB;  // the rows' maxima: those of the first member, which may differ from the others'
  const size_t slot = (size_t)seq * a.n_slots + chunk;
  if (half0 == 1)
#pragma unroll
    for (int u = 0; u < NO; ++u) *reinterpret_cast<float4v*>(halves + (u * 64 + lane) * 4) = O[u];
#pragma unroll
  for (int r = 0; r < NQ; ++r) {
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      if (member + PARTS * i >= CB) break;
      const float z = sum_of_wave(z_sum[r][i]);
      if (lane == 0) fin[(hw * NQ + r) * VB + member + PARTS * i] = make_float2(z, blk_max[r][i]);
    }
    if (member > 0) continue;
    const float sum = sum_of_wave(run_sum[r]);
    if (lane == 0) tops[hw * NQ + r] = run_max[r];
    if (lane == 0 && hw < nh && r < nr)
      reinterpret_cast<float2*>(a.ml_part)[(slot * m.n_heads + h0 + hw) * m.qpk + row0 + r] = make_float2(run_max[r], sum);
  }
  lds_barrier();
  const int vb = vb0;
  if (vb < CB && half0 == 0) {
#pragma unroll
    for (int u = 0; u < NO; ++u) O[u] += *reinterpret_cast<const float4v*>(halves + (u * 64 + lane) * 4);
    const int vg = 128 * vb / rv;              // the columns' group in the unit
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[NO];
#pragma unroll
      for (int u = 0; u < NO; ++u) {
        y[u] = O[u][e];
        y[u] += __shfl_xor(y[u], 16 * NQ);
      }
      const int row = 4 * kg + e, h = row / NQ, r = row % NQ;
      if (h >= nh || h >= HEADS || r >= nr || kg >= NQ || (un.n_groups() > 1 && h / per_group != vg)) continue;
      const float2 f = fin[row * VB + vb];
      const float worth = (tops[row] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(f.y - tops[row])) / kWeightScale;
#pragma unroll
      for (int u = 0; u < NO; ++u) y[u] = (y[u] * (u & 1 ? 0.0625f : 1.f) - f.x) * worth;
      const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
      float* const o = a.o_part + slot * a.o_stride + (size_t)m.qpk * ohead + (size_t)(row0 + r) * rv + 128 * vb - vg * rv + 8 * col + 4 * quarter;
#pragma unroll
      for (int u = 0; u < NO; u += 4) *reinterpret_cast<float4v*>(o + u) = float4v{y[u], y[u + 1], y[u + 2], y[u + 3]};
    }
  }
}

namespace {
template <typename T, int NQ, int VB> PagedQFn pick(const PagedQForm& f) {
  if (f.slices == 2) return pagedq_kernel<T, 8, 2, NQ, 4, VB>;
  if (f.ks == 8) return pagedq_kernel<T, 8, 1, NQ, 2, VB>;
  return f.k_blocks == 2 ? pagedq_kernel<T, 4, 1, NQ, 2, VB> : pagedq_kernel<T, 4, 1, NQ, 1, VB>;
}
template <typename T, int NQ> PagedQFn pick(const PagedQForm& f) { return f.v_blocks == 2 ? pick<T, NQ, 2>(f) : pick<T, NQ, 4>(f); }
}  // namespace

// (every number of rows is a translation unit of its own)
template <> PagedQFn pagedq_rows_form<PALU_PAGEDQ_ROWS>(int act, const PagedQForm& f) {
  return act == PALU_F16 ? pick<F16, PALU_PAGEDQ_ROWS>(f) : pick<BF16, PALU_PAGEDQ_ROWS>(f);
}

}  // namespace palu
