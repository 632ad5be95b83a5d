// Decode attention over a paged latent cache: a sliding window with a few first rows (sinks), and a prefix that the
// sequences of a batch share.
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v
//
// One workgroup takes a unit (up to four key/value heads of one group, NH) and a run of tiles of 64 tokens, for up to
// 16 * PT packed query rows (heads x rows).  Per tile:
//   keys    a wavefront rebuilds its head's (its FQ-th of the features of) keys of 16 tokens at a time, K^T = B_k^T H_k^T,
//           with the weights resident in registers and the latents in LDS (staged one tile ahead), rotates them in
//           float32 and multiplies by the rotated queries on the matrix cores; the partial scores over its features
//           go to LDS.
//   softmax eight threads per row add the partial scores, mask, and keep the running maximum and sum in float32.
//   values  every wavefront contracts the probabilities of all rows with its 32 columns of the value latents, which it
//           holds in registers since the tile began (one load per row and lane, two columns: the transposition that
//           the matrix operand wants is a byte permute).
// Partial results (unnormalised sums, maxima, row sums) are merged, normalised and multiplied by B_v in paged_merge_kernel.
//
// Rotation.  The angle of position t0 + i is that of t0 plus that of i: cos and sin of i < 16 lie in LDS for good and
// those of each 16 tokens' first position are fetched from the table a tile ahead (512 bytes), instead of 512 bytes per
// token.  Two products of numbers that are right to 1e-7.
// Rounding.  The matrix instructions take 16-bit operands.  A float16 layer's output is rounded to 2^-11 relative, so
// the rotated keys, the queries and the probabilities enter as pairs of float16 numbers hi + lo (2^-21).  A bfloat16
// layer's output is rounded to 2^-8: keys and queries enter as one float16 number each (2^-11), probabilities as a pair
// of bfloat16 numbers.  Keys are scaled by 1/8 and the queries by 8 (exact): magnitudes up to 524032 stay in range.

#include "paged.h"

namespace palu {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));

namespace {

constexpr float kKeyScale = 0.125f;
constexpr int kAngPitch = 132;                 // floats per token of the LDS angles: 64 cos, 64 sin, 4 of padding (16 tokens on 16 x 4 banks)
constexpr int kScorePitch = 68;                // floats per row of scores; the row's probabilities take its place (hi, then lo)

template <typename T> __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c);
template <> __device__ __forceinline__ float4v mma<F16>(uint4v a, uint4v b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ float4v mma<BF16>(uint4v a, uint4v b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// two float32 numbers as a pair of 16-bit ones hi, and what the rounding left as another, lo
template <typename T> __device__ __forceinline__ uint32_t pack2(float x, float y);
template <> __device__ __forceinline__ uint32_t pack2<F16>(float x, float y) {
  return __builtin_bit_cast(uint32_t, half2v{(_Float16)x, (_Float16)y});
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <> __device__ __forceinline__ uint32_t pack2<BF16>(float x, float y) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}
template <typename T> __device__ __forceinline__ void split2(float x, float y, uint32_t* hi, uint32_t* lo) {
  uint32_t h = pack2<T>(x, y);
  asm("" : "+v"(h));           // lo has to be measured from these very bits: where x is a product, the compiler may round it to hi in one step and
  *hi = h;                     // take the conversion of the float32 product, another number now and then, for hi's value
  *lo = pack2<T>(x - T::to_float((uint16_t)h), y - T::to_float((uint16_t)(h >> 16)));
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 16 bytes per lane from g to LDS byte m0 + 16 * lane; counted by vmcnt, without a register
__device__ __forceinline__ void load_to_lds(const void* g, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(m0), "v"(g) : "memory");
}
__device__ __forceinline__ void wait_and_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();
}

}  // namespace

template <typename T, int NH, bool BIGK, int VB, int PT, bool SHARED>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_kernel(PagedArgs a) {
  constexpr bool PAIR = __is_same(T, F16);     // queries and keys as pairs hi + lo
  constexpr int FQ = BIGK ? 4 : 2;             // the 128 features of a head go to this many wavefronts
  constexpr int FT = 8 / FQ;                   // tiles of 16 features per wavefront: low halves of the rotation pairs, then high halves
  constexpr int TS = 8 / (NH * FQ);            // ... and the tokens of a tile to this many
  constexpr int TPW = 4 / TS;                  // sub-tiles of 16 tokens per wavefront
  constexpr int KSM = BIGK ? 16 : 8;           // steps of 32 latent channels, at most
  constexpr int NK = FQ == 2 ? 2 : 1;          // contraction steps of 32 features per wavefront
  constexpr int NRT = PT > NH ? PT / NH : 1;   // tiles of 16 query rows per head
  constexpr int NBUF = BIGK ? 1 : 2;
  constexpr int HROW = BIGK ? 1024 : 512;      // bytes of LDS per token, at most
  constexpr int ROWS = 16 * PT;
  static_assert(NH * FQ * TS == 8, "eight wavefronts");

  __shared__ __attribute__((aligned(16))) unsigned char Hs[NBUF][kPagedTile * HROW];
  __shared__ __attribute__((aligned(16))) unsigned char Qs[NH * NRT * FQ * NK * (PAIR ? 2 : 1) * 1024];
  __shared__ __attribute__((aligned(16))) float Ang[16 * kAngPitch];
  __shared__ __attribute__((aligned(16))) float Base[2][4][kDHead];
  __shared__ __attribute__((aligned(16))) float Sc[FQ][ROWS * kScorePitch];
  __shared__ __attribute__((aligned(16))) float Al[ROWS];
  __shared__ __attribute__((aligned(16))) int Row[4][kPagedTile];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, kg = lane >> 4;

  // ---- what this workgroup does
  const int bid = blockIdx.x;
  const PagedUnit un = a.units[bid % a.n_units];
  int rest = bid / a.n_units;
  const int rb = rest % a.n_row_blocks;
  rest /= a.n_row_blocks;
  const int seq = SHARED ? 0 : rest / a.n_slots;
  const int chunk = SHARED ? rest : rest % a.n_slots;
  int L = SHARED ? a.max_len : (a.seq_lens ? a.seq_lens[seq] : a.max_len);
  L = max(0, min(L, a.max_len));
  const PagedSpan span = paged_span(L, a.first, a.window, a.n_sink);
  const int n_chunks = (span.n_tiles + a.chunk_tiles - 1) / a.chunk_tiles;
  if (chunk >= n_chunks) return;
  const int i0 = (int)((long long)span.n_tiles * chunk / n_chunks), i1 = (int)((long long)span.n_tiles * (chunk + 1) / n_chunks);

  const PagedMeta& m = a.meta;
  const int g = un.group(), nh = un.nh(), h0 = un.h0();
  const int rk = m.k_off[g + 1] - m.k_off[g], rv = m.v_off[g + 1] - m.v_off[g];
  const int nks = rk / 32;
  const int row0 = rb * a.block_rows;
  const int nr = min(a.block_rows, a.rows - row0);         // rows per head
  const int n_packed = nh * nr;

  const int hh = wave % NH, fq = wave / NH % FQ, ts = wave / (NH * FQ);
  const int fbase = (64 / FQ) * fq;                         // first rotation pair of this wavefront

  // position of tile i, and the row of the cache that its token holds (a masked one: that of the first attended token)
  auto tile_pos = [&](int i) { return kPagedTile * (i < span.sink_tiles ? i : span.tile0 + i - span.sink_tiles); };
  auto row_of = [&](int i, int x) __attribute__((always_inline)) {
    const int t0 = tile_pos(i);
    int t = t0 + x;
    const int head = t0 < span.sink ? t0 : max(t0, span.lo);
    if (t >= L || (t >= span.sink && t < span.lo)) t = head;
    int page = a.page_table[(size_t)seq * a.table_stride + (t >> a.page_shift)];
    page = max(0, min(page, a.n_pages - 1));
    return (page << a.page_shift) + (t & ((1 << a.page_shift) - 1));
  };
  auto base_of = [&](int i, int x) __attribute__((always_inline)) {   // x: sub-tile * 128 + (cos | sin) * 64 + pair
    const int p = min(tile_pos(i) + 16 * (x >> 7), a.rope_len - 1);
    return a.rope[rope_f32_index(p, x & 63, (x >> 6) & 1, kRopeTableStride)];
  };

  // latents of tile i into LDS: 16-byte piece p of token t at piece p ^ (t % 8), so that 8 tokens' same pieces lie on all banks
  const int pieces = (rk / 8 + 7) & ~7;                     // per token, rounded up to whole groups of 8
  const int n_ops = pieces / 8;                             // 64 * pieces / 512 threads
  const uint32_t inv = ((1u << 20) + pieces - 1) / pieces;
  const uint16_t* hk = a.hk + m.k_off[g];
  auto stage = [&](int i) __attribute__((always_inline)) {
    const int* rows = Row[i & 3];
    const uint32_t dst = lds_addr(Hs[NBUF == 2 ? i & 1 : 0]);
#pragma unroll
    for (int k = 0; k < KSM / 2; ++k) {
      if (k < n_ops) {
        const uint32_t id = (uint32_t)((wave * n_ops + k) * 64 + lane);
        const uint32_t t = (id * inv) >> 20;
        uint32_t p = (id - t * pieces) ^ (t & 7);
        if ((int)p * 8 >= rk) p = 0;
        load_to_lds(hk + (size_t)rows[t] * a.R_k + p * 8, __builtin_amdgcn_readfirstlane(dst + (wave * n_ops + k) * 1024));
      }
    }
  };

  // ---- prologue
  if (tid < 64) Row[i0 & 3][tid] = row_of(i0, tid);
  else if (tid < 128 && i0 + 1 < i1) Row[(i0 + 1) & 3][tid - 64] = row_of(i0 + 1, tid - 64);
  Base[i0 & 1][tid >> 7][tid & 127] = base_of(i0, tid);
  for (int x = tid; x < 16 * kDHead; x += kPagedThreads) {
    const int t = x & 15, c = x >> 4;
    Ang[t * kAngPitch + c] = kKeyScale * a.rope[rope_f32_index(t, c & 63, c >> 6, kRopeTableStride)];
  }
  // rotated queries, as operands of the score product: [head][row tile][feature part][step][hi | lo][lane] x 16 bytes
  for (int x = tid; x < n_packed * kHalf; x += kPagedThreads) {
    const int f = x & 63, pr = x >> 6;
    const int h = pr / nr, r = pr - h * nr;
    const int hq = (h0 + h) * m.qpk;
    int b = seq, qh = row0 + r;
    if (SHARED) { b = qh / m.qpk; qh -= b * m.qpk; }
    const uint16_t* qp = a.q + ((size_t)b * m.n_heads * m.qpk + hq + qh) * kDHead;
    const float x0 = T::to_float(qp[f]), x1 = T::to_float(qp[f + kHalf]);
    int pos = a.q_pos ? a.q_pos[b] : (a.seq_lens ? a.seq_lens[b] : a.pos_len) - 1;
    pos = max(0, min(pos, a.rope_len - 1));
    const float k = a.scale / kKeyScale;
    const float c = a.rope[rope_f32_index(pos, f, 0, kRopeTableStride)] * k, s = a.rope[rope_f32_index(pos, f, 1, kRopeTableStride)] * k;
    const float y0 = x0 * c - x1 * s, y1 = x1 * c + x0 * s;
    const int part = f / (64 / FQ), o = f % (64 / FQ);
    int ln, e0, e1, step1;
    if (FQ == 2) { ln = o >> 3; e0 = e1 = 4 * (o & 1) + ((o & 7) >> 1); step1 = 1; }
    else { ln = o >> 2; e0 = o & 3; e1 = 4 + e0; step1 = 0; }
    unsigned char* base = Qs + (size_t)((h * NRT + (r >> 4)) * FQ + part) * NK * (PAIR ? 2 : 1) * 1024 + (ln * 16 + (r & 15)) * 16;
    uint32_t hi, lo;
    split2<F16>(y0, y1, &hi, &lo);
    unsigned char* b1 = base + step1 * (PAIR ? 2 : 1) * 1024;
    *reinterpret_cast<uint16_t*>(base + 2 * e0) = (uint16_t)hi;
    *reinterpret_cast<uint16_t*>(b1 + 2 * e1) = (uint16_t)(hi >> 16);
    if (PAIR) {
      *reinterpret_cast<uint16_t*>(base + 1024 + 2 * e0) = (uint16_t)lo;
      *reinterpret_cast<uint16_t*>(b1 + 1024 + 2 * e1) = (uint16_t)(lo >> 16);
    }
  }
  __syncthreads();
  stage(i0);

  // weights: rows (features) of tile j at lane row m: FQ = 2: pair fbase + 2 m + j, low halves (tiles 0, 1) and high halves (2, 3);
  // FQ = 4: pair fbase + m (tiles 0 and 1).  Eight consecutive latent channels per lane.
  uint4v W[KSM][FT];
  const int width = (m.head_off[g + 1] - m.head_off[g]) * kDHead;
  {
    const uint16_t* B = a.Bk + m.bk_off[g] + (size_t)(h0 - m.head_off[g] + (hh < nh ? hh : 0)) * kDHead + fbase;
#pragma unroll
    for (int ks = 0; ks < KSM; ++ks) {
#pragma unroll
      for (int j = 0; j < FT; ++j) W[ks][j] = uint4v{0, 0, 0, 0};
      if (ks < nks) {
        const uint16_t* p = B + (size_t)(32 * ks + 8 * kg) * width;
#pragma unroll
        for (int side = 0; side < 2; ++side) {
          uint32_t v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t* q = p + (size_t)e * width + side * kHalf;
            v[e] = FQ == 2 ? *reinterpret_cast<const uint32_t*>(q + 2 * col) : (uint32_t)q[col];
          }
          if (FQ == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              W[ks][2 * side][i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x05040100u);
              W[ks][2 * side + 1][i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302u);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) W[ks][side][i] = v[2 * i] | (v[2 * i + 1] << 16);
          }
        }
      }
    }
  }

  // value columns of this wavefront: 32 per block; up to four blocks are taken by two wavefronts each, 32 tokens to either
  const int n_blocks = rv / 32;
  const bool halves = VB == 1 && n_blocks <= 4;
  const int vblock = halves ? wave & 3 : wave;
  const uint16_t* hv = a.hv + m.v_off[g] + vblock * 32 + 2 * col;

  float4v O[VB][PT][2];
#pragma unroll
  for (int v = 0; v < VB; ++v)
#pragma unroll
    for (int p = 0; p < PT; ++p) O[v][p][0] = O[v][p][1] = float4v{0, 0, 0, 0};
  const int n_pt = (n_packed + 15) / 16;

  // softmax state: thread (row, eighth); rows the row may see
  const int srow = tid >> 3, soct = tid & 7;
  float run_max = -INFINITY, run_sum = 0.f;
  int limit = L;
  if (SHARED && srow < n_packed) {
    const int b = (row0 + srow % nr) / m.qpk;
    limit = min(L, a.seq_lens ? a.seq_lens[b] : L);
  }
  wait_and_barrier();

  for (int i = i0; i < i1; ++i) {
    const int t0 = tile_pos(i);
    // requests: the next tile's latents, this tile's values, the angles and rows of later tiles
    if (NBUF == 2 && i + 1 < i1) stage(i + 1);
    uint32_t V[VB][2][8];
#pragma unroll
    for (int v = 0; v < VB; ++v) {
      if (vblock + 8 * v < n_blocks) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (!halves || k == (wave >> 2)) {
            const int4 r0 = *reinterpret_cast<const int4*>(&Row[i & 3][32 * k + 8 * kg]);
            const int4 r1 = *reinterpret_cast<const int4*>(&Row[i & 3][32 * k + 8 * kg + 4]);
            const int r[8] = {r0.x, r0.y, r0.z, r0.w, r1.x, r1.y, r1.z, r1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) V[v][k][e] = *reinterpret_cast<const uint32_t*>(hv + (size_t)r[e] * a.R_v + v * 256);
          }
        }
      }
    }
    float next_base = 0.f;
    int next_row = 0;
    if (i + 1 < i1) next_base = base_of(i + 1, tid);
    if (i + 2 < i1 && tid < 64) next_row = row_of(i + 2, tid);

    // ---- keys and scores
    if (hh < nh) {
      const unsigned char* H = Hs[NBUF == 2 ? i & 1 : 0];
      const int off0 = (kg ^ (lane & 7)) * 16, off1 = ((4 + kg) ^ (lane & 7)) * 16;
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        const int tt = ts * TPW + x;
        const unsigned char* hrow = H + (16 * tt + col) * pieces * 16;
        float4v acc[FT];
#pragma unroll
        for (int j = 0; j < FT; ++j) acc[j] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KSM; ++ks) {
          if (ks < nks) {
            const uint4v h = *reinterpret_cast<const uint4v*>(hrow + (ks >> 1) * 128 + ((ks & 1) ? off1 : off0));
#pragma unroll
            for (int j = 0; j < FT; ++j) acc[j] = mma<T>(W[ks][j], h, acc[j]);
          }
        }
        // rotate; lane: token col, pairs fbase + (FQ == 2 ? 8 kg + 2 i + j : 4 kg + i)
        constexpr int NP = 4 * NK;
        const float* ang = Ang + col * kAngPitch + fbase + NP * kg;
        const float* bas = &Base[i & 1][tt][fbase + NP * kg];
        uint32_t khi[NK][4], klo[NK][4];
        float lo[NP], hi[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const float c1 = ang[p], s1 = ang[p + kHalf], c0 = bas[p], s0 = bas[p + kHalf];
          const float c = c1 * c0 - s1 * s0, s = s1 * c0 + c1 * s0;
          const int j = FQ == 2 ? p & 1 : 0, e = FQ == 2 ? p >> 1 : p;
          const float kl = acc[j][e], kh = acc[FT / 2 + j][e];
          lo[FQ == 2 ? 4 * j + e : e] = kl * c - kh * s;
          hi[FQ == 2 ? 4 * j + e : e] = kh * c + kl * s;
        }
#pragma unroll
        for (int e = 0; e < NP; e += 2) {
          uint32_t x0, x1, y0, y1;
          if (PAIR) {
            split2<F16>(lo[e], lo[e + 1], &x0, &x1);
            split2<F16>(hi[e], hi[e + 1], &y0, &y1);
          } else {
            x0 = pack2<F16>(lo[e], lo[e + 1]);
            y0 = pack2<F16>(hi[e], hi[e + 1]);
            x1 = y1 = 0;
          }
          if (FQ == 2) { khi[0][e / 2] = x0; khi[NK - 1][e / 2] = y0; klo[0][e / 2] = x1; klo[NK - 1][e / 2] = y1; }
          else { khi[0][e / 2] = x0; khi[0][2 + e / 2] = y0; klo[0][e / 2] = x1; klo[0][2 + e / 2] = y1; }
        }
#pragma unroll
        for (int rt = 0; rt < NRT; ++rt) {
          if (rt * 16 < nr) {
            const unsigned char* qf = Qs + (size_t)((hh * NRT + rt) * FQ + fq) * NK * (PAIR ? 2 : 1) * 1024 + lane * 16;
            float4v s = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < NK; ++k) {
              const uint4v kh = {khi[k][0], khi[k][1], khi[k][2], khi[k][3]};
              const uint4v qh = *reinterpret_cast<const uint4v*>(qf + k * (PAIR ? 2 : 1) * 1024);
              s = mma<F16>(kh, qh, s);
              if (PAIR) {
                const uint4v kl = {klo[k][0], klo[k][1], klo[k][2], klo[k][3]};
                const uint4v ql = *reinterpret_cast<const uint4v*>(qf + (2 * k + 1) * 1024);
                s = mma<F16>(kh, ql, s);
                s = mma<F16>(kl, qh, s);
              }
            }
            const int r = rt * 16 + col;                   // lane: query row col, tokens 4 kg ..
            if (r < nr) *reinterpret_cast<float4v*>(&Sc[fq][(hh * nr + r) * kScorePitch + 16 * tt + 4 * kg]) = s;
          }
        }
      }
    }
    __syncthreads();

    // ---- softmax
    if (srow < n_packed) {
      float s[8];
      float* row = &Sc[0][srow * kScorePitch];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = row[8 * soct + e];
#pragma unroll
      for (int f = 1; f < FQ; ++f)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += Sc[f][srow * kScorePitch + 8 * soct + e];
      float top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = t0 + 8 * soct + e;
        if (t >= limit || (t >= span.sink && t < span.lo)) s[e] = -INFINITY;
        top = fmaxf(top, s[e]);
      }
      top = fmaxf(top, __shfl_xor(top, 1));
      top = fmaxf(top, __shfl_xor(top, 2));
      top = fmaxf(top, __shfl_xor(top, 4));
      const float now = fmaxf(run_max, top);
      const float zero = now == -INFINITY ? 0.f : now;       // no row seen yet: exp2(-inf) = 0 below
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
      // all eight threads of the row have read their scores (the maximum went through all of them)
      unsigned char* P = reinterpret_cast<unsigned char*>(row);
      *reinterpret_cast<uint4v*>(P + 16 * soct) = uint4v{ph[0], ph[1], ph[2], ph[3]};
      *reinterpret_cast<uint4v*>(P + 128 + 16 * soct) = uint4v{pl[0], pl[1], pl[2], pl[3]};
      if (soct == 0) Al[srow] = alpha;
    }
    if (NBUF == 1 && i + 1 < i1) stage(i + 1);
    if (i + 1 < i1) Base[(i + 1) & 1][tid >> 7][tid & 127] = next_base;
    if (i + 2 < i1 && tid < 64) Row[(i + 2) & 3][tid] = next_row;
    wait_and_barrier();

    // ---- values
#pragma unroll
    for (int v = 0; v < VB; ++v) {
      if (vblock + 8 * v < n_blocks) {
        uint4v Vf[2][2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            Vf[k][0][e] = __builtin_amdgcn_perm(V[v][k][2 * e + 1], V[v][k][2 * e], 0x05040100u);
            Vf[k][1][e] = __builtin_amdgcn_perm(V[v][k][2 * e + 1], V[v][k][2 * e], 0x07060302u);
          }
#pragma unroll
        for (int p = 0; p < PT; ++p) {
          if (p < n_pt) {
            const float4v al = *reinterpret_cast<const float4v*>(&Al[16 * p + 4 * kg]);
            O[v][p][0] *= al;
            O[v][p][1] *= al;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              if (!halves || k == (wave >> 2)) {
                const unsigned char* P = reinterpret_cast<const unsigned char*>(&Sc[0][(16 * p + col) * kScorePitch]) + 64 * k + 16 * kg;
                const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 128);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  O[v][p][j] = mma<T>(hi, Vf[k][j], O[v][p][j]);
                  O[v][p][j] = mma<T>(lo, Vf[k][j], O[v][p][j]);
                }
              }
            }
          }
        }
      }
    }
    // the scores of the next tile go where these probabilities lie
    __syncthreads();
  }

  // ---- partial results
  run_sum += __shfl_xor(run_sum, 1);
  run_sum += __shfl_xor(run_sum, 2);
  run_sum += __shfl_xor(run_sum, 4);
  const size_t slot = SHARED ? chunk : (size_t)seq * a.n_slots + chunk;
  if (srow < n_packed && soct == 0) {
    const int h = srow / nr, r = srow - h * nr;
    float2* ml = reinterpret_cast<float2*>(a.ml_part) + slot * m.n_heads * a.rows + (size_t)(h0 + h) * a.rows + row0 + r;
    *ml = make_float2(run_max, run_sum);
  }
  if (halves) {                                 // the two wavefronts of a column block add up
    float4v* X = reinterpret_cast<float4v*>(Hs[0]);
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (wave >= 4) X[((wave - 4) * PT * 2 + p * 2 + j) * 64 + lane] = O[0][p][j];
    __syncthreads();
    if (wave >= 4) return;
#pragma unroll
    for (int p = 0; p < PT; ++p)
#pragma unroll
      for (int j = 0; j < 2; ++j) O[0][p][j] += X[(wave * PT * 2 + p * 2 + j) * 64 + lane];
  }
#pragma unroll
  for (int v = 0; v < VB; ++v) {
    if (vblock + 8 * v >= n_blocks) continue;
#pragma unroll
    for (int p = 0; p < PT; ++p) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pr = 16 * p + 4 * kg + e;
        if (pr < n_packed) {
          const int h = pr / nr, r = pr - h * nr;
          const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
          float* o = a.o_part + slot * a.o_stride + (size_t)a.rows * ohead + (size_t)(row0 + r) * rv + (vblock + 8 * v) * 32 + 2 * col;
          *reinterpret_cast<float2*>(o) = make_float2(O[v][p][0][e], O[v][p][1][e]);
        }
      }
    }
  }
}

// Partial results of 16 rows (sequence, query head) of one key/value head: merged, normalised, split into pairs of 16-bit
// numbers hi + lo, and multiplied by the head's 128 columns of B_v.  grid (tiles of 16 rows, key/value heads), 256 threads;
// a wavefront makes 32 columns.
template <typename T>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedMergeArgs a) {
  constexpr int kMaxR = 512, kPitch = kMaxR + 8;
  __shared__ __attribute__((aligned(16))) uint16_t Oh[2][16 * kPitch];
  __shared__ float Part[256 * 4];
  __shared__ float Inv[16], Top[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, kg = lane >> 4;
  const PagedMeta& m = a.meta;
  const int h = blockIdx.y, g = m.group_of_head[h];
  const int rv = m.v_off[g + 1] - m.v_off[g];
  const int rows = a.batch * m.qpk, row0 = blockIdx.x * 16;
  const int n = min(16, rows - row0);
  const int ohead = m.o_off[g] + (h - m.head_off[g]) * rv;

  // where partial result s of row r lies: the sequence's own ones first, then those of the shared tokens
  auto own_slots = [&](int b) {
    int L = a.seq_lens ? a.seq_lens[b] : a.max_len;
    L = max(0, min(L, a.max_len));
    return (paged_span(L, a.first, a.window, a.n_sink).n_tiles + a.chunk_tiles - 1) / a.chunk_tiles;
  };
  auto ml_of = [&](int row, int b, int n_own, int s) {
    const float* p = s < n_own ? a.ml_part + (((size_t)(b * a.n_slots + s) * m.n_heads + h) * m.qpk + row - b * m.qpk) * 2
                               : a.ml_shared + (((size_t)(s - n_own) * m.n_heads + h) * rows + row) * 2;
    return *reinterpret_cast<const float2*>(p);
  };

  // maximum and sum of every row: 16 threads each
  {
    const int r = tid >> 4;
    float top = -INFINITY, sum = 0.f;
    if (r < n) {
      const int row = row0 + r, b = row / m.qpk, n_own = own_slots(b);
      for (int s = tid & 15; s < n_own + a.n_shared; s += 16) {
        const float2 x = ml_of(row, b, n_own, s);
        const float now = fmaxf(top, x.x);
        if (now > -INFINITY) sum = sum * __builtin_amdgcn_exp2f(top - now) + x.y * __builtin_amdgcn_exp2f(x.x - now);
        top = now;
      }
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
      const float t2 = __shfl_xor(top, d), s2 = __shfl_xor(sum, d), now = fmaxf(top, t2);
      if (now > -INFINITY) sum = sum * __builtin_amdgcn_exp2f(top - now) + s2 * __builtin_amdgcn_exp2f(t2 - now);
      top = now;
    }
    if ((tid & 15) == 0) {
      Top[r] = top;
      Inv[r] = sum == 0.f ? 0.f : 1.f / sum;
    }
  }
  __syncthreads();

  // weighted sums: thread (row, 4 columns, every n_parts-th partial result)
  const int quads = rv / 4;
  const int items = n * quads;
  const int n_parts = max(1, 256 / items);
  for (int x = tid; x < items * n_parts; x += 256) {
    const int part = x / items, y = x - part * items, r = y / quads, c = (y - r * quads) * 4;
    const int row = row0 + r, b = row / m.qpk, n_own = own_slots(b);
    const float top = Top[r];
    float4v o = {0, 0, 0, 0};
    for (int s = part; s < n_own + a.n_shared; s += n_parts) {
      const float2 ml = ml_of(row, b, n_own, s);
      if (ml.x == -INFINITY) continue;                      // saw no row
      const float w = __builtin_amdgcn_exp2f(ml.x - top);
      const float* p = s < n_own ? a.o_part + (size_t)(b * a.n_slots + s) * a.o_stride + (size_t)m.qpk * ohead + (size_t)(row - b * m.qpk) * rv + c
                                 : a.o_shared + (size_t)(s - n_own) * a.o_shared_stride + (size_t)rows * ohead + (size_t)row * rv + c;
      o += *reinterpret_cast<const float4v*>(p) * w;
    }
    if (n_parts > 1) {
      *reinterpret_cast<float4v*>(&Part[x * 4]) = o;
    } else {
      o *= Inv[r];
      uint2v hi, lo;
      split2<T>(o.x, o.y, &((uint32_t*)&hi)[0], &((uint32_t*)&lo)[0]);
      split2<T>(o.z, o.w, &((uint32_t*)&hi)[1], &((uint32_t*)&lo)[1]);
      *reinterpret_cast<uint2v*>(&Oh[0][r * kPitch + c]) = hi;
      *reinterpret_cast<uint2v*>(&Oh[1][r * kPitch + c]) = lo;
    }
  }
  if (n_parts > 1) {
    __syncthreads();
    if (tid < items) {
      const int r = tid / quads, c = (tid - r * quads) * 4;
      float4v o = {0, 0, 0, 0};
      for (int p = 0; p < n_parts; ++p) o += *reinterpret_cast<const float4v*>(&Part[(p * items + tid) * 4]);
      o *= Inv[r];
      uint2v hi, lo;
      split2<T>(o.x, o.y, &((uint32_t*)&hi)[0], &((uint32_t*)&lo)[0]);
      split2<T>(o.z, o.w, &((uint32_t*)&hi)[1], &((uint32_t*)&lo)[1]);
      *reinterpret_cast<uint2v*>(&Oh[0][r * kPitch + c]) = hi;
      *reinterpret_cast<uint2v*>(&Oh[1][r * kPitch + c]) = lo;
    }
  }
  __syncthreads();

  // times B_v: columns 32 wave + 2 col (+ 1)
  const int width = (m.head_off[g + 1] - m.head_off[g]) * kDHead;
  const uint16_t* B = a.Bv + m.bv_off[g] + (size_t)(h - m.head_off[g]) * kDHead + 32 * wave + 2 * col;
  float4v acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll 2
  for (int ks = 0; ks < rv / 32; ++ks) {
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const uint32_t*>(B + (size_t)(32 * ks + 8 * kg + e) * width);
    uint4v f0, f1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f0[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x05040100u);
      f1[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x07060302u);
    }
    const uint4v hi = *reinterpret_cast<const uint4v*>(&Oh[0][col * kPitch + 32 * ks + 8 * kg]);
    const uint4v lo = *reinterpret_cast<const uint4v*>(&Oh[1][col * kPitch + 32 * ks + 8 * kg]);
    acc[0] = mma<T>(hi, f0, acc[0]);
    acc[1] = mma<T>(hi, f1, acc[1]);
    acc[0] = mma<T>(lo, f0, acc[0]);
    acc[1] = mma<T>(lo, f1, acc[1]);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int r = 4 * kg + e;
    if (r < n) {
      const int row = row0 + r, b = row / m.qpk;
      uint16_t* o = a.out + ((size_t)b * m.n_heads * m.qpk + h * m.qpk + row - b * m.qpk) * kDHead + 32 * wave + 2 * col;
      *reinterpret_cast<uint32_t*>(o) = pack2<T>(acc[0][e], acc[1][e]);
    }
  }
}

namespace {
template <typename T, int NH, bool BIGK, int PT, bool SHARED>
PagedFn pick_v(bool big_v) {
  return big_v ? paged_kernel<T, NH, BIGK, 2, PT, SHARED> : paged_kernel<T, NH, BIGK, 1, PT, SHARED>;
}
template <typename T, bool SHARED>
PagedFn pick(int nh, bool big_k, bool big_v, int pt) {
  if (big_k) {
    if (nh == 2) return pt == 1 ? pick_v<T, 2, true, 1, SHARED>(big_v) : pick_v<T, 2, true, 2, SHARED>(big_v);
    return pt == 1 ? pick_v<T, 1, true, 1, SHARED>(big_v) : pick_v<T, 1, true, 2, SHARED>(big_v);
  }
  if (nh == 4) return pt == 1 ? pick_v<T, 4, false, 1, SHARED>(big_v) : pick_v<T, 4, false, 4, SHARED>(big_v);
  if (nh == 2) return pt == 1 ? pick_v<T, 2, false, 1, SHARED>(big_v) : pick_v<T, 2, false, 4, SHARED>(big_v);
  return pt == 1 ? pick_v<T, 1, false, 1, SHARED>(big_v) : pick_v<T, 1, false, 4, SHARED>(big_v);
}
}  // namespace

PagedFn paged_fn(int act, int nh, bool big_k, bool big_v, int pt, bool shared) {
  if (act == PALU_F16) return shared ? pick<F16, true>(nh, big_k, big_v, pt) : pick<F16, false>(nh, big_k, big_v, pt);
  return shared ? pick<BF16, true>(nh, big_k, big_v, pt) : pick<BF16, false>(nh, big_k, big_v, pt);
}
PagedMergeFn paged_merge_fn(int act) {
  return act == PALU_F16 ? paged_merge_kernel<F16> : paged_merge_kernel<BF16>;
}

}  // namespace palu
