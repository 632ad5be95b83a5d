// Decode attention over a paged latent cache: a sliding window with a few first rows (sinks), and a prefix that the
// sequences of a batch share.
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v
//
// One workgroup of eight wavefronts takes a unit (up to NH key/value heads) and a run of tiles of 32 tokens, for up to
// 16 * PT packed query rows (heads x rows).  Per tile:
//   keys    a wavefront rebuilds its FQ-th of its head's features for 16 tokens at a time, K^T = B_k^T H_k^T, with the
//           weights resident in registers, rotates them in float32 and multiplies by the rotated queries on the matrix
//           cores; the partial scores over its features go to LDS.
//   softmax four threads per row add the partial scores, mask, and keep the running maximum and sum in float32.
//   values  every wavefront contracts the probabilities of all rows with its 32 columns of the value latents (read as two
//           columns of eight tokens per lane: the transposition that the matrix operand wants is a byte permute).
// Few rows (pipelined): the three run in one interval on three consecutive tiles, keys of tile n, softmax of n - 1,
// values of n - 2, with one barrier per tile.  Many rows: keys of n and values of n - 1, barrier, softmax of n, barrier.
// Latents, page-table entries and angles come by loads that write to LDS directly, n_stages - 1 tiles ahead, counted
// and never drained while tiles follow: what bounds these kernels with few rows is the cache's traffic, and 5.3 TB/s
// at 2 us latency take 40 KB in flight per compute unit.
// Partial results (unnormalised sums, maxima, row sums) are merged, normalised and multiplied by B_v in paged_merge_kernel.
//
// Rotation.  The angle of position t0 + i is that of t0 plus that of i: cos and sin of i < 16 stay in registers (or LDS)
// and those of each 16 tokens' first position are fetched from the table (512 bytes), instead of 512 bytes per token.
// Products of numbers that are right to 1e-7.
// Rounding.  The matrix instructions take 16-bit operands.  A float16 layer's output is rounded to 2^-11 relative, so
// the rotated keys, the queries and the probabilities enter as pairs of float16 numbers hi + lo (2^-21).  A bfloat16
// layer's output is rounded to 2^-8: keys and queries enter as one float16 number each (2^-11), probabilities as a pair
// of bfloat16 numbers.  Keys are scaled by 1/8 and the queries by 8 (exact): magnitudes up to 524032 stay in range.

#include "paged.h"

namespace palu {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));

namespace {

constexpr float kKeyScale = 0.125f;
template <int N> struct IntC { static constexpr int value = N; };

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
// 16 (4) bytes per lane from g to LDS byte m0 + 16 (4) * lane; counted by vmcnt, without a register
__device__ __forceinline__ void load_to_lds(const void* g, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(m0), "v"(g) : "memory");
}
__device__ __forceinline__ void load_to_lds4(const void* g, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(m0), "v"(g) : "memory");
}
// waits until at most n (rounded down to what is listed) of this wavefront's vector-memory operations are outstanding
__device__ __forceinline__ void wait_vm(int n) {
  if (n >= 24) asm volatile("s_waitcnt vmcnt(24)" ::: "memory");
  else if (n >= 20) asm volatile("s_waitcnt vmcnt(20)" ::: "memory");
  else if (n >= 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
  else if (n >= 12) asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
  else if (n >= 10) asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
  else if (n >= 8) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  else if (n >= 6) asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
  else if (n == 5) asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
  else if (n == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
  else if (n == 3) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
  else if (n == 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
  else if (n == 1) asm volatile("s_waitcnt vmcnt(1)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
// This wavefront's LDS operations are done, and so are the other wavefronts'; loads to LDS go on.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace

template <typename T, int NH, int FQ, int PT, int VB>
__global__ __launch_bounds__(kPagedThreads, 2) void paged_kernel(PagedArgs a) {
  constexpr bool PAIR = __is_same(T, F16);     // queries and keys as pairs hi + lo
  constexpr bool PIPE = PT == 1 && FQ == 2;    // one interval per tile; else two
  constexpr int FT = 8 / FQ;                   // tiles of 16 features per wavefront: low halves of the rotation pairs, then high halves
  constexpr int TS = 8 / (NH * FQ);            // the sub-tiles (16 tokens) of a tile go to this many wavefronts
  constexpr int SUB = kPagedTile / 16;
  constexpr int TPW = SUB / TS;                // sub-tiles per wavefront
  constexpr int KSM = 4 * FQ;                  // steps of 32 latent channels, at most
  constexpr int NK = FQ == 2 ? 2 : 1;          // contraction steps of 32 features per wavefront
  constexpr int NP = 4 * NK;                   // rotation pairs per lane
  constexpr int HL = PAIR ? 2 : 1;
  constexpr int NRT = PT > NH ? PT / NH : 1;   // tiles of 16 query rows per head
  constexpr int VLAG = PIPE ? 2 : 1;           // a tile's values are contracted so many intervals behind its keys
  static_assert(NH * FQ * TS == 8 && TS <= SUB, "eight wavefronts");

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
  const int k_cols = un.n_groups() * rk, v_cols = un.n_groups() * rv;
  const int nks = rk / 32;
  const int row0 = rb * a.block_rows;
  const int nr = min(a.block_rows, a.rows - row0);           // rows per head
  const int n_packed = nh * nr;
  const int NB = a.n_stages;
  const PagedLds ld = paged_lds(k_cols, v_cols, n_packed, PT, FQ, PAIR, PIPE, !PIPE, NB);
  const uint32_t lds0 = lds_addr(lds);

  const int hh = wave % NH, fq = wave / NH % FQ, ts = wave / (NH * FQ);
  const int fbase = (64 / FQ) * fq;                          // first rotation pair of this wavefront
  const bool works = hh < nh;
  const int hg = un.n_groups() > 1 ? (works ? hh : 0) / per_group : 0;   // the head's group inside the unit

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

  // ---- requests of interval n: keys and angles of tile n + NB - 1, values of n - VLAG + NB - 1, entries of n + E.
  // 16-byte piece p of a key row goes to piece p ^ (t % 8) (eight tokens' same pieces lie on all banks), of a value row to
  // p ^ 4 (t / 8) (the four tokens that a lane group reads at a time do).
  const uint32_t inv_k = ((1u << 20) + ld.k_pieces - 1) / ld.k_pieces, inv_v = ((1u << 20) + ld.v_pieces - 1) / ld.v_pieces;
  const int ops_k = ld.k_pieces / 2, ops_v = ld.v_pieces / 2;   // of 64 pieces, dealt out to the wavefronts
  const uint16_t* hk = a.hk + m.k_off[g];
  const uint16_t* hv = a.hv + m.v_off[g];
  const int* entries = reinterpret_cast<const int*>(lds + ld.entries);
  auto request = [&](int n) __attribute__((always_inline)) {
    const int jk = n + NB - 1, jv = n - VLAG + NB - 1, je = n + E;
    if (jk < i1) {
      const int t0 = tile_pos(jk);
      const int slot = jk % NB;
      const int* ent = entries + (jk % kPagedEntrySlots) * kPagedTile;
#pragma unroll
      for (int k = 0; k < KSM / 4; ++k) {
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
  float ang_c[NP], ang_s[NP];
  if (PIPE) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      ang_c[p] = kKeyScale * a.rope[rope_f32_index(col, fbase + NP * kg + p, 0, kRopeTableStride)];
      ang_s[p] = kKeyScale * a.rope[rope_f32_index(col, fbase + NP * kg + p, 1, kRopeTableStride)];
    }
  } else {
    float* ang = reinterpret_cast<float*>(lds + ld.ang);
    for (int x = tid; x < 16 * kDHead; x += kPagedThreads) {
      const int t = x & 15, c = x >> 4;
      ang[t * kPagedAngPitch + c] = kKeyScale * a.rope[rope_f32_index(t, c & 63, c >> 6, kRopeTableStride)];
    }
  }
  // rotated queries: [packed row][feature part][step][hi | lo][lane group] x 16 bytes
  for (int x = tid; x < n_packed * kHalf; x += kPagedThreads) {
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
    const int part = f / (64 / FQ), o = f % (64 / FQ);
    int ln, e0, e1, step1;
    if (FQ == 2) { ln = o >> 3; e0 = e1 = 4 * (o & 1) + ((o & 7) >> 1); step1 = 1; }
    else { ln = o >> 2; e0 = o & 3; e1 = 4 + e0; step1 = 0; }
    unsigned char* base = lds + ld.q + pr * ld.q_pitch + (part * NK * HL * 4 + ln) * 16;
    uint32_t hi, lo;
    split2<F16>(y0, y1, &hi, &lo);
    unsigned char* b1 = base + step1 * HL * 64;
    *reinterpret_cast<uint16_t*>(base + 2 * e0) = (uint16_t)hi;
    *reinterpret_cast<uint16_t*>(b1 + 2 * e1) = (uint16_t)(hi >> 16);
    if (PAIR) {
      *reinterpret_cast<uint16_t*>(base + 64 + 2 * e0) = (uint16_t)lo;
      *reinterpret_cast<uint16_t*>(b1 + 64 + 2 * e1) = (uint16_t)(lo >> 16);
    }
  }

  // weights: rows (features) of tile j at lane row m: FQ = 2: pair fbase + 2 m + j, low halves (tiles 0, 1) and high halves (2, 3);
  // FQ = 4: pair fbase + m (tiles 0 and 1).  Eight consecutive latent channels per lane.
  uint4v W[KSM][FT];
  {
    const int width = per_group * kDHead;
    const uint16_t* B = a.Bk + m.bk_off[g] + (size_t)hg * rk * width + (size_t)((works ? hh : 0) + h0 - m.head_off[g] - hg * per_group) * kDHead + fbase;
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

  const int n_blocks = v_cols / 32;                          // of 32 value columns, one (VB) per wavefront
  const int n_pt = (n_packed + 15) / 16;
  float4v O[VB][PT][2];
#pragma unroll
  for (int v = 0; v < VB; ++v)
#pragma unroll
    for (int p = 0; p < PT; ++p) O[v][p][0] = O[v][p][1] = float4v{0, 0, 0, 0};

  // softmax state of thread (row, quarter); rows the row may see
  const int srow = tid >> 2, squart = tid & 3;
  float run_max = -INFINITY, run_sum = 0.f;
  int limit = L;
  if (shared && srow < n_packed) limit = min(L, a.seq_lens ? a.seq_lens[(row0 + srow % nr) / m.qpk] : L);

  wait_vm(0);
  lds_barrier();

  // queries of a pipelined form stay in registers
  uint4v Q[PIPE ? NK * HL : 1];
  auto query = [&](int rt, int k, int hl) __attribute__((always_inline)) {
    const int r = hh * nr + min(rt * 16 + col, nr - 1);
    return *reinterpret_cast<const uint4v*>(lds + ld.q + r * ld.q_pitch + (((fq * NK + k) * HL + hl) * 4 + kg) * 16);
  };
  if (PIPE && works) {
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int hl = 0; hl < HL; ++hl) Q[k * HL + hl] = query(0, k, hl);
  }

  // ---- keys of tile n and their scores, KS > 0: rank 32 KS
  auto keys = [&](int n, auto ks_const) __attribute__((always_inline)) {
    constexpr int KS = decltype(ks_const)::value;
    const int slot = n % NB;
    const unsigned char* H = lds + ld.k + slot * ld.stage_k + (hg * rk / 64) * 128;
    const int off0 = (kg ^ (lane & 7)) * 16, off1 = ((4 + kg) ^ (lane & 7)) * 16;
    float* Sc = reinterpret_cast<float*>(lds + ld.s) + ((PIPE ? (n & 1) * FQ : 0) + fq) * (PT * 16 * kPagedScorePitch);
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      const int tt = ts * TPW + x;
      const unsigned char* hrow = H + (16 * tt + col) * ld.k_pieces * 16;
      float4v acc[FT];
#pragma unroll
      for (int j = 0; j < FT; ++j) acc[j] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < (KS ? KS : KSM); ++ks) {
        if (KS || ks < nks) {
          const uint4v h = *reinterpret_cast<const uint4v*>(hrow + (ks >> 1) * 128 + ((ks & 1) ? off1 : off0));
#pragma unroll
          for (int j = 0; j < FT; ++j) acc[j] = mma<T>(W[ks][j], h, acc[j]);
        }
      }
      // rotate; lane: token col, pairs fbase + (FQ == 2 ? 8 kg + 2 i + j : 4 kg + i)
      const float* bas = reinterpret_cast<const float*>(lds + ld.base) + (slot * SUB + tt) * kDHead + fbase + NP * kg;
      const float* ang = reinterpret_cast<const float*>(lds + ld.ang) + col * kPagedAngPitch + fbase + NP * kg;
      uint32_t khi[NK][4], klo[NK][4];
      float lo[NP], hi[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const float c1 = PIPE ? ang_c[p] : ang[p], s1 = PIPE ? ang_s[p] : ang[p + kHalf], c0 = bas[p], s0 = bas[p + kHalf];
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
          float4v s = {0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < NK; ++k) {
            const uint4v kh = {khi[k][0], khi[k][1], khi[k][2], khi[k][3]};
            const uint4v qh = PIPE ? Q[k * HL] : query(rt, k, 0);
            s = mma<F16>(kh, qh, s);
            if (PAIR) {
              const uint4v kl = {klo[k][0], klo[k][1], klo[k][2], klo[k][3]};
              const uint4v ql = PIPE ? Q[k * HL + HL - 1] : query(rt, k, HL - 1);
              s = mma<F16>(kh, ql, s);
              s = mma<F16>(kl, qh, s);
            }
          }
          const int r = rt * 16 + col;                       // lane: query row col, tokens 4 kg ..
          if (r < nr) *reinterpret_cast<float4v*>(&Sc[(hh * nr + r) * kPagedScorePitch + 16 * tt + 4 * kg]) = s;
        }
      }
    }
  };

  // ---- softmax of tile n
  auto softmax = [&](int n) __attribute__((always_inline)) {
    if (srow >= n_packed) return;
    const int buf = PIPE ? n & 1 : 0;
    const int t0 = tile_pos(n) + 8 * squart;
    const float* row = reinterpret_cast<const float*>(lds + ld.s) + buf * FQ * (PT * 16 * kPagedScorePitch) + srow * kPagedScorePitch + 8 * squart;
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = row[e];
#pragma unroll
    for (int f = 1; f < FQ; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += row[f * (PT * 16 * kPagedScorePitch) + e];
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
    unsigned char* P = lds + ld.p + buf * (PT * 16 * kPagedProbPitch) + srow * kPagedProbPitch + 16 * squart;
    *reinterpret_cast<uint4v*>(P) = uint4v{ph[0], ph[1], ph[2], ph[3]};
    *reinterpret_cast<uint4v*>(P + 64) = uint4v{pl[0], pl[1], pl[2], pl[3]};
    if (squart == 0) reinterpret_cast<float*>(lds + ld.alpha)[buf * PT * 16 + srow] = alpha;
  };

  // ---- values of tile n
  auto values = [&](int n) __attribute__((always_inline)) {
    const int buf = PIPE ? n & 1 : 0;
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
#pragma unroll
        for (int p = 0; p < PT; ++p) {
          if (p < n_pt) {
            const float4v al = *reinterpret_cast<const float4v*>(lds + ld.alpha + (buf * PT * 16 + 16 * p + 4 * kg) * 4);
            const unsigned char* P = lds + ld.p + (buf * PT * 16 + 16 * p + col) * kPagedProbPitch + 16 * kg;
            const uint4v hi = *reinterpret_cast<const uint4v*>(P), lo = *reinterpret_cast<const uint4v*>(P + 64);
            O[v][p][0] = mma<T>(hi, f0, O[v][p][0] * al);
            O[v][p][1] = mma<T>(hi, f1, O[v][p][1] * al);
            O[v][p][0] = mma<T>(lo, f0, O[v][p][0]);
            O[v][p][1] = mma<T>(lo, f1, O[v][p][1]);
          }
        }
      }
    }
  };

  for (int n = i0; n < i1 + VLAG; ++n) {
    request(n);
    if (PIPE && n > i0 && n <= i1 && wave == 0) softmax(n - 1);
    if (n - VLAG >= i0) values(n - VLAG);
    if (n < i1 && works) {
      if (nks == 8) keys(n, IntC<8>());
      else if (nks == 4) keys(n, IntC<4>());
      else if (nks == 2) keys(n, IntC<2>());
      else keys(n, IntC<0>());
    }
    if (!PIPE) {
      lds_barrier();
      if (n < i1) softmax(n);
    }
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
    const int bg = block * 32 / rv;                          // the group whose columns these are
    const int c = block * 32 - bg * rv + 2 * col;
#pragma unroll
    for (int p = 0; p < PT; ++p) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pr = 16 * p + 4 * kg + e;
        if (pr < n_packed) {
          const int h = pr / nr, r = pr - h * nr;
          if (un.n_groups() > 1 && h / per_group != bg) continue;
          const int ohead = m.o_off[g] + (h0 + h - m.head_off[g]) * rv;
          float* o = a.o_part + slot * a.o_stride + (size_t)a.rows * ohead + (size_t)(row0 + r) * rv + c;
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
template <typename T>
PagedFn pick(const PagedForm& f) {
  if (f.fq == 4) return f.vb == 1 ? paged_kernel<T, 2, 4, 1, 1> : paged_kernel<T, 2, 4, 1, 2>;
  if (f.nh == 4) {
    if (f.pt == 1) return f.vb == 1 ? paged_kernel<T, 4, 2, 1, 1> : paged_kernel<T, 4, 2, 1, 2>;
    return f.vb == 1 ? paged_kernel<T, 4, 2, 4, 1> : paged_kernel<T, 4, 2, 2, 2>;
  }
  if (f.pt == 1) return f.vb == 1 ? paged_kernel<T, 2, 2, 1, 1> : paged_kernel<T, 2, 2, 1, 2>;
  return f.vb == 1 ? paged_kernel<T, 2, 2, 4, 1> : paged_kernel<T, 2, 2, 2, 2>;
}
}  // namespace

PagedFn paged_fn(int act, const PagedForm& f) { return act == PALU_F16 ? pick<F16>(f) : pick<BF16>(f); }
PagedMergeFn paged_merge_fn(int act) {
  return act == PALU_F16 ? paged_merge_kernel<F16> : paged_merge_kernel<BF16>;
}

}  // namespace palu
