// Device-side helpers of the kernels for attention over a paged latent cache.
#pragma once

#include "paged.h"

namespace palu {

namespace {

constexpr float kKeyScale = 0.125f;
// Probabilities, exp2(score - running maximum) <= 1, are held times this (so are their sums and those of the latents, whose quotient is
// what counts): a pair of float16 numbers has steps of 2^-24, so that those of rows that one row outweighs are right to 2^-40 of the
// largest and not to 2^-25, which was 4 % of e^-14.  bfloat16 pairs are as exact at any size.
template <typename T> constexpr float kProbScale = __is_same(T, F16) ? 32768.f : 1.f;
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
// x less the 16-bit number in the low half of h.  As a multiply-add it takes a float16 operand as it is.
template <typename T> __device__ __forceinline__ float less(float x, uint32_t h, float minus_one = -1.f) {
  return __builtin_fmaf(T::to_float((uint16_t)h), minus_one, x);
}
template <typename T> __device__ __forceinline__ void split2(float x, float y, uint32_t* hi, uint32_t* lo) {
  uint32_t h = pack2<T>(x, y);
  asm("" : "+v"(h));           // lo has to be measured from these very bits: where x is a product, the compiler may round it to hi in one step and
  *hi = h;                     // take the conversion of the float32 product, another number now and then, for hi's value
  *lo = pack2<T>(less<T>(x, h), less<T>(y, h >> 16));
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
// Waits until at most n of this wavefront's vector-memory operations are outstanding, or fewer: 16, 8, 4, 2 or none.  (A branch for every
// number took 400 cycles a tile.)
__device__ __forceinline__ void wait_vm(int n) {
  if (n >= 8) {
    if (n >= 16) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
  } else {
    if (n >= 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else if (n >= 2) asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
}
// the larger of x over 8 lanes
template <int CTRL> __device__ __forceinline__ float max_with(float x) {
  const int u = __builtin_bit_cast(int, x);
  return fmaxf(x, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float max_of_8(float x) {           // lane ^ 1, ^ 2 in a quad, mirrored in 8 lanes
  return max_with<0x141>(max_with<0x4E>(max_with<0xB1>(x)));
}
// This wavefront's LDS operations are done, and so are the other wavefronts'; loads to LDS go on.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// What a workgroup does.
struct PagedWork {
  const PagedArgs& a;
  const PagedPart t;
  PagedUnit un;
  bool shared;
  int rb, seq, chunk, L;
  PagedSpan span;
  int i0, i1;                                  // its tiles
  int g, nh, h0, rk, rv, per_group, k_cols, v_cols;
  int row0, nr, n_packed;                      // query rows per head and in all

  __device__ __forceinline__ PagedWork(const PagedArgs& args) : a(args), t((int)blockIdx.x < args.n_first ? args.part[0] : args.part[1]) {
    const int bid = (int)blockIdx.x >= a.n_first ? blockIdx.x - a.n_first : blockIdx.x;
    un = a.units[bid % a.n_units];
    int rest = bid / a.n_units;
    rb = rest % t.n_row_blocks;
    rest /= t.n_row_blocks;
    shared = t.shared != 0;
    seq = shared ? 0 : rest / t.n_slots;
    chunk = rest - seq * t.n_slots;
    L = shared || !a.seq_lens ? t.max_len : a.seq_lens[seq];
    L = __builtin_amdgcn_readfirstlane(max(0, min(L, t.max_len)));
    span = paged_span(L, t.first, t.window, t.n_sink);
    const int n_chunks = (span.n_tiles + t.chunk_tiles - 1) / t.chunk_tiles;
    i0 = i1 = 0;
    if (chunk >= n_chunks) return;
    i0 = (int)((long long)span.n_tiles * chunk / n_chunks);
    i1 = (int)((long long)span.n_tiles * (chunk + 1) / n_chunks);
    const PagedMeta& m = a.meta;
    g = un.group();
    nh = un.nh();
    h0 = un.h0();
    rk = m.k_off[g + 1] - m.k_off[g];
    rv = m.v_off[g + 1] - m.v_off[g];
    per_group = m.head_off[g + 1] - m.head_off[g];           // a unit of several groups takes whole ones
    k_cols = un.n_groups() * rk;
    v_cols = un.n_groups() * rv;
    row0 = rb * t.block_rows;
    nr = min(t.block_rows, t.rows - row0);
    n_packed = nh * nr;
  }
  __device__ __forceinline__ bool idle() const { return i0 >= i1; }
  // position of tile i, and the position whose row its token x reads (a masked token: the first attended one's)
  __device__ __forceinline__ int tile_pos(int i) const { return kPagedTile * (i < span.sink_tiles ? i : span.tile0 + i - span.sink_tiles); }
  __device__ __forceinline__ int token_of(int t0, int x) const {
    const int pos = t0 + x, head = t0 < span.sink ? t0 : max(t0, span.lo);
    return pos >= L || (pos >= span.sink && pos < span.lo) ? head : pos;
  }
  __device__ __forceinline__ const int32_t* entry_of(int i, int x) const {
    return a.page_table + (size_t)seq * a.table_stride + (token_of(tile_pos(i), x) >> a.page_shift);
  }
  __device__ __forceinline__ int row_of(int i, int x, int entry) const {
    return (max(0, min(entry, a.n_pages - 1)) << a.page_shift) + (token_of(tile_pos(i), x) & ((1 << a.page_shift) - 1));
  }
  // sequence of row r of a head's rows
  __device__ __forceinline__ int sequence_of(int r) const { return shared ? (row0 + r) / a.meta.qpk : seq; }
  // rows of the cache that it may see
  __device__ __forceinline__ int limit_of(int r) const { return shared ? min(L, a.seq_lens ? a.seq_lens[sequence_of(r)] : L) : L; }
  // element offset of the weights of head hh of the unit, whose group is its hg-th
  __device__ __forceinline__ size_t weights_of(int hh, int hg) const {
    const int width = per_group * kDHead;
    return a.meta.bk_off[g] + (size_t)hg * rk * width + (size_t)(hh + h0 - a.meta.head_off[g] - hg * per_group) * kDHead;
  }
  __device__ __forceinline__ size_t slot() const { return shared ? (size_t)chunk : (size_t)seq * t.n_slots + chunk; }
  __device__ __forceinline__ void store_ml(int hh, int r, float top, float sum) const {
    reinterpret_cast<float2*>(t.ml_part)[slot() * a.meta.n_heads * t.rows + (size_t)(h0 + hh) * t.rows + row0 + r] = make_float2(top, sum);
  }
  // packed row pr, value columns c and c + 1 of the unit; rows of other groups than the columns' are dropped
  __device__ __forceinline__ void store_o(int pr, int c, float x, float y) const {
    const int h = pr / nr, r = pr - h * nr, cg = c / rv;
    if (un.n_groups() > 1 && h / per_group != cg) return;
    const int ohead = a.meta.o_off[g] + (h0 + h - a.meta.head_off[g]) * rv;
    *reinterpret_cast<float2*>(t.o_part + slot() * t.o_stride + (size_t)t.rows * ohead + (size_t)(row0 + r) * rv + c - cg * rv) = make_float2(x, y);
  }
  // Rotated and scaled queries as pairs of float16 numbers, [packed row][hi | lo][feature].  A wavefront takes a row of all heads, which has
  // one position (whose angles lie in 128 cache lines), and has ROWS of them in flight.
  template <typename T, int ROWS> __device__ __forceinline__ void rotate_queries(unsigned char* q, int pitch) const {
    constexpr int kWaves = kPagedThreads / 64, kHeads = 4;
    const int f = threadIdx.x & 63;
    const float k = a.scale / kKeyScale;
    for (int first = threadIdx.x >> 6; first < nr; first += kWaves * ROWS) {
      int pos[ROWS];
      float x0[ROWS][kHeads], x1[ROWS][kHeads], c[ROWS], s[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int r = min(first + i * kWaves, nr - 1), b = sequence_of(r), qh = shared ? row0 + r - b * a.meta.qpk : row0 + r;
        pos[i] = a.q_pos ? a.q_pos[b] : (a.seq_lens ? max(0, min(a.seq_lens[b], a.pos_len)) : a.pos_len) - 1;
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const uint16_t* qp = a.q + ((size_t)b * a.meta.n_heads * a.meta.qpk + (h0 + min(h, nh - 1)) * a.meta.qpk + qh) * kDHead;
          x0[i][h] = T::to_float(qp[f]);
          x1[i][h] = T::to_float(qp[f + kHalf]);
        }
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        pos[i] = max(0, min(pos[i], a.rope_len - 1));
        c[i] = a.rope[rope_f32_index(pos[i], f, 0, kRopeTableStride)] * k;
        s[i] = a.rope[rope_f32_index(pos[i], f, 1, kRopeTableStride)] * k;
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        if (first + i * kWaves >= nr) break;
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          if (h >= nh) break;
          const int pr = h * nr + first + i * kWaves;
          const float y0 = x0[i][h] * c[i] - x1[i][h] * s[i], y1 = x1[i][h] * c[i] + x0[i][h] * s[i];
          uint32_t hi, lo;
          split2<F16>(y0, y1, &hi, &lo);
          uint16_t* y = reinterpret_cast<uint16_t*>(q + pr * pitch) + f;
          y[0] = (uint16_t)hi;
          y[kHalf] = (uint16_t)(hi >> 16);
          y[kDHead] = (uint16_t)lo;
          y[kDHead + kHalf] = (uint16_t)(lo >> 16);
        }
      }
    }
  }
};

// A ring of n stages of `size` bytes from LDS byte `first` on: the stages before and behind `at`.
struct PagedRing {
  int first, size, n;
  __device__ __forceinline__ int stage(int i) const { return first + i % n * size; }
  __device__ __forceinline__ int before(int at) const { return at == first ? first + (n - 1) * size : at - size; }
  __device__ __forceinline__ int behind(int at) const { return at + size == first + n * size ? first : at + size; }
};

// A sub-tile's 16 tokens are columns of its keys in the order 0 4 8 12 1 5 .., so that a lane's four scores are of tokens 4 apart:
// operands of the value product whose lane groups read tokens side by side.
__device__ __forceinline__ int paged_token(int col) { return 4 * (col & 3) + (col >> 2); }
// Piece p of a staged row lies at piece p ^ key: of keys so that eight lanes that read eight tokens' same piece find it on all
// banks, of values so that the four tokens that the lane groups read do.
__device__ __forceinline__ int paged_key_swizzle(int x) { return 4 * (x & 1) + (x >> 2 & 3); }
__device__ __forceinline__ int paged_value_swizzle(int x) { return 4 * (x & 3); }
// where a lane that moves piece p (of `cols` columns from column col0 on; pieces behind the last repeat the first) finds it in a row
__device__ __forceinline__ const unsigned char* paged_source(const uint16_t* base, int col0, int cols, int p) {
  return reinterpret_cast<const unsigned char*>(base + col0 + (p * 8 < cols ? p * 8 : 0));
}

// Angles of the first position of every 16 tokens, a lane per rotation pair: those before, turned by 16 positions, from anchors every
// kPagedAnchorTiles tiles (and where positions jump) that come from the table, whose rows of one position lie in 128 cache lines:
// every tile's from there took a quarter of the time.  A turn rounds twice at 2^-24; after the 15 of a run between anchors, and composed
// with the angle of the position among the 16, cos and sin are off by up to 8e-7 (1e-7 right behind an anchor; the table 6e-8).
struct PagedAngles {
  const PagedWork& w;
  unsigned char* lds;
  uint32_t lds0;
  int anchors, slots, lane;
  float c, s, turn_c, turn_s;                  // of the next 16 tokens; of 16 positions

  __device__ __forceinline__ bool anchor(int j) const { return j < w.i1 && ((j - w.i0) % kPagedAnchorTiles == 0 || j == w.span.sink_tiles); }
  __device__ __forceinline__ int slot(int j) const { return anchors + (j & (slots - 1)) * (kDHead * 4); }
  __device__ __forceinline__ void fetch(int pos, int at) const {
    const int p = min(pos, w.a.rope_len - 1);
    load_to_lds4(w.a.rope + rope_f32_index(p, lane, 0, kRopeTableStride), lds0 + at);
    load_to_lds4(w.a.rope + rope_f32_index(p, lane, 1, kRopeTableStride), lds0 + at + kHalf * 4);
  }
  __device__ __forceinline__ void request(int j) const {
    if (anchor(j)) fetch(w.tile_pos(j), slot(j));
  }
  // by one wavefront: anchors before tile i0 + ahead, and the angles of 16 positions in a slot that none of these has
  __device__ __forceinline__ void begin(int ahead) const {
    for (int j = w.i0; j < w.i0 + ahead; ++j) request(j);
    fetch(16, slot(w.i0 + slots - 1));
  }
  // when these are there
  __device__ __forceinline__ void start() {
    const float* at = reinterpret_cast<const float*>(lds + slot(w.i0 + slots - 1));
    turn_c = at[lane];
    turn_s = at[kHalf + lane];
    reach(w.i0);
  }
  // at tile j
  __device__ __forceinline__ void reach(int j) {
    if (!anchor(j)) return;
    const float* at = reinterpret_cast<const float*>(lds + slot(j));
    c = at[lane];
    s = at[kHalf + lane];
  }
  __device__ __forceinline__ void turn() {
    const float next = __builtin_fmaf(c, turn_c, -(s * turn_s));
    s = __builtin_fmaf(s, turn_c, c * turn_s);
    c = next;
  }
};

}  // namespace

}  // namespace palu
