// Partial results of attention over a paged latent cache: merged, normalised and multiplied by B_v.

#include "paged_dev.h"

namespace palu {

// A workgroup takes R rows (sequence, query head) of one key/value head: weights exp2(max - largest max) of their partial results, the
// weighted sums of the latents, normalised and split into pairs of 16-bit numbers hi + lo (float16: 2^-21, or 2^-25 absolute below
// 1/8), times the head's 128 columns of B_v (a wavefront makes 32; its weights are requested first, and arrive meanwhile).
// grid (blocks of R rows, key/value heads), 256 threads.
// Bound by the latency of its few dependent steps where there are few rows, else by reading the partial results: R is as
// small as it takes for a workgroup or two per compute unit.
template <typename T, int R>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedMergeArgs a) {
  constexpr int kPitch = PALU_PAGED_MAX_RANK + 8, kBlock = 64;
  __shared__ __attribute__((aligned(16))) uint16_t Oh[2][R * kPitch];
  __shared__ __attribute__((aligned(16))) float Part[256 * 4];
  __shared__ float Weight[R][kBlock];
  __shared__ float Inv[R], Top[R];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, kg = lane >> 4;
  const PagedMeta& m = a.meta;
  const int h = blockIdx.y, g = m.group_of_head[h];
  const int rv = m.v_off[g + 1] - m.v_off[g];
  const int rows = a.batch * m.qpk, row0 = blockIdx.x * R;
  const int n = min(R, rows - row0);
  const int ohead = m.o_off[g] + (h - m.head_off[g]) * rv;

  // B_v: columns 32 wave + 2 col (+ 1)
  const int width = (m.head_off[g + 1] - m.head_off[g]) * kDHead;
  const uint16_t* B = a.Bv + m.bv_off[g] + (size_t)(h - m.head_off[g]) * kDHead + 32 * wave + 2 * col;
  uint32_t V[8][8];
#pragma unroll
  for (int ks = 0; ks < 8; ++ks)
    if (32 * ks < rv)
#pragma unroll
      for (int e = 0; e < 8; ++e) V[ks][e] = *reinterpret_cast<const uint32_t*>(B + (size_t)(32 * ks + 8 * kg + e) * width);

  // the sequences' own partial results first, then those of the shared tokens
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

  // maximum and sum of every row: 256 / R threads each.  A partial result that saw no row has the maximum -inf and the sum 0; one of
  // nothing but NaN scores, which a maximum passes over, -inf and NaN: its sum counts all the same, and the row becomes NaN.
  constexpr int kPer = 256 / R < 64 ? 256 / R : 64;
  if (tid < kPer * R) {
    const int r = tid / kPer;
    float top = -INFINITY, sum = 0.f;
    if (r < n) {
      const int row = row0 + r, b = row / m.qpk, n_own = own_slots(b);
      for (int s = tid % kPer; s < n_own + a.n_shared; s += kPer) {
        const float2 x = ml_of(row, b, n_own, s);
        const float now = fmaxf(top, x.x);
        sum = now > -INFINITY ? sum * __builtin_amdgcn_exp2f(top - now) + x.y * __builtin_amdgcn_exp2f(x.x - now) : sum + x.y;
        top = now;
      }
    }
#pragma unroll
    for (int d = 1; d < kPer; d *= 2) {
      const float t2 = __shfl_xor(top, d), s2 = __shfl_xor(sum, d), now = fmaxf(top, t2);
      sum = now > -INFINITY ? sum * __builtin_amdgcn_exp2f(top - now) + s2 * __builtin_amdgcn_exp2f(t2 - now) : sum + s2;
      top = now;
    }
    if (tid % kPer == 0) {
      Top[r] = top;
      Inv[r] = sum == 0.f ? 0.f : 1.f / sum;
    }
  }

  // weighted sums: thread (row, 4 columns) or, with few of these, every n_parts-th partial result of one
  const int quads = rv / 4, items = n * quads, n_parts = max(1, 256 / items);
  int most = 0;                                              // partial results of a row
  for (int b = row0 / m.qpk; b <= (row0 + n - 1) / m.qpk; ++b) most = max(most, own_slots(b));
  most += a.n_shared;
  constexpr int kItems = (R * PALU_PAGED_MAX_RANK / 4 + 255) / 256;
  float4v o[kItems];
#pragma unroll
  for (int i = 0; i < kItems; ++i) o[i] = float4v{0, 0, 0, 0};
  for (int s0 = 0; s0 < most; s0 += kBlock) {
    __syncthreads();
    for (int x = tid; x < n * kBlock; x += 256) {
      const int r = x / kBlock, s = s0 + x % kBlock, row = row0 + r, b = row / m.qpk, n_own = own_slots(b);
      float w = -1.f;                                        // a partial result that saw no row is none, whatever it holds
      if (s < n_own + a.n_shared) {
        const float top = ml_of(row, b, n_own, s).x;
        if (top > -INFINITY) w = __builtin_amdgcn_exp2f(top - Top[r]);
      }
      Weight[r][s - s0] = w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int x = tid + 256 * i;
      if (x < items * n_parts) {
        const int part = x / items, y = x - part * items, r = y / quads, c = (y - r * quads) * 4;
        const int row = row0 + r, b = row / m.qpk, n_own = own_slots(b), end = min(n_own + a.n_shared - s0, kBlock);
        const float* own = a.o_part + (size_t)(b * a.n_slots) * a.o_stride + (size_t)m.qpk * ohead + (size_t)(row - b * m.qpk) * rv + c;
        const float* shared = a.o_shared + (size_t)rows * ohead + (size_t)row * rv + c;
#pragma unroll 4
        for (int k = part; k < end; k += n_parts) {
          const int s = s0 + k;
          const float w = Weight[r][k];
          const float4v p = *reinterpret_cast<const float4v*>(s < n_own ? own + (size_t)s * a.o_stride : shared + (size_t)(s - n_own) * a.o_shared_stride);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] += w < 0.f ? 0.f : w * p[e];
        }
      }
    }
  }
  auto put = [&](int r, int c, float4v x) {
    x *= Inv[r];
    uint32_t hi[2], lo[2];
    split2<T>(x[0], x[1], &hi[0], &lo[0]);
    split2<T>(x[2], x[3], &hi[1], &lo[1]);
    *reinterpret_cast<uint2v*>(&Oh[0][r * kPitch + c]) = uint2v{hi[0], hi[1]};
    *reinterpret_cast<uint2v*>(&Oh[1][r * kPitch + c]) = uint2v{lo[0], lo[1]};
  };
  __syncthreads();
  if (n_parts > 1) {
    if (tid < items * n_parts) *reinterpret_cast<float4v*>(&Part[tid * 4]) = o[0];
    __syncthreads();
    if (tid < items) {
      float4v x = o[0];
      for (int p = 1; p < n_parts; ++p) x += *reinterpret_cast<const float4v*>(&Part[(p * items + tid) * 4]);
      put(tid / quads, tid % quads * 4, x);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kItems; ++i)
      if (tid + 256 * i < items) put((tid + 256 * i) / quads, (tid + 256 * i) % quads * 4, o[i]);
  }
  __syncthreads();

  float4v acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  auto product = [&](int ks, const uint32_t (&v)[8]) __attribute__((always_inline)) {
    uint4v f0, f1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f0[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x05040100u);
      f1[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x07060302u);
    }
    const int r = min(col, R - 1);                           // (rows behind the last: the same again)
    const uint4v hi = *reinterpret_cast<const uint4v*>(&Oh[0][r * kPitch + 32 * ks + 8 * kg]);
    const uint4v lo = *reinterpret_cast<const uint4v*>(&Oh[1][r * kPitch + 32 * ks + 8 * kg]);
    acc[0] = mma<T>(hi, f0, acc[0]);
    acc[1] = mma<T>(hi, f1, acc[1]);
    acc[0] = mma<T>(lo, f0, acc[0]);
    acc[1] = mma<T>(lo, f1, acc[1]);
  };
#pragma unroll
  for (int ks = 0; ks < 8; ++ks)
    if (32 * ks < rv) product(ks, V[ks]);
  for (int ks = 8; 32 * ks < rv; ++ks) {
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const uint32_t*>(B + (size_t)(32 * ks + 8 * kg + e) * width);
    product(ks, v);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int r = 4 * kg + e;
    if (r < n) {
      const int row = row0 + r, b = row / m.qpk;
      uint16_t* out = a.out + ((size_t)b * m.n_heads * m.qpk + h * m.qpk + row - b * m.qpk) * kDHead + 32 * wave + 2 * col;
      *reinterpret_cast<uint32_t*>(out) = pack2<T>(acc[0][e], acc[1][e]);
    }
  }
}

template <typename T> PagedMergeFn paged_merge_form(int rows) {
  switch (rows) {
    case 1: return paged_merge_kernel<T, 1>;
    case 2: return paged_merge_kernel<T, 2>;
    case 4: return paged_merge_kernel<T, 4>;
    default: return paged_merge_kernel<T, 8>;
  }
}
template PagedMergeFn paged_merge_form<F16>(int);
template PagedMergeFn paged_merge_form<BF16>(int);

}  // namespace palu
