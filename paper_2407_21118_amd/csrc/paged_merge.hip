// Partial results of attention over a paged latent cache: merged, normalised and multiplied by B_v.

#include "paged_dev.h"

namespace palu {

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

template <typename T> PagedMergeFn paged_merge_form() { return paged_merge_kernel<T>; }
template PagedMergeFn paged_merge_form<F16>();
template PagedMergeFn paged_merge_form<BF16>();

}  // namespace palu
