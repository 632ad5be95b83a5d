// Decode attention over a paged latent cache held in 4 bits, with a sliding window and a few first rows (sinks).
//
//   out = softmax_t( RoPE(q, p) . RoPE(H_k[t] B_k, t) / sqrt(d_h) ) H_v[t] B_v,   H[t, r] = (code - zero) * scale
//
// Partial results (unnormalised sums, maxima, row sums) are merged, normalised and multiplied by B_v in paged_merge_kernel.  This kernel is for rotations whose
// slow half turns too fast to be folded with the query (pagedq_fold.hip).

#include "pagedq.h"

namespace palu {

namespace {

// One (sequence, key/value head, run of tiles) per workgroup, everything in float32 on the vector units.
template <typename T>
__global__ __launch_bounds__(kPagedQThreads) void pagedq_plain_kernel(PagedQArgs a) {
  constexpr int kRows = 8;                     // query rows at a time
  __shared__ float H[kPagedTile][132];         // 128 channels of the tile's latents, dequantized
  __shared__ float K[kPagedTile][kDHead + 1];  // rotated keys
  __shared__ float Q[kRows][kDHead];
  __shared__ float P[kRows][kPagedTile], Alpha[kRows];
  __shared__ int Row[kPagedTile];
  const PagedMeta& m = a.meta;
  const int tid = threadIdx.x;
  const int h = blockIdx.x % m.n_heads, rest = blockIdx.x / m.n_heads, chunk = rest % a.n_slots, seq = rest / a.n_slots;
  const int g = m.group_of_head[h], rk = m.k_off[g + 1] - m.k_off[g], rv = m.v_off[g + 1] - m.v_off[g];
  const int L = max(0, min(a.seq_lens ? a.seq_lens[seq] : a.max_len, a.max_len));
  const PagedSpan span = paged_span(L, 0, a.window, a.n_sink);
  const int n_chunks = (span.n_tiles + a.chunk_tiles - 1) / a.chunk_tiles;
  if (chunk >= n_chunks) return;
  const int i0 = (int)((long long)span.n_tiles * chunk / n_chunks), i1 = (int)((long long)span.n_tiles * (chunk + 1) / n_chunks);
  const int width = (m.head_off[g + 1] - m.head_off[g]) * kDHead;
  const uint16_t* B = a.Bk + m.bk_off[g] + (size_t)(h - m.head_off[g]) * kDHead;
  const size_t slot = (size_t)seq * a.n_slots + chunk;
  const int ohead = m.o_off[g] + (h - m.head_off[g]) * rv;
  const int q_pos = max(0, min(a.q_pos ? a.q_pos[seq] : L - 1, a.rope_len - 1));

  auto held = [&](const PagedQSide& s, int row, int block, int c) __attribute__((always_inline)) {   // channel c of a block
    const uint8_t byte = s.codes[(size_t)row * s.row_bytes + block * 64 + (c >> 1)];
    const size_t at = (size_t)row * s.n_blocks + block;
    return ((float)(c & 1 ? byte >> 4 : byte & 15) - F16::to_float(s.zero[at])) * F16::to_float(s.scale[at]);
  };
  for (int r0 = 0; r0 < m.qpk; r0 += kRows) {
    const int nr = min(kRows, m.qpk - r0);
    __syncthreads();
    for (int x = tid; x < nr * kHalf; x += kPagedQThreads) {
      const int r = x / kHalf, f = x % kHalf;
      const uint16_t* q = a.q + ((size_t)seq * m.n_heads * m.qpk + h * m.qpk + r0 + r) * kDHead;
      const float c = a.rope[rope_f32_index(q_pos, f, 0, kRopeTableStride)], s = a.rope[rope_f32_index(q_pos, f, 1, kRopeTableStride)];
      const float x0 = T::to_float(q[f]), x1 = T::to_float(q[f + kHalf]);
      Q[r][f] = (x0 * c - x1 * s) * a.scale;
      Q[r][f + kHalf] = (x1 * c + x0 * s) * a.scale;
    }
    float O[kRows][2] = {};                    // value columns tid and tid + 256
    float run_max = -INFINITY, run_sum = 0.f;  // of row tid
    for (int i = i0; i < i1; ++i) {
      const int t0 = kPagedTile * (i < span.sink_tiles ? i : span.tile0 + i - span.sink_tiles);
      __syncthreads();
      if (tid < kPagedTile) {                  // row of the cache, -1 where the token is not attended
        const int t = t0 + tid;
        int row = -1;
        if (t < L && (t < span.sink || t >= span.lo))
          row = (max(0, min(a.page_table[(size_t)seq * a.table_stride + (t >> a.page_shift)], a.n_pages - 1)) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
        Row[tid] = row;
      }
      float acc[16] = {};                      // feature tid % 128 of tokens 16 (tid / 128) ..
      const int f = tid & 127, x0 = 16 * (tid >> 7);
      for (int block = 0; block < rk / 128; ++block) {
        __syncthreads();
        for (int x = tid; x < kPagedTile * 128; x += kPagedQThreads) {
          const int t = x >> 7, c = x & 127;
          H[t][c] = Row[t] < 0 ? 0.f : held(a.k, Row[t], m.k_off[g] / 128 + block, c);
        }
        __syncthreads();
        for (int c = 0; c < 128; c += 4) {
          float b[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) b[e] = T::to_float(B[(size_t)(block * 128 + c + e) * width + f]);
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const float4v hh = *reinterpret_cast<const float4v*>(&H[x0 + x][c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[x] = __builtin_fmaf(hh[e], b[e], acc[x]);
          }
        }
      }
      for (int x = 0; x < 16; ++x) K[x0 + x][f] = acc[x];
      __syncthreads();
      for (int x = tid; x < kPagedTile * kHalf; x += kPagedQThreads) {
        const int t = x / kHalf, p = x % kHalf, pos = min(t0 + t, a.rope_len - 1);
        const float c = a.rope[rope_f32_index(pos, p, 0, kRopeTableStride)], s = a.rope[rope_f32_index(pos, p, 1, kRopeTableStride)];
        const float lo = K[t][p], hi = K[t][p + kHalf];
        K[t][p] = lo * c - hi * s;
        K[t][p + kHalf] = hi * c + lo * s;
      }
      __syncthreads();
      for (int x = tid; x < nr * kPagedTile; x += kPagedQThreads) {
        const int r = x / kPagedTile, t = x % kPagedTile;
        float s = 0.f;
        for (int e = 0; e < kDHead; ++e) s = __builtin_fmaf(K[t][e], Q[r][e], s);
        P[r][t] = Row[t] < 0 ? -INFINITY : s;
      }
      __syncthreads();
      if (tid < nr) {
        float now = run_max;
        for (int t = 0; t < kPagedTile; ++t) now = fmaxf(now, P[tid][t]);
        const float zero = now == -INFINITY ? 0.f : now, alpha = __builtin_amdgcn_exp2f(run_max - zero);
        float sum = 0.f;
        for (int t = 0; t < kPagedTile; ++t) {
          const float p = __builtin_amdgcn_exp2f(P[tid][t] - zero);
          P[tid][t] = p;
          sum += p;
        }
        run_max = now;
        run_sum = run_sum * alpha + sum;
        Alpha[tid] = alpha;
      }
      __syncthreads();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int c = tid + 256 * half;
        if (c >= rv) continue;
#pragma unroll
        for (int r = 0; r < kRows; ++r) O[r][half] *= r < nr ? Alpha[r] : 0.f;
        for (int t = 0; t < kPagedTile; ++t) {
          if (Row[t] < 0) continue;
          const float v = held(a.v, Row[t], m.v_off[g] / 128 + (c >> 7), c & 127);
#pragma unroll
          for (int r = 0; r < kRows; ++r) O[r][half] = __builtin_fmaf(r < nr ? P[r][t] : 0.f, v, O[r][half]);
        }
      }
    }
    if (tid < nr) reinterpret_cast<float2*>(a.ml_part)[(slot * m.n_heads + h) * m.qpk + r0 + tid] = make_float2(run_max, run_sum);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int c = tid + 256 * half;
      if (c < rv)
#pragma unroll
        for (int r = 0; r < kRows; ++r)
          if (r < nr) a.o_part[slot * a.o_stride + (size_t)m.qpk * ohead + (size_t)(r0 + r) * rv + c] = O[r][half];
    }
  }
}

}  // namespace

PagedQFn pagedq_plain_form(int act) { return act == PALU_F16 ? pagedq_plain_kernel<F16> : pagedq_plain_kernel<BF16>; }

}  // namespace palu
