// Down-projection of new tokens from 4-bit weights, both sides of a layer in one launch.
//
//   h[t, c] = sum_g s[c, g] ( sum_k x[t, k] w[c, k]  -  z[c, g] sum_k x[t, k] )     over the groups g of 128 inputs k
//
// A workgroup takes 16 columns c (one row of codes each) and up to 64 tokens; its eight wavefronts take the groups in turn and add up
// their sums in LDS.  A lane of the matrix operand has 32 consecutive inputs of one column, 16 bytes of codes, for four instructions
// of eight inputs a lane; the sums of x come from the same instruction with ones for weights, which lays them out like the products.
// Codes enter as they are: in float16 as the subnormal numbers c * 2^-24 (exact, also on the matrix cores), in bfloat16 as 128 + c,
// the offset going to the zero-point.  So every product is exact and sums are float32; the only rounding to 16 bits is the result's.

#include "encode_w4.h"

namespace palu {

namespace {

template <typename T> struct W4Codes;
template <> struct W4Codes<F16> {
  static constexpr uint32_t kOne = 0x3c003c00u, kOffset = 0u;
  static constexpr float kUnit = 16777216.f, kZero = 0.f;    // a code is worth 1 / kUnit; what is added to it
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
};
template <> struct W4Codes<BF16> {
  static constexpr uint32_t kOne = 0x3f803f80u, kOffset = 0x43004300u;
  static constexpr float kUnit = 1.f, kZero = 128.f;
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// Eight codes as eight 16-bit numbers, in the order 0 4 1 5 2 6 3 7
template <typename T> __device__ __forceinline__ uint4v spread(uint32_t w, uint32_t offset) {
  uint4v r;
#pragma unroll
  for (int u = 0; u < 4; ++u) r[u] = ((w >> (4 * u)) & 0x000f000fu) | offset;
  return r;
}
// eight 16-bit numbers in that order
__device__ __forceinline__ uint4v reorder(uint4v x) {
  return uint4v{__builtin_amdgcn_perm(x.z, x.x, 0x05040100u), __builtin_amdgcn_perm(x.z, x.x, 0x07060302u),
                __builtin_amdgcn_perm(x.w, x.y, 0x05040100u), __builtin_amdgcn_perm(x.w, x.y, 0x07060302u)};
}

template <typename T, int NT>
__global__ __launch_bounds__(kW4Threads) void encode_w4_kernel(EncodeW4Args a) {
  constexpr int kWaves = kW4Threads / 64;
  __shared__ float part[kWaves][NT * 16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, kg = lane >> 4;
  const int s = (int)blockIdx.x >= a.side[0].tiles;
  const EncodeW4Side& sd = a.side[s];
  const int c0 = 16 * (blockIdx.x - (s ? a.side[0].tiles : 0));
  const int t0 = blockIdx.y * (NT * 16), groups = a.d / 128;
  const uint32_t offset = W4Codes<T>::kOffset == 0 ? 0u : per_lane_constant(W4Codes<T>::kOffset);
  const uint4v ones = {W4Codes<T>::kOne, W4Codes<T>::kOne, W4Codes<T>::kOne, W4Codes<T>::kOne};
  const uint8_t* codes = sd.codes + (size_t)(c0 + col) * (a.d / 2) + kg * 16;
  const uint16_t* scale = sd.scale + (size_t)(c0 + col) * groups;
  const uint16_t* zero = sd.zero + (size_t)(c0 + col) * groups;
  const uint16_t* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = a.x + (size_t)min(t0 + 16 * n + col, a.n_tok - 1) * a.d + kg * 32;   // (tokens behind the last: the last again)
  float4v h[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) h[n] = float4v{0, 0, 0, 0};
  for (int g = wave; g < groups; g += kWaves) {
    const uint4v w = *reinterpret_cast<const uint4v*>(codes + g * 64);
    const float sc = F16::to_float(scale[g]), z = F16::to_float(zero[g]) + W4Codes<T>::kZero;
    float4v dot[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) dot[n] = sum[n] = float4v{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4v b = spread<T>(w[j], offset);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint4v v = reorder(*reinterpret_cast<const uint4v*>(x[n] + g * 128 + j * 8));
        dot[n] = W4Codes<T>::mma(v, b, dot[n]);
        sum[n] = W4Codes<T>::mma(v, ones, sum[n]);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) h[n][e] += sc * (dot[n][e] * W4Codes<T>::kUnit - z * sum[n][e]);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][16 * n + 4 * kg + e][col] = h[n][e];
  __syncthreads();
  for (int i = threadIdx.x; i < NT * 16 * 16; i += kW4Threads) {
    const int t = i >> 4, c = i & 15;
    if (t0 + t >= a.n_tok) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += part[w][t][c];
    const long long row = a.dst_row ? a.dst_row[t0 + t] : t0 + t;
    if (row >= 0) sd.latent[row * sd.stride + c0 + c] = T::from_float(sum);
  }
}

template <typename T> EncodeW4Fn pick(int tiles) {
  return tiles == 1 ? encode_w4_kernel<T, 1> : (tiles == 2 ? encode_w4_kernel<T, 2> : encode_w4_kernel<T, 4>);
}

}  // namespace

EncodeW4Fn encode_w4_form(int act, int tiles) { return act == PALU_F16 ? pick<F16>(tiles) : pick<BF16>(tiles); }

}  // namespace palu
