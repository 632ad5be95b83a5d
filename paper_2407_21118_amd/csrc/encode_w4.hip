// Down-projection of new tokens from 4-bit weights, both sides of a layer in one launch.
//
//   h[t, c] = sum_g s[c, g] ( sum_k x[t, k] w[c, k]  -  z[c, g] sum_k x[t, k] )     over the groups g of 128 inputs k
//
// A workgroup takes 16 or 64 columns c (one row of codes each) and 16 or 32 tokens; its eight wavefronts take the groups, four in turn, and add up
// their sums in LDS.  The sums of x come from the matrix instruction, too, with ones for weights, which lays them out like the products.
// Codes enter as 16 + c, a normal number with the code in its uppermost bits, the offset going to the zero-point.  So every product is exact and sums
// are float32; the only rounding to 16 bits is the result's.  (The matrix cores keep 24 bits below the largest exponent of an instruction's products and
// take a subnormal operand's for 2^-14: codes as the float16 numbers c * 2^-24 lost what lies 2^-15 below the largest input.)
// Bound by latency: the weights' bytes (8.4 MB of 4096 inputs by 4096 columns) are worth 1.6 us, and a kernel without its loop takes 2.4; it takes
// 4.8 us for a token, 6.1 for 24; 333 tokens by 1024 columns 13.6 (a workgroup's 32 by 64 results: 12.5).  64 tokens by 64 columns were slower (22 us a
// round of workgroups).  4096 tokens by 4096 columns take 354 us, 390 TFLOP/s: codes are spread for the matrix instructions anew for every 32 tokens, which keeps
// the matrix pipe at 20 %.

#include "encode_w4.h"
#include "paged_dev.h"

namespace palu {

namespace {

template <typename T> struct W4Codes;
template <> struct W4Codes<F16> {
  static constexpr uint32_t kOne = 0x3c003c00u, kSixteen = 0x4c004c00u;
  static constexpr int kShift = 6;             // of a code, to add it to 16
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
};
template <> struct W4Codes<BF16> {
  static constexpr uint32_t kOne = 0x3f803f80u, kSixteen = 0x41804180u;
  static constexpr int kShift = 3;
  static __device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// Eight codes as eight 16-bit numbers 16 + c
template <typename T> __device__ __forceinline__ uint4v spread(uint32_t w, uint32_t sixteen) {
  const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  uint4v r;
#pragma unroll
  for (int u = 0; u < 4; ++u) r[u] = __builtin_amdgcn_perm(odd, even, 0x0c040c00u + 0x00010001u * u) << W4Codes<T>::kShift | sixteen;
  return r;
}

// Number i of lane group g (of four of 16 lanes) goes to number g of lane group i
__device__ __forceinline__ uint4v transpose(uint4v w) {
  uint32_t x[4] = {w[0], w[1], w[2], w[3]};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto r = __builtin_amdgcn_permlane32_swap(x[i], x[i + 2], false, false);
    x[i] = r[0];
    x[i + 2] = r[1];
  }
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const auto r = __builtin_amdgcn_permlane16_swap(x[i], x[i + 1], false, false);
    x[i] = r[0];
    x[i + 1] = r[1];
  }
  return uint4v{x[0], x[1], x[2], x[3]};
}

template <typename T, int NT, int NC, int U>
__global__ __launch_bounds__(kW4Threads, 2) void encode_w4_kernel(EncodeW4Args a) {
  constexpr int kWaves = kW4Threads / 64, kPitch = 16 * NC + 1;
  constexpr int kRows = NT * 16 * 256;         // bytes of a group's inputs
  __shared__ __attribute__((aligned(16))) unsigned char lds[kWaves * U * kRows > kWaves * NT * 16 * kPitch * 4 ? kWaves * U * kRows : kWaves * NT * 16 * kPitch * 4];
  float (*const part)[NT * 16][kPitch] = reinterpret_cast<float (*)[NT * 16][kPitch]>(lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, kg = lane >> 4;
  const int s = (int)blockIdx.y >= a.side[0].tiles;
  const EncodeW4Side& sd = a.side[s];
  const int c0 = 16 * NC * (blockIdx.y - (s ? a.side[0].tiles : 0));
  const int t0 = blockIdx.x * (NT * 16), groups = a.d / 128;
  const uint32_t sixteen = per_lane_constant(W4Codes<T>::kSixteen);
  const uint4v ones = {W4Codes<T>::kOne, W4Codes<T>::kOne, W4Codes<T>::kOne, W4Codes<T>::kOne};
  const uint8_t* const codes = sd.codes + (size_t)(c0 + col) * (a.d / 2) + kg * 16;
  const uint16_t* const scale = sd.scale + (size_t)(c0 + (NC == 1 ? col : lane)) * groups;
  const uint16_t* const zero = sd.zero + (size_t)(c0 + (NC == 1 ? col : lane)) * groups;
  const bool wide = groups % 4 == 0 && ((reinterpret_cast<uintptr_t>(sd.scale) | reinterpret_cast<uintptr_t>(sd.zero)) & 7) == 0;
  auto four = [&](const uint16_t* p, int here) __attribute__((always_inline)) {    // the first `here` of four numbers (and others)
    if (wide) return *reinterpret_cast<const uint2v*>(p);
    return uint2v{(uint32_t)p[0] | (uint32_t)p[min(1, here - 1)] << 16, (uint32_t)p[min(2, here - 1)] | (uint32_t)p[min(3, here - 1)] << 16};
  };
  // Inputs go by LDS, in pieces of 16 bytes: token t's piece p at place p ^ t of its 16.  An instruction takes 256 bytes of each of four tokens.  (Read as
  // operands, 64 bytes of each of 16 tokens, they lie a power of two apart in few sets of the first cache: 24 tokens of 4096 inputs by 4096 columns took 11.6 us
  // against 7.0.)
  const uint16_t* x[4 * NT];
#pragma unroll
  for (int i = 0; i < 4 * NT; ++i) {
    const int t = 4 * i + kg;                  // (tokens behind the last: the last again)
    x[i] = a.x + (size_t)min(t0 + t, a.n_tok - 1) * a.d + ((col ^ t) & 15) * 8;
  }
  unsigned char* const mine = lds + wave * U * kRows;
  const uint32_t mine0 = lds_addr(mine);
  float4v h[NT][NC];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < NC; ++c) h[n][c] = float4v{0, 0, 0, 0};
  // Four groups in turn per wavefront, every workgroup from others on: tokens lie a power of two apart, and all would ask the same channels of L2.
  const int quads = (groups + 3) / 4;
  for (int q0 = wave; q0 < quads; q0 += kWaves) {
    const int q = (q0 + (int)blockIdx.y) % quads, here = min(4, groups - 4 * q);
    // a lane takes four scales and zero-points of one column of the workgroup, and hands them to those that need them
    const uint2v mine_s = four(scale + 4 * q, here), mine_z = four(zero + 4 * q, here);
    uint2v sc[NC], z[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        sc[c][e] = NC == 1 ? mine_s[e] : (uint32_t)__shfl((int)mine_s[e], 16 * c + col);
        z[c][e] = NC == 1 ? mine_z[e] : (uint32_t)__shfl((int)mine_z[e], 16 * c + col);
      }
#pragma unroll
    for (int i0 = 0; i0 < 4; i0 += U) {
      uint4v w[U][NC];                         // U groups' loads before anything else
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int g = 4 * q + min(i0 + i, here - 1);
#pragma unroll
        for (int c = 0; c < NC; ++c) w[i][c] = *reinterpret_cast<const uint4v*>(codes + (size_t)(16 * c) * (a.d / 2) + g * 64);
#pragma unroll
        for (int k = 0; k < 4 * NT; ++k)
          if (k == 0 || t0 + 4 * k < a.n_tok) load_to_lds(x[k] + g * 128, mine0 + i * kRows + k * 1024);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < U; ++i) {
        if (i0 + i >= here) break;
        float4v dot[NT][NC], sum[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          sum[n] = float4v{0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < NC; ++c) dot[n][c] = float4v{0, 0, 0, 0};
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) w[i][c] = transpose(w[i][c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint4v v[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            v[n] = *reinterpret_cast<const uint4v*>(mine + i * kRows + (16 * n + col) * 256 + (((4 * j + kg) ^ col) & 15) * 16);
            sum[n] = W4Codes<T>::mma(v[n], ones, sum[n]);
          }
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uint4v b = spread<T>(w[i][c][j], sixteen);
#pragma unroll
            for (int n = 0; n < NT; ++n) dot[n][c] = W4Codes<T>::mma(v[n], b, dot[n][c]);
          }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int k = i0 + i;
          const float s1 = F16::to_float((uint16_t)(sc[c][k >> 1] >> (16 * (k & 1)))), z1 = F16::to_float((uint16_t)(z[c][k >> 1] >> (16 * (k & 1))));
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[n][c][e] = __builtin_fmaf(s1, __builtin_fmaf(-z1, sum[n][e], __builtin_fmaf(-16.f, sum[n][e], dot[n][c][e])), h[n][c][e]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the inputs have been read)
    }
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][16 * n + 4 * kg + e][16 * c + col] = h[n][c][e];
  __syncthreads();
  for (int i = threadIdx.x; i < NT * 16 * NC * 16; i += kW4Threads) {
    const int t = i / (16 * NC), c = i % (16 * NC);
    if (t0 + t >= a.n_tok) continue;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < kWaves; ++u) sum += part[u][t][c];
    const long long row = a.dst_row ? a.dst_row[t0 + t] : t0 + t;
    if (row >= 0) sd.latent[row * sd.stride + c0 + c] = T::from_float(sum);
  }
}

template <typename T> EncodeW4Fn pick(const EncodeW4Form& f) {
  if (f.columns == 4) return encode_w4_kernel<T, 2, 4, 2>;
  return f.tokens == 1 ? encode_w4_kernel<T, 1, 1, 4> : encode_w4_kernel<T, 2, 1, 2>;
}

}  // namespace

EncodeW4Fn encode_w4_form(int act, const EncodeW4Form& f) { return act == PALU_F16 ? pick<F16>(f) : pick<BF16>(f); }

}  // namespace palu
