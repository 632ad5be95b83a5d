// Rows of a quantized latent cache: quantized as they are written, and read back.  Both sides of a layer in one launch.
//
// 16 lanes take a block of 128 channels, 8 of them each: 16 bytes of the latents, and 4, 3 or 2 bytes of codes.
//   write  s = f16((max - min) / (2^B - 1)), 0 -> 1;  z = f16(clamp(rint(-min / s)));  c = clamp(rint(x / s) + z, 0, 2^B - 1), every step one
//          float32 operation (ties to even): the numbers that quant_kernel writes
//   read   (c - z) * s: the difference and the product are exact in float32 for zero-points up to 2^12 (else each is rounded to 2^-24),
//          then one rounding to the layer's type
// Bound by the memory: a value is 2 bytes on one side and 1/2 + 1/32 on the other.

#include "cache_rows.h"

namespace palu {

namespace {

// the larger / smaller of x over 16 lanes: lane ^ 1, ^ 2 in a quad, mirrored in 8 lanes, mirrored in 16
template <int CTRL> __device__ __forceinline__ float from_lane(float x) {
  const int u = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float max_of_16(float x) {
  x = fmaxf(x, from_lane<0xB1>(x));
  x = fmaxf(x, from_lane<0x4E>(x));
  x = fmaxf(x, from_lane<0x141>(x));
  return fmaxf(x, from_lane<0x140>(x));
}
__device__ __forceinline__ float min_of_16(float x) {
  x = fminf(x, from_lane<0xB1>(x));
  x = fminf(x, from_lane<0x4E>(x));
  x = fminf(x, from_lane<0x141>(x));
  return fminf(x, from_lane<0x140>(x));
}

// 8 channels of a latent row
template <bool WIDE> __device__ __forceinline__ uint4v load8(const uint16_t* p) {
  if constexpr (WIDE) return *reinterpret_cast<const uint4v*>(p);
  return uint4v{(uint32_t)p[0] | (uint32_t)p[1] << 16, (uint32_t)p[2] | (uint32_t)p[3] << 16, (uint32_t)p[4] | (uint32_t)p[5] << 16,
                (uint32_t)p[6] | (uint32_t)p[7] << 16};
}
template <bool WIDE> __device__ __forceinline__ void store8(uint16_t* p, uint4v v) {
  if constexpr (WIDE) {
    *reinterpret_cast<uint4v*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[2 * i] = (uint16_t)v[i];
      p[2 * i + 1] = (uint16_t)(v[i] >> 16);
    }
  }
}

// The block of 128 channels that these 16 lanes take: of latent row `i`, `block` of side `s`
struct CacheItem {
  long long i, row;
  int s, block;
  bool valid;
  __device__ __forceinline__ CacheItem(const CacheRowsArgs& a, long long item) {
    const int per_row = a.side[0].n_blocks + a.side[1].n_blocks;
    i = (long long)((unsigned)item / (unsigned)per_row);     // (the host keeps items below 2^32)
    block = (int)(item - i * per_row);
    s = block >= a.side[0].n_blocks;
    block -= s ? a.side[0].n_blocks : 0;
    valid = i < a.n;
    row = !valid ? -1 : (a.row ? (long long)a.row[i] : i);
    valid = row >= 0 && row < a.n_rows;
  }
};

template <typename T, bool WIDE>
__global__ __launch_bounds__(kCacheRowsThreads) void quant_rows_kernel(CacheRowsArgs a) {
  const int l = threadIdx.x & 15;
  const CacheItem it(a, (long long)blockIdx.x * kCacheRowsItems + (threadIdx.x >> 4));
  const CacheSide& sd = a.side[it.s];
  if (!it.valid) return;                       // (all 16 lanes of a block alike)
  const uint4v raw = load8<WIDE>(sd.latent + it.i * sd.stride + it.block * 128 + l * 8);
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = T::to_float((uint16_t)raw[e]);
    x[2 * e + 1] = T::to_float((uint16_t)(raw[e] >> 16));
  }
  float low = x[0], high = x[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    low = fminf(low, x[e]);
    high = fmaxf(high, x[e]);
  }
  low = min_of_16(low);
  high = max_of_16(high);
  const float top = (float)((1 << sd.bits) - 1);
  uint16_t s16 = F16::from_float(__fdiv_rn(__fsub_rn(high, low), top));
  if ((s16 & 0x7fffu) == 0) s16 = 0x3c00u;
  const float s = F16::to_float(s16);
  const uint16_t z16 = F16::from_float(fminf(fmaxf(rintf(__fdiv_rn(-low, s)), -65504.f), 65504.f));
  const float z = F16::to_float(z16);
  uint32_t c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = (uint32_t)fminf(fmaxf(__fadd_rn(rintf(__fdiv_rn(x[e], s)), z), 0.f), top);
  const int R = sd.n_blocks * 128;
  uint8_t* codes = sd.codes + it.row * (long long)(R / 8 * sd.bits);
  const int at = it.block * 16 + l;            // 8 channels
  if (sd.bits == 4) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= c[e] << (4 * e);
    reinterpret_cast<uint32_t*>(codes)[at] = w;
  } else {
    uint32_t w = 0, third = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w |= (c[e] & 3u) << (2 * e);
      third |= (c[e] >> 2) << e;
    }
    reinterpret_cast<uint16_t*>(codes)[at] = (uint16_t)w;
    if (sd.bits == 3) codes[R / 4 + at] = (uint8_t)third;
  }
  if (l == 0) {
    sd.scale[it.row * sd.n_blocks + it.block] = s16;
    sd.zero[it.row * sd.n_blocks + it.block] = z16;
  }
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(kCacheRowsThreads) void dequant_rows_kernel(CacheRowsArgs a) {
  const int l = threadIdx.x & 15;
  const CacheItem it(a, (long long)blockIdx.x * kCacheRowsItems + (threadIdx.x >> 4));
  const CacheSide& sd = a.side[it.s];
  if (!it.valid) return;
  const int R = sd.n_blocks * 128, at = it.block * 16 + l;
  const uint8_t* codes = sd.codes + it.row * (long long)(R / 8 * sd.bits);
  uint32_t w;
  if (sd.bits == 4) w = reinterpret_cast<const uint32_t*>(codes)[at];
  else w = expand_low_bits(reinterpret_cast<const uint16_t*>(codes)[at], sd.bits == 3 ? codes[R / 4 + at] : 0u, sd.bits == 3);
  const float s = F16::to_float(sd.scale[it.row * sd.n_blocks + it.block]), z = F16::to_float(sd.zero[it.row * sd.n_blocks + it.block]);
  uint4v out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint16_t x = T::from_float(((float)((w >> (8 * e)) & 15u) - z) * s), y = T::from_float(((float)((w >> (8 * e + 4)) & 15u) - z) * s);
    out[e] = (uint32_t)x | (uint32_t)y << 16;
  }
  store8<WIDE>(sd.latent + it.i * sd.stride + it.block * 128 + l * 8, out);
}

template <typename T> CacheRowsFn pick(bool quantize, bool wide) {
  if (quantize) return wide ? quant_rows_kernel<T, true> : quant_rows_kernel<T, false>;
  return wide ? dequant_rows_kernel<T, true> : dequant_rows_kernel<T, false>;
}

}  // namespace

CacheRowsFn cache_rows_form(int act, bool quantize, bool wide) {
  return act == PALU_F16 ? pick<F16>(quantize, wide) : pick<BF16>(quantize, wide);
}

}  // namespace palu
