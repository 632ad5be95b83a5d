// Rows of a quantized latent cache: quantized as they are written, and read back.  Both sides of a layer in one launch.
//
// 8 lanes take a block of 128 channels, 8 of either half each: twice 16 bytes of the latents, and 4, 3 or 2 bytes of codes.
//   write  s = f16((max - min) / (2^B - 1)), 0 -> 1;  z = f16(clamp(rint(-min / s)));  c = clamp(rint(x / s) + z, 0, 2^B - 1), every step one
//          float32 operation (ties to even): the numbers that quant_kernel writes
//   read   (c - z) * s, rounded once to the layer's type: exact in float32 for whole zero-points up to 2^12 (13 bits by 11), else a float32
//          number with its last bit set where it is inexact, which the second rounding cannot take for a tie (16384 bfloat16 rows of 4096 channels a
//          side whose zero-points have fractions: 85 us against 57)
// Bound by the memory, and writing by the vector unit beside it: a value is 2 bytes on one side and 1/2 + 1/32 on the other.  16384 rows of 4096 channels
// are read in 42 us, 16000 written in 39, 4.1 and 4.2 TB/s of the 5.1 of a copy.  (16 lanes a block, with the side's numbers indexed by lane: 70; chosen
// from registers: 54, bound by the address units, of which 8 lanes a block take half as many row numbers, scales and zero-points.  Two or four blocks per
// lane, all loads first: the same.)

#include "cache_rows.h"
#include "paged_dev.h"

namespace palu {

namespace {

// the larger / smaller of x over 8 lanes: lane ^ 1, ^ 2 in a quad, mirrored in 8 lanes
template <int CTRL> __device__ __forceinline__ float from_lane(float x) {
  const int u = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float max_over_8(float x) {
  x = fmaxf(x, from_lane<0xB1>(x));
  x = fmaxf(x, from_lane<0x4E>(x));
  return fmaxf(x, from_lane<0x141>(x));
}
__device__ __forceinline__ float min_over_8(float x) {
  x = fminf(x, from_lane<0xB1>(x));
  x = fminf(x, from_lane<0x4E>(x));
  return fminf(x, from_lane<0x141>(x));
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

// x + y in float32, with the last bit set where that is inexact: of the two neighbours the odd one.  (What the rounding leaves is a float32 number.)
__device__ __forceinline__ float sum_to_odd(float x, float y) {
  const float sum = x + y, back = sum - x, left = (x - (sum - back)) + (y - back);
  int u = __builtin_bit_cast(int, sum);
  if (fabsf(left) > 0.f && (u & 1) == 0) u += (u ^ __builtin_bit_cast(int, left)) >> 31 | 1;       // (towards what is left; not for what is not a number)
  return __builtin_bit_cast(float, u);
}

// Its side, chosen from registers (an index into the arguments, which differs by lane, would load them by lane)
__device__ __forceinline__ CacheSide side_of(const CacheRowsArgs& a, int s) {
  const CacheSide &k = a.side[0], &v = a.side[1];
  return CacheSide{s ? v.latent : k.latent, s ? v.codes : k.codes, s ? v.scale : k.scale, s ? v.zero : k.zero, s ? v.stride : k.stride,
                   s ? v.n_blocks : k.n_blocks, s ? v.bits : k.bits};
}
// The block of 128 channels that these 8 lanes take: of latent row `i`, `block` of side `s`
struct CacheItem {
  long long i, row;
  int s, block;
  bool valid;
  __device__ __forceinline__ CacheItem(const CacheRowsArgs& a) {
    const int per_row = a.side[0].n_blocks + a.side[1].n_blocks;
    const unsigned first = blockIdx.x * (unsigned)kCacheRowsItems;         // (the host keeps them below 2^32)
    const unsigned i0 = first / (unsigned)per_row;
    const int x = (int)(first - i0 * (unsigned)per_row) + (int)(threadIdx.x >> 3);
    const int q = (int)(((float)x + 0.5f) / (float)per_row);               // x / per_row: 1/2 per_row from a whole number at least
    i = (long long)i0 + q;
    block = x - q * per_row;
    s = block >= a.side[0].n_blocks;
    block -= s ? a.side[0].n_blocks : 0;
    row = i >= a.n ? -1 : (a.row ? (long long)a.row[i] : i);
    valid = row >= 0 && row < a.n_rows;
  }
};

template <typename T, bool WIDE>
__global__ __launch_bounds__(kCacheRowsThreads) void quant_rows_kernel(CacheRowsArgs a) {
  const int l = threadIdx.x & 7;
  const CacheItem it(a);
  if (!it.valid) return;                       // (all lanes of a block alike)
  const CacheSide sd = side_of(a, it.s);
  uint4v raw[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) raw[p] = load8<WIDE>(sd.latent + it.i * sd.stride + it.block * 128 + 64 * p + l * 8);
  float x[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t two = raw[e >> 2][e & 3];
    x[2 * e] = T::to_float((uint16_t)two);
    x[2 * e + 1] = T::to_float((uint16_t)(two >> 16));
  }
  float low = x[0], high = x[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) {
    low = fminf(low, x[e]);
    high = fmaxf(high, x[e]);
  }
  low = min_over_8(low);
  high = max_over_8(high);
  const float top = (float)((1 << sd.bits) - 1);
  uint16_t s16 = F16::from_float(__fdiv_rn(__fsub_rn(high, low), top));
  if ((s16 & 0x7fffu) == 0) s16 = 0x3c00u;
  const float s = F16::to_float(s16);
  const uint16_t z16 = F16::from_float(fminf(fmaxf(rintf(__fdiv_rn(-low, s)), -65504.f), 65504.f));
  const float z = F16::to_float(z16);
  // x / s to the nearest float32 number in three operations: q = x * r is off by 2.5 units in the last place at most, x - q s is exact (s has 11 bits),
  // and what the last fma rounds is off by 2^-21 units while no quotient of two 11-bit numbers lies within 2^-12 units of where the rounding turns.
  // (For a finite s and numbers below 2^60, where nothing overflows.  A quotient too small for this is 0 after rint anyway.)
  float q[16];
  if ((s16 & 0x7c00u) != 0x7c00u && fmaxf(fabsf(low), fabsf(high)) < 0x1p60f) {
    const float r = __builtin_amdgcn_rcpf(s);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float near = x[e] * r;
      q[e] = __builtin_fmaf(__builtin_fmaf(-near, s, x[e]), r, near);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) q[e] = __fdiv_rn(x[e], s);
  }
  const int R = sd.n_blocks * 128;
  uint8_t* codes = sd.codes + it.row * (long long)(R / 8 * sd.bits);
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    float c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = __builtin_amdgcn_fmed3f(__fadd_rn(rintf(q[8 * p + e]), z), 0.f, top);       // (0 for what is not a number)
    const int at = it.block * 16 + 8 * p + l;              // 8 channels
    if (sd.bits == 4) {
      uint32_t w[2];                           // four codes are a whole number below 2^16
#pragma unroll
      for (int k = 0; k < 2; ++k) w[k] = (uint32_t)__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[4 * k + 3], 16.f, c[4 * k + 2]), 16.f, c[4 * k + 1]), 16.f, c[4 * k]);
      reinterpret_cast<uint32_t*>(codes)[at] = w[0] | w[1] << 16;
    } else {
      uint32_t w = 0, third = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w |= ((uint32_t)c[e] & 3u) << (2 * e);
        third |= ((uint32_t)c[e] >> 2) << e;
      }
      reinterpret_cast<uint16_t*>(codes)[at] = (uint16_t)w;
      if (sd.bits == 3) codes[R / 4 + at] = (uint8_t)third;
    }
  }
  if (l == 0) {
    sd.scale[it.row * sd.n_blocks + it.block] = s16;
    sd.zero[it.row * sd.n_blocks + it.block] = z16;
  }
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(kCacheRowsThreads) void dequant_rows_kernel(CacheRowsArgs a) {
  const int l = threadIdx.x & 7;
  const CacheItem it(a);
  if (!it.valid) return;
  const CacheSide sd = side_of(a, it.s);
  const int R = sd.n_blocks * 128;
  const uint8_t* codes = sd.codes + it.row * (long long)(R / 8 * sd.bits);
  uint32_t w[2], third[2] = {0, 0};
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int at = it.block * 16 + 8 * p + l;
    w[p] = sd.bits == 4 ? reinterpret_cast<const uint32_t*>(codes)[at] : reinterpret_cast<const uint16_t*>(codes)[at];
    if (sd.bits == 3) third[p] = codes[R / 4 + at];
  }
  const uint16_t s16 = sd.scale[it.row * sd.n_blocks + it.block];
  // (c - z) s = c s - z s: both products are exact (15 and 22 bits), so one fma rounds the difference once, if at all
  const float s = F16::to_float(s16), z = F16::to_float(sd.zero[it.row * sd.n_blocks + it.block]), off = -(z * s);
  const bool infinite = (s16 & 0x7fffu) == 0x7c00u;          // (there the products' difference is not a number)
  const bool seldom = __any(infinite || !(fabsf(z) <= 4096.f && z == rintf(z)));
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const uint32_t c = sd.bits == 4 ? w[p] : expand_low_bits(w[p], third[p], sd.bits == 3);
    const uint32_t even = c & 0x0f0f0f0fu, odd = (c >> 4) & 0x0f0f0f0fu;
    uint4v out;
    if (!seldom) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c0 = (float)((even >> (8 * e)) & 255u), c1 = (float)((odd >> (8 * e)) & 255u);
        out[e] = pack2<T>(__builtin_fmaf(c0, s, off), __builtin_fmaf(c1, s, off));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c0 = (float)((even >> (8 * e)) & 255u), c1 = (float)((odd >> (8 * e)) & 255u);
        out[e] = pack2<T>(infinite ? (c0 - z) * s : sum_to_odd(c0 * s, off), infinite ? (c1 - z) * s : sum_to_odd(c1 * s, off));
      }
    }
    store8<WIDE>(sd.latent + it.i * sd.stride + it.block * 128 + 64 * p + l * 8, out);
  }
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
