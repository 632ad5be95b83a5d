// What the host side and the kernels that move whole rows of a quantized latent cache share (cache_rows.hip).
#pragma once

#include "palu_dev.h"

namespace palu {

struct CacheSide {
  uint16_t* latent;          // rows of the layer's type: read when quantizing, written when reading back
  uint8_t* codes;            // rows of R * bits / 8 bytes
  uint16_t* scale;           // float16, rows of n_blocks
  uint16_t* zero;
  long long stride;          // elements between latent rows
  int n_blocks;              // blocks of 128 channels, 0: this side takes no part
  int bits;                  // 4, 3 or 2
};
struct CacheRowsArgs {
  CacheSide side[2];
  const int32_t* row;        // cache row of latent row i, or NULL: i; outside [0, n_rows): latent row i is left out
  long long n;               // latent rows
  long long n_rows;          // rows of the cache
};
using CacheRowsFn = void (*)(CacheRowsArgs);
// wide: latent rows begin on whole 16 bytes
CacheRowsFn cache_rows_form(int act, bool quantize, bool wide);
constexpr int kCacheRowsThreads = 256, kCacheRowsItems = kCacheRowsThreads / 8;          // workgroup; blocks (of 8 threads each) that it takes

}  // namespace palu
