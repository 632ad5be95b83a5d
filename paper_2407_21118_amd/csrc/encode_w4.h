// What the host side and the kernels of the projection from 4-bit weights share (encode_w4.hip).
#pragma once

#include "palu_dev.h"

namespace palu {

struct EncodeW4Side {
  const uint8_t* codes;      // [R, d / 2]
  const uint16_t* scale;     // float16 [R, d / 128]
  const uint16_t* zero;
  uint16_t* latent;
  long long stride;          // elements between latent rows
  int tiles;                 // workgroups side by side: R / 16 / columns
};
struct EncodeW4Args {
  EncodeW4Side side[2];
  const uint16_t* x;         // [n_tok, d]
  const int32_t* dst_row;    // or NULL: row t
  int n_tok, d;
};
using EncodeW4Fn = void (*)(EncodeW4Args);
constexpr int kW4Threads = 512;
// Blocks of 16 tokens and of 16 columns that a workgroup takes: 1 or 2 by 1, 2 by 4
struct EncodeW4Form {
  int tokens, columns;
};
EncodeW4Fn encode_w4_form(int act, const EncodeW4Form& f);

}  // namespace palu
