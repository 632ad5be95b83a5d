// What the host side and the kernels of attention over a paged 4-bit latent cache share (pagedq.hip).
#pragma once

#include "paged.h"

namespace palu {

struct PagedQSide {
  const uint8_t* codes;      // [n_pages * page_rows, R / 2]
  const uint16_t* scale;     // float16 [n_pages * page_rows, R / 128]
  const uint16_t* zero;
  int row_bytes, n_blocks;   // R / 2, R / 128
};
struct PagedQArgs {
  PagedQSide k, v;
  const uint16_t* q;         // [batch, n_heads * qpk, 128], before RoPE
  const uint16_t* Bk;
  const float* rope;         // angle table, layout in palu_dev.h
  const int32_t* q_pos;      // [batch] or NULL: the newest row's
  const int32_t* page_table; // [batch, table_stride]
  const int32_t* seq_lens;   // [batch] or NULL: max_len
  float* o_part;             // partial results as in PagedPart, rows per head: meta.qpk
  float* ml_part;
  long long o_stride;
  int n_pages, page_shift, table_stride, rope_len;
  int max_len, window, n_sink;
  int chunk_tiles, n_slots;
  float scale;               // log2(e) / sqrt(128)
  PagedMeta meta;
};
static_assert(sizeof(PagedQArgs) <= 4096, "kernel arguments");
using PagedQFn = void (*)(PagedQArgs);
constexpr int kPagedQThreads = 256;
PagedQFn pagedq_plain_form(int act);

}  // namespace palu
