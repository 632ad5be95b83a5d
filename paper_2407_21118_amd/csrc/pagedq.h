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
constexpr int kPagedQStep = 64;                // tokens per step: two tiles
constexpr int kPagedQLow = 32;                 // rotation pairs from this one on are folded with the query (pagedq.hip)
constexpr int kPagedQNodes = 8;                // positions at which they are
constexpr int kPagedQSpan = 256;               // positions between two foldings, at most

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
  int n_units, n_row_blocks; // pagedq_kernel: units, blocks of query rows of a head
  int span_steps;            // steps between two foldings
  float scale;               // log2(e) / sqrt(128)
  float w_low[kDHead / 2 - kPagedQLow];        // radians per position of the folded pairs
  PagedMeta meta;
  PagedUnit units[PALU_MAX_HEADS];
};
static_assert(sizeof(PagedQArgs) <= 4096, "kernel arguments");
using PagedQFn = void (*)(PagedQArgs);
constexpr int kPagedQThreads = 256;
PagedQFn pagedq_plain_form(int act);
// The instantiations, by ks: steps of 32 key channels of a wavefront, 4 or 8; slices: wavefronts that share a head's channels (2: ranks above
// 256); rows: query rows of a head, 1, 2 or 4; piped: several steps at work at once, where LDS holds what that takes, for k_blocks and v_blocks blocks
// of 128 key and value columns of a unit (else up to 2 * slices and 4)
struct PagedQForm {
  int ks, slices, rows, k_blocks, v_blocks, piped;
};
constexpr int kPagedQPipedBlocks = 3, kPagedQPipedRows = 2;
template <int ROWS> PagedQFn pagedq_rows_form(int act, const PagedQForm& f);
template <> PagedQFn pagedq_rows_form<1>(int, const PagedQForm&);
template <> PagedQFn pagedq_rows_form<2>(int, const PagedQForm&);
template <> PagedQFn pagedq_rows_form<4>(int, const PagedQForm&);
inline PagedQFn pagedq_form(int act, const PagedQForm& f) {
  return f.rows == 1 ? pagedq_rows_form<1>(act, f) : (f.rows == 2 ? pagedq_rows_form<2>(act, f) : pagedq_rows_form<4>(act, f));
}

// LDS of a workgroup, in bytes from its start
struct PagedQLds {
  int k_pitch;               // bytes per staged key row: k_cols float16 numbers
  int k_size, raw_size, v_size;                // of a step's keys, raw key codes, raw value codes
  int k, raw, v, p, p_cb, p_size, alpha, k_tok, k_zero, v_tok, basis, anchors, rows, scores, flags, total;
};
constexpr int kPagedQProbPitch = kPagedQStep * 2 + 16;
__host__ __device__ constexpr PagedQLds pagedq_lds(int k_cols, int v_cols, int slices, int rows, bool piped) {
  PagedQLds l = {};
  const int blocks = v_cols / 128, bufs = piped ? 2 : 1, p_rows = rows == 1 ? 8 : (slices == 1 ? 32 : 16);
  l.k_pitch = k_cols * 2;
  l.k_size = kPagedQStep * l.k_pitch;
  l.raw_size = kPagedQStep * k_cols / 2;
  l.v_size = kPagedQStep * v_cols / 2;
  l.k = 0;
  l.raw = l.k + bufs * l.k_size;
  l.v = l.raw + bufs * l.raw_size;
  l.p = l.v + (piped ? 3 : 2) * l.v_size;
  l.p_cb = p_rows * kPagedQProbPitch;          // probabilities of a block of value columns
  l.p_size = blocks * l.p_cb;
  l.alpha = l.p + 2 * l.p_size;                // [2][blocks][16]
  l.k_tok = l.alpha + 2 * blocks * 16 * 4;     // [4][2][64]: ratio and scale, by slice or group
  l.k_zero = l.k_tok + kPagedQStep * 4 * 2 * 8;        // [4][4][64]: the zero-point for the codes, what is left of it
  l.v_tok = l.k_zero + kPagedQStep * 4 * 4 * 4;        // [4][blocks][64]: scale, zero-point
  l.basis = l.v_tok + kPagedQStep * 4 * blocks * 4;
  l.anchors = l.basis + kPagedQSpan * kPagedQNodes * 4;        // [4]
  l.rows = l.anchors + 4 * kDHead * 4;                 // [8][64]
  l.scores = l.rows + 8 * kPagedQStep * 4;
  l.flags = l.scores + (slices == 1 ? 0 : 2 * rows * kPagedQStep * 4);
  l.total = l.flags + 16;
  return l;
}

__host__ __device__ constexpr PagedQLds pagedq_lds(int ks, int slices, int rows, int k_blocks, int v_blocks, bool piped) {
  return pagedq_lds(128 * (piped ? k_blocks : 2 * slices), 128 * (piped ? v_blocks : 4), slices, rows, piped);
}

}  // namespace palu
