// What the host side and the kernels of attention over a paged 4-bit latent cache share (pagedq_fold.hip and, for angles that turn too fast, pagedq.hip).
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
constexpr int kPagedQLow = 32;                 // rotation pairs from this one on are folded with the query (pagedq_fold.hip)
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
// The instantiations, by ks: steps of 32 key channels of a wavefront, 4 or 8; slices: parts of a head's channels (2: ranks above 256); rows: query
// rows of a head, 1 or 2; k_blocks, v_blocks: of 128 key and value columns of a unit, at most
struct PagedQForm {
  int ks, slices, rows, k_blocks, v_blocks;
};
constexpr int kPagedQMaxClasses = 8;
template <int ROWS> PagedQFn pagedq_rows_form(int act, const PagedQForm& f);
template <> PagedQFn pagedq_rows_form<1>(int, const PagedQForm&);
template <> PagedQFn pagedq_rows_form<2>(int, const PagedQForm&);
inline PagedQFn pagedq_form(int act, const PagedQForm& f) {
  return f.rows == 1 ? pagedq_rows_form<1>(act, f) : pagedq_rows_form<2>(act, f);
}

constexpr int kPagedQFoldThreads = 512;        // of pagedq_kernel

// Whether an interval has two parts with a barrier between: one step's keys in LDS at a time, weights and values a step earlier (pagedq_kernel)
__host__ __device__ constexpr bool pagedq_two_phases(int slices, int rows, int v_blocks) { return slices == 2 || (rows > 1 && v_blocks == 4); }

__host__ __device__ constexpr int pagedq_key_scales(int ks, int k_blocks) { return k_blocks * 4 / ks; }

// LDS of a workgroup, in bytes from its start
struct PagedQLds {
  int k_pitch;               // bytes per staged key row: float16 numbers
  int k_size, v_size;        // of a step's keys, raw value codes
  int k, v, p, p_cb, p_size, alpha, k_tok, k_zero, v_tok, basis, anchors, rows, scores, nodes, turns, q, stage, flags, total;
};
constexpr int kPagedQProbPitch = kPagedQStep * 2 + 16, kPagedQTurnPitch = 2 * kPagedQLow * 4 + 16;
__host__ __device__ constexpr PagedQLds pagedq_lds(const PagedQForm& f) {
  PagedQLds l = {};
  const bool two = pagedq_two_phases(f.slices, f.rows, f.v_blocks);
  const int p_rows = 8 * f.rows;
  l.k_pitch = 256 * f.k_blocks;
  l.k_size = kPagedQStep * l.k_pitch;
  l.v_size = kPagedQStep * 64 * f.v_blocks;
  l.p_cb = p_rows * kPagedQProbPitch;          // probabilities of a block of value columns
  l.p_size = f.v_blocks * l.p_cb;
  // (the small ones first, within the 64 KiB that an instruction's offset reaches)
  l.alpha = 0;                                 // [2][blocks][16]
  l.k_tok = l.alpha + 2 * f.v_blocks * 16 * 4; // [4][slices or groups][64]: ratio and scale
  l.k_zero = l.k_tok + kPagedQStep * 4 * pagedq_key_scales(f.ks, f.k_blocks) * 8;      // [4][blocks][64]: the zero-point for the codes, what is left of it
  l.v_tok = l.k_zero + kPagedQStep * 4 * f.k_blocks * 4;       // [4][blocks][64]: scale, zero-point
  l.anchors = l.v_tok + kPagedQStep * 4 * f.v_blocks * 4;      // [4]
  l.rows = l.anchors + 4 * kDHead * 4;                 // [8][64]
  l.scores = l.rows + 8 * kPagedQStep * 4;             // [2 or 1][heads * rows][parts][64]
  l.nodes = l.scores + (two ? 1 : 2) * (4 / f.slices) * f.rows * (2 * f.slices) * kPagedQStep * 4;
  l.turns = l.nodes + kPagedQNodes * kPagedQTurnPitch; // cos and sin of the folded pairs from a span's begin to its nodes
  l.q = l.turns + 16 * kPagedQTurnPitch;               // of the others from a sub-tile's begin to its tokens
  l.stage = l.q + (4 / f.slices) * f.rows * kDHead * 4;        // [heads * rows][128]
  l.flags = l.stage + (2 * f.k_blocks + 2 * f.v_blocks + 1) * kPagedQStep * 4;         // scales and zero-points, page entries on their way
  l.basis = l.flags + 16;
  l.p = l.basis + kPagedQSpan * kPagedQNodes * 4;
  l.v = l.p + 2 * l.p_size;
  l.k = l.v + (two ? 2 : 3) * l.v_size;
  l.total = l.k + (two ? 1 : 2) * l.k_size;
  return l;
}

}  // namespace palu
