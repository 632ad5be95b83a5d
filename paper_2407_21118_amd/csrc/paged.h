// What the host side and the kernels of attention over a paged latent cache share (paged.hip).
#pragma once

#include "palu_dev.h"

namespace palu {

constexpr int kPagedTile = 32;                 // tokens per tile: positions 32 i .. 32 i + 31
constexpr int kPagedThreads = 512;             // eight wavefronts, two per SIMD

// Layer metadata; heads are KEY/VALUE heads here.  Everything indexed by the group is 32 bits wide: beside an array of 16-bit
// numbers with the same index the compiler addresses these from a base that lies on no whole word, and scalar loads drop its low bits.
struct PagedMeta {
  int n_heads;
  int n_groups;
  int qpk;                                     // query heads per key/value head
  int k_off[PALU_MAX_GROUPS + 1];
  int v_off[PALU_MAX_GROUPS + 1];
  int bk_off[PALU_MAX_GROUPS + 1];             // element offset of group j inside the concatenated B_k
  int bv_off[PALU_MAX_GROUPS + 1];
  int o_off[PALU_MAX_GROUPS];                  // value ranks of all heads before group j, summed: where its partial results begin
  int head_off[PALU_MAX_GROUPS + 1];
  uint8_t group_of_head[PALU_MAX_HEADS];
};

// Rows that a sequence of L rows attends: t < sink and lo <= t < L, in tiles 0 .. sink_tiles - 1 and from tile0 on.
struct PagedSpan {
  int sink, lo, sink_tiles, tile0, n_tiles;
};
// first: rows before it belong to the shared prefix and are attended elsewhere (no window, no sinks then)
__host__ __device__ __forceinline__ PagedSpan paged_span(int L, int first, int window, int n_sink) {
  PagedSpan s;
  s.lo = first;
  s.sink = 0;
  if (window > 0 && L - window > n_sink) {     // else the window reaches the first rows: everything is attended
    s.lo = L - window;
    s.sink = n_sink;
  }
  s.sink_tiles = (s.sink + kPagedTile - 1) / kPagedTile;
  s.tile0 = s.lo / kPagedTile;
  if (s.tile0 < s.sink_tiles) s.tile0 = s.sink_tiles;
  const int end = (L + kPagedTile - 1) / kPagedTile;
  s.n_tiles = L <= s.lo ? 0 : s.sink_tiles + (end > s.tile0 ? end - s.tile0 : 0);
  return s;
}

// A unit: up to four adjacent key/value heads whose keys one workgroup rebuilds, of one group or of several adjacent ones
// of equal ranks and size, whose latents lie side by side.
struct PagedUnit {
  uint32_t bits;                               // first head | heads << 8 | group of the first << 16 | groups << 24
  __host__ __device__ int h0() const { return bits & 255; }
  __host__ __device__ int nh() const { return (bits >> 8) & 255; }
  __host__ __device__ int group() const { return (bits >> 16) & 255; }
  __host__ __device__ int n_groups() const { return bits >> 24; }
};

constexpr int kPagedProbPitch = 144;           // bytes per row of probabilities: a tile's hi, its lo and 16 bytes
constexpr int kPagedScorePitch = 20;           // floats per row of scores: 16 tokens and 16 bytes
constexpr int kPagedAngPitch = kDHead + 4;     // floats per token of angles
constexpr int kPagedMaxStages = 6;
constexpr int kPagedAnchorTiles = 8;           // every so many tiles the angles come from the table
constexpr int kPagedLdsBytes = 160 * 1024;     // of a compute unit

// One barrier per tile, or one per half of a tile where two tiles' scores, angles and probabilities leave no LDS for two stages of wide rows
__host__ __device__ constexpr bool paged_whole(int parts, int row_tiles) { return parts == 2 && row_tiles != 2; }

// LDS of a workgroup, in bytes from its start.  Tiles are staged n_stages deep, rows in 16-byte pieces, as many of them as a power
// of two (at least 8, of values 16).  Queries lie where scores and probabilities come later.
struct PagedLds {
  int k_pieces, v_pieces;
  int slots;                                   // tiles whose tokens' rows of the cache and whose first angles are held; of page-table entries: twice as many
  int q_pitch;                                 // bytes per packed query row
  int stage_k, stage_v;                        // bytes per staged tile
  int k, v, anchors, entries, rows, ang, alpha, s, p, q, total;
};
// n_groups groups of the unit, ks steps of 32 key channels each; rows: packed query rows, in row_tiles tiles of 16; parts: partial scores
// that are added up
__host__ __device__ __forceinline__ PagedLds paged_lds(int n_groups, int ks, int v_cols, int rows, int row_tiles, int parts, int n_stages) {
  PagedLds l;
  const int k_pieces = n_groups * ks * 4;
  l.k_pieces = k_pieces <= 8 ? 8 : (k_pieces <= 16 ? 16 : (k_pieces <= 32 ? 32 : 64));
  l.v_pieces = v_cols <= 128 ? 16 : (v_cols <= 256 ? 32 : 64);
  l.q_pitch = kDHead * 2 * 2 + 16;             // pairs
  l.stage_k = kPagedTile * l.k_pieces * 16;
  l.stage_v = kPagedTile * l.v_pieces * 16;
  l.slots = n_stages <= 3 ? 4 : 8;
  l.k = 0;
  l.v = l.k + n_stages * l.stage_k;
  l.anchors = l.v + n_stages * l.stage_v;
  l.entries = l.anchors + l.slots * kDHead * 4;
  l.rows = l.entries + 2 * l.slots * kPagedTile * 4;
  l.ang = l.rows + l.slots * kPagedTile * 4;
  const int held = paged_whole(parts, row_tiles) ? 2 : 1;    // tiles whose angles and probabilities are held
  l.alpha = l.ang + held * kPagedTile * kPagedAngPitch * 4;
  l.p = l.alpha + held * row_tiles * 16 * 4;
  l.s = l.p + held * (row_tiles * 16 + 1) * kPagedProbPitch;
  l.total = l.s + (held == 2 ? 4 : 3) * parts * (rows + 1) * kPagedScorePitch * 4;
  l.q = l.p;
  const int q_end = l.q + rows * l.q_pitch;
  if (l.total < q_end) l.total = q_end;
  return l;
}

// Tokens that are attended in the same way: every sequence's own, or the shared prefix's.
struct PagedPart {
  float* o_part;                               // [slot][rows * sum of value ranks over the heads]: sums of exp2(score - max) * latent, times kProbScale
  float* ml_part;                              // [slot][head][row][2]: the maximum and the sum, times kProbScale
  long long o_stride;                          // floats of o_part per slot
  int max_len, first, window, n_sink;
  int shared;                                  // the tokens are those of the shared prefix
  int rows;                                    // query rows per key/value head: qpk, or batch * qpk where the tokens are shared
  int n_row_blocks, block_rows;
  int chunk_tiles;                             // tiles per workgroup, at most
  int n_slots;                                 // partial results per sequence, or of the shared tokens
};

struct PagedArgs {
  const uint16_t* hk;                          // [n_pages * page_rows, R_k]
  const uint16_t* hv;
  const uint16_t* q;                           // [batch, n_heads * qpk, 128], before RoPE
  const uint16_t* Bk;
  const float* rope;                           // angle table, layout in palu_dev.h
  const int32_t* q_pos;                        // [batch] or NULL: the newest row's
  const int32_t* page_table;                   // [batch, table_stride]
  const int32_t* seq_lens;                     // [batch] or NULL: pos_len
  long long R_k, R_v;
  int n_pages, page_shift, table_stride, rope_len;
  int pos_len;                                 // rows of a sequence where seq_lens is NULL, else at most
  int n_units;
  int n_stages;                                // tiles staged in LDS
  int max_packed;                              // packed query rows that LDS is laid out for (more than 16: as many as accumulators go)
  int n_first;                                 // workgroups of part 0; those behind them are part 1's
  float scale;                                 // log2(e) / sqrt(128)
  PagedPart part[2];
  PagedMeta meta;
  PagedUnit units[PALU_MAX_HEADS];
};
static_assert(sizeof(PagedArgs) <= 4096, "kernel arguments");

struct PagedMergeArgs {
  const float* o_part;                         // the sequences' own partial results ...
  const float* ml_part;
  const float* o_shared;                       // ... and those of the shared tokens (n_shared slots)
  const float* ml_shared;
  const uint16_t* Bv;
  const int32_t* seq_lens;
  uint16_t* out;                               // [batch, n_heads * qpk, 128]
  int max_len, first, window, n_sink;
  int batch;
  int chunk_tiles, n_slots, n_shared;
  long long o_stride, o_shared_stride;
  PagedMeta meta;
};

using PagedFn = void (*)(PagedArgs);
// The instantiations, by ks: steps of 32 key channels, 2, 4, 6, 8 (units of up to four heads), 12 or 16 (of two); vb: blocks of 256 value
// columns; many: more than 16 packed query rows, up to 16 per head
struct PagedForm {
  int ks, vb;
  bool many;
  int parts() const { return ks > 8 ? 4 : 2; }           // wavefronts that share a head's features
  int unit_heads() const { return 8 / parts(); }
  int row_tiles() const { return many ? (vb == 1 ? 4 : 2) : 1; }
  int max_rows() const { return 16 * row_tiles(); }      // packed
};
template <typename T> PagedFn paged_form(const PagedForm& f);
using PagedMergeFn = void (*)(PagedMergeArgs);
// rows: of one key/value head per workgroup, 1, 2, 4 or 8
template <typename T> PagedMergeFn paged_merge_form(int rows);

}  // namespace palu
