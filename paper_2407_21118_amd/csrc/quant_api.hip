// Host side of what a layer with a 4-bit paged cache and 4-bit projections takes beside the other entry points: rows quantized and read
// back, the projection, attention (part of the translation unit api.hip).

#include "cache_rows.h"
#include "encode_w4.h"
#include "pagedq.h"

namespace {

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int cache_rows_impl(const palu_layer_desc* desc, bool quantize, const void* hk, int64_t hk_stride, const void* hv, int64_t hv_stride, int64_t n_tok,
                    const uint8_t* k_codes, const void* k_scale, const void* k_zero, const uint8_t* v_codes, const void* v_scale,
                    const void* v_zero, int64_t n_rows, const int32_t* row, void* stream) {
  Meta m;
  const int st = check_desc(desc, &m, 1, true);
  if (st != PALU_OK) return st;
  if (n_tok < 0 || n_rows <= 0 || n_rows > 0x7fffffffLL || !aligned(row, 4)) return PALU_ERR_INVALID_ARG;
  CacheRowsArgs a;
  std::memset(&a, 0, sizeof(a));
  bool wide = true;
  for (int s = 0; s < 2; ++s) {
    const int bits = latent_bits(s ? desc->v_latent_dtype : desc->k_latent_dtype);
    if (bits == 0) continue;
    const int R = s ? m.v_off[m.n_groups] : m.k_off[m.n_groups];
    const void *latent = s ? hv : hk, *codes = s ? v_codes : k_codes, *scale = s ? v_scale : k_scale, *zero = s ? v_zero : k_zero;
    const int64_t stride = s ? hv_stride : hk_stride;
    if ((!latent && n_tok > 0) || !codes || !scale || !zero || stride < R) return PALU_ERR_INVALID_ARG;   // (of no rows: whatever stands for them)
    if (!aligned(latent, 2) || !aligned(codes, 4) || !aligned(scale, 2) || !aligned(zero, 2)) return PALU_ERR_INVALID_ARG;
    wide = wide && aligned(latent, 16) && stride % 8 == 0;
    a.side[s] = CacheSide{(uint16_t*)latent, (uint8_t*)codes, (uint16_t*)scale, (uint16_t*)zero, stride, R / 128, bits};
  }
  if (a.side[0].n_blocks + a.side[1].n_blocks == 0) return PALU_ERR_INVALID_ARG;
  if (n_tok == 0) return PALU_OK;
  a.row = row;
  a.n = n_tok;
  a.n_rows = n_rows;
  const long long items = n_tok > (1LL << 32) ? 1LL << 62 : (long long)n_tok * (a.side[0].n_blocks + a.side[1].n_blocks);
  if (items > (0xffffffffLL - 2 * kCacheRowsThreads) / 16) return PALU_ERR_UNSUPPORTED;      // work items of a launch
  hipLaunchKernelGGL(cache_rows_form(desc->act_dtype, quantize, wide), dim3((unsigned)((items + kCacheRowsItems - 1) / kCacheRowsItems)),
                     dim3(kCacheRowsThreads), 0, static_cast<hipStream_t>(stream), a);
  return launch_ok();
}

// Units that one launch takes: key/value heads whose keys have the same form.
struct PagedQClass {
  PagedQForm form;
  int lds_bytes, n_units;
  PagedUnit units[PALU_MAX_HEADS];
};
// (key ranks of 128, in one group or two, 256, above; one or two, three or four value blocks)
static_assert(kPagedQMaxClasses == 4 * 2, "classes");
struct PagedQCall {
  PagedMeta meta;
  int n_sink, max_tiles, chunk_tiles, n_slots;
  int span_steps;                              // 0: the plain kernel
  int n_cls, n_row_blocks;
  PagedQClass cls[kPagedQMaxClasses];
  long long o_stride;
  size_t ml_at, total;
};

// The largest span over which the folded pairs, of which the fastest turns theta^(-1/2) a position, turn by 1.3 radians either way from its middle
// (their polynomials of degree 7 are then right to 2e-6); 0: not even one step's
int pagedq_span_steps(float theta) {
  const double w = theta > 0.f ? 1.0 / std::sqrt((double)theta) : 0.0;
  for (int steps = kPagedQSpan / kPagedQStep; steps > 0; steps /= 2)
    if (w * (0.5 * kPagedQStep * steps) <= 1.3) return steps;
  return 0;
}

int plan_pagedq(const palu_layer_desc* desc, int batch, int max_len, int window, int n_sink, PagedQCall* c) {
  int st = check_paged_desc(desc, &c->meta, true);
  if (st != PALU_OK) return st;
  if (batch <= 0 || max_len <= 0 || window < 0 || n_sink < 0) return PALU_ERR_INVALID_ARG;
  if (batch > 65535 || max_len > (1 << 30)) return PALU_ERR_UNSUPPORTED;
  c->n_sink = window > 0 ? n_sink : 0;
  c->max_tiles = paged_max_tiles(max_len, 0, window, c->n_sink);
  const PagedMeta& m = c->meta;
  auto rk = [&](int j) { return m.k_off[j + 1] - m.k_off[j]; };
  auto rv = [&](int j) { return m.v_off[j + 1] - m.v_off[j]; };
  auto heads = [&](int j) { return m.head_off[j + 1] - m.head_off[j]; };
  long long sum_rv = 0, units = 0;
  for (int j = 0; j < m.n_groups; ++j) sum_rv += (long long)heads(j) * rv(j);
  c->o_stride = sum_rv * m.qpk;
  c->span_steps = pagedq_span_steps(desc->rope_theta);
  c->n_cls = 0;
  // (four rows at a time do not fit the registers: 4 x 16384 rows of four query rows a head took 178 us against 120 in two passes)
  const int rows = std::min(m.qpk, 2);
  c->n_row_blocks = ceil_div(m.qpk, rows);
  // Units, as for unquantized latents: whole adjacent groups side by side, or parts of one
  auto side_by_side = [&](int j, int unit_heads) {           // groups from j on
    int n = 1;
    while (j + n < m.n_groups && rk(j + n) == rk(j) && rv(j + n) == rv(j) && heads(j + n) == heads(j) && (n + 1) * heads(j) <= unit_heads &&
           (n + 1) * rk(j) <= 256 && (n + 1) * rv(j) <= 256)
      ++n;
    return n;
  };
  for (int first = 0, more = c->span_steps > 0; more; first += 4) {      // heads of a group (or of groups side by side) from `first` on
    more = 0;
    for (int j = 0, n; j < m.n_groups; j += n) {
      PagedQForm f{rk(j) == 128 ? 4 : 8, rk(j) > 256 ? 2 : 1, rows, 0, 0};
      n = side_by_side(j, 4 / f.slices);
      f.k_blocks = f.slices == 2 ? 4 : n * rk(j) / 128;
      f.v_blocks = std::max(2, n * rv(j) / 128 + (n * rv(j) / 128 == 3));      // 2 or 4
      PagedQClass* cl = nullptr;
      for (int k = 0; k < c->n_cls; ++k)
        if (std::memcmp(&c->cls[k].form, &f, sizeof(f)) == 0) cl = &c->cls[k];
      for (int h = first; h < std::min(first + 4, n * heads(j)); h += 4 / f.slices) {
        if (!cl) {
          cl = &c->cls[c->n_cls++];
          std::memset(cl, 0, sizeof(*cl));
          std::memcpy(&cl->form, &f, sizeof(f));
          cl->lds_bytes = pagedq_lds(f).total;
          if (cl->lds_bytes > kPagedLdsBytes) return PALU_ERR_UNSUPPORTED;
        }
        const int nh = std::min(4 / f.slices, n * heads(j) - h);
        cl->units[cl->n_units++].bits = (uint32_t)(m.head_off[j] + h) | (uint32_t)nh << 8 | (uint32_t)j << 16 | (uint32_t)n << 24;
        ++units;
      }
      more = more || first + 4 < n * heads(j);
    }
  }
  const int cus = device_cu_count();
  if (c->span_steps == 0) {
    const long long wgs = (long long)batch * m.n_heads;
    const int slots = (int)std::max<long long>(1, std::min<long long>(c->max_tiles, 4LL * cus / wgs));
    c->chunk_tiles = ceil_div(c->max_tiles, slots);
  } else {
    // Tiles per workgroup: one is resident per compute unit; its start and end are priced as eight tiles, a slot more is merged in a twentieth
    const long long wgs = (long long)batch * units * c->n_row_blocks;
    const long long most = std::min<long long>(1024, std::max<long long>(16, 4LL * cus / wgs));
    double best = 1e300;
    for (int n = 1; n <= std::min<long long>(ceil_div(c->max_tiles, 2), most); ++n) {
      const int tiles = ceil_div(ceil_div(c->max_tiles, n), 2) * 2, used = ceil_div(c->max_tiles, tiles);
      if (best < 1e300 && wgs * used * kPagedQFoldThreads > 0xffffffffLL) break;           // (work items of a launch)
      const double cost = paged_makespan(wgs * used, 8.0 + tiles, 0, 8.0 + tiles, cus) + 0.05 * used;
      if (cost >= best) continue;
      best = cost;
      c->chunk_tiles = tiles;
    }
  }
  c->n_slots = ceil_div(c->max_tiles, c->chunk_tiles);
  c->ml_at = align_up((size_t)batch * c->n_slots * c->o_stride * sizeof(float));
  c->total = c->ml_at + align_up((size_t)batch * c->n_slots * m.qpk * m.n_heads * 2 * sizeof(float));
  const long long launched = (long long)batch * c->n_slots * (c->span_steps ? units * c->n_row_blocks : m.n_heads);
  if (launched * kPagedQFoldThreads > 0xffffffffLL) return PALU_ERR_UNSUPPORTED;
  return PALU_OK;
}

}  // namespace

extern "C" {

int palu_quant_latent_kv(const palu_layer_desc* desc, const void* hk, int64_t hk_row_stride_elems, const void* hv, int64_t hv_row_stride_elems,
                         int64_t n_tok, uint8_t* k_codes, void* k_scale, void* k_zero, uint8_t* v_codes, void* v_scale, void* v_zero,
                         int64_t n_rows, const int32_t* dst_row, void* stream) {
  return cache_rows_impl(desc, true, hk, hk_row_stride_elems, hv, hv_row_stride_elems, n_tok, k_codes, k_scale, k_zero, v_codes, v_scale,
                         v_zero, n_rows, dst_row, stream);
}

int palu_dequant_latent_kv(const palu_layer_desc* desc, const uint8_t* k_codes, const void* k_scale, const void* k_zero, const uint8_t* v_codes,
                           const void* v_scale, const void* v_zero, int64_t n_rows, const int32_t* src_row, int64_t n_tok, void* hk,
                           int64_t hk_row_stride_elems, void* hv, int64_t hv_row_stride_elems, void* stream) {
  return cache_rows_impl(desc, false, hk, hk_row_stride_elems, hv, hv_row_stride_elems, n_tok, k_codes, k_scale, k_zero, v_codes, v_scale,
                         v_zero, n_rows, src_row, stream);
}

int palu_encode_kv_w4(const palu_layer_desc* desc, const void* x, int32_t n_tok, const uint8_t* Akt, const void* Ak_scale, const void* Ak_zero,
                      const uint8_t* Avt, const void* Av_scale, const void* Av_zero, void* hk, int64_t hk_row_stride_elems, void* hv,
                      int64_t hv_row_stride_elems, const int32_t* dst_row, void* stream) {
  Meta m;
  const int st = check_desc(desc, &m, 1, true);
  if (st != PALU_OK) return st;
  if (n_tok < 0 || !Akt || !Ak_scale || !Ak_zero || !Avt || !Av_scale || !Av_zero) return PALU_ERR_INVALID_ARG;
  if (n_tok > 0 && (!x || !hk || !hv)) return PALU_ERR_INVALID_ARG;            // (of no tokens: whatever stands for them)
  if (!aligned(x, 16) || !aligned(Akt, 16) || !aligned(Avt, 16) || !aligned(dst_row, 4)) return PALU_ERR_INVALID_ARG;
  for (const void* p : {Ak_scale, Ak_zero, Av_scale, Av_zero, (const void*)hk, (const void*)hv})
    if (!aligned(p, 2)) return PALU_ERR_INVALID_ARG;
  const int Rk = m.k_off[m.n_groups], Rv = m.v_off[m.n_groups];
  if (hk_row_stride_elems < Rk || hv_row_stride_elems < Rv) return PALU_ERR_INVALID_ARG;
  if (n_tok == 0) return PALU_OK;
  // 16 columns a workgroup, or 64 where that is faster: a round of workgroups over the compute units takes 5.5 us with 16 and 12.5 with 64 columns of
  // 4096 inputs.  (128 tokens of 4096 columns: 23 against 14 us; 32: 6.5 against 12.6.)
  EncodeW4Form f{n_tok <= 16 ? 1 : 2, 1};
  const long long blocks = ((long long)n_tok + 16 * f.tokens - 1) / (16 * f.tokens);
  const long long cus = device_cu_count(), tiles = blocks * ((Rk + Rv) / 16);
  if (Rk % 64 == 0 && Rv % 64 == 0 && f.tokens == 2 && 4 * ((tiles + cus - 1) / cus) > 9 * ((tiles / 4 + cus - 1) / cus)) f.columns = 4;
  EncodeW4Args a;
  std::memset(&a, 0, sizeof(a));
  a.side[0] = EncodeW4Side{Akt, (const uint16_t*)Ak_scale, (const uint16_t*)Ak_zero, (uint16_t*)hk, hk_row_stride_elems, Rk / (16 * f.columns)};
  a.side[1] = EncodeW4Side{Avt, (const uint16_t*)Av_scale, (const uint16_t*)Av_zero, (uint16_t*)hv, hv_row_stride_elems, Rv / (16 * f.columns)};
  a.x = static_cast<const uint16_t*>(x);
  a.dst_row = dst_row;
  a.n_tok = n_tok;
  a.d = m.n_heads * PALU_D_HEAD;
  if (blocks * kW4Threads > 0xffffffffLL) return PALU_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(encode_w4_form(desc->act_dtype, f), dim3((unsigned)blocks, (unsigned)(a.side[0].tiles + a.side[1].tiles)), dim3(kW4Threads), 0,
                     static_cast<hipStream_t>(stream), a);
  return launch_ok();
}

int palu_attn_paged_quant_workspace_bytes(const palu_layer_desc* desc, int32_t batch, int32_t max_len, int32_t window, int32_t n_sink,
                                          size_t* out_bytes) {
  PagedQCall c;
  const int st = plan_pagedq(desc, batch, max_len, window, n_sink, &c);
  if (st != PALU_OK) return st;
  if (!out_bytes) return PALU_ERR_INVALID_ARG;
  *out_bytes = c.total;
  return PALU_OK;
}

int palu_attn_paged_quant(const palu_layer_desc* desc, int32_t batch, int32_t max_len, int32_t window, int32_t n_sink,
                          const void* q, const int32_t* q_pos, const uint8_t* hk, const void* hk_scale, const void* hk_zero,
                          const uint8_t* hv, const void* hv_scale, const void* hv_zero, int32_t n_pages, int32_t page_rows,
                          const int32_t* page_table, int32_t table_stride, const int32_t* seq_lens, const void* Bk, const void* Bv,
                          const void* rope_table, int32_t rope_table_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  PagedQCall c;
  int st = plan_pagedq(desc, batch, max_len, window, n_sink, &c);
  if (st != PALU_OK) return st;
  if (!q || !hk || !hk_scale || !hk_zero || !hv || !hv_scale || !hv_zero || !page_table || !Bk || !Bv || !rope_table || !out || !workspace)
    return PALU_ERR_INVALID_ARG;
  if (n_pages <= 0 || page_rows <= 0 || table_stride <= 0) return PALU_ERR_INVALID_ARG;
  if ((long long)table_stride * page_rows < max_len || rope_table_len < max_len) return PALU_ERR_INVALID_ARG;
  for (const void* x : {q, (const void*)hk, (const void*)hv, Bk, Bv, rope_table, (const void*)out, (const void*)workspace})
    if (!aligned(x, 16)) return PALU_ERR_INVALID_ARG;
  for (const void* x : {(const void*)q_pos, (const void*)page_table, (const void*)seq_lens})
    if (!aligned(x, 4)) return PALU_ERR_INVALID_ARG;
  for (const void* x : {hk_scale, hk_zero, hv_scale, hv_zero})
    if (!aligned(x, 2)) return PALU_ERR_INVALID_ARG;
  if ((page_rows & (page_rows - 1)) != 0 || (long long)n_pages * page_rows > 0x7fffffffLL) return PALU_ERR_UNSUPPORTED;
  if (workspace_bytes < c.total) return PALU_ERR_WORKSPACE_TOO_SMALL;

  unsigned char* ws = static_cast<unsigned char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const PagedMeta& m = c.meta;
  PagedQArgs a;
  std::memset(&a, 0, sizeof(a));
  const int Rk = m.k_off[m.n_groups], Rv = m.v_off[m.n_groups];
  a.k = PagedQSide{hk, (const uint16_t*)hk_scale, (const uint16_t*)hk_zero, Rk / 2, Rk / 128};
  a.v = PagedQSide{hv, (const uint16_t*)hv_scale, (const uint16_t*)hv_zero, Rv / 2, Rv / 128};
  a.q = static_cast<const uint16_t*>(q);
  a.Bk = static_cast<const uint16_t*>(Bk);
  a.rope = static_cast<const float*>(rope_table);
  a.q_pos = q_pos;
  a.page_table = page_table;
  a.seq_lens = seq_lens;
  a.o_part = reinterpret_cast<float*>(ws);
  a.ml_part = reinterpret_cast<float*>(ws + c.ml_at);
  a.o_stride = c.o_stride;
  a.n_pages = n_pages;
  a.page_shift = __builtin_ctz((unsigned)page_rows);
  a.table_stride = table_stride;
  a.rope_len = rope_table_len;
  a.max_len = max_len;
  a.window = window;
  a.n_sink = c.n_sink;
  a.chunk_tiles = c.chunk_tiles;
  a.n_slots = c.n_slots;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)PALU_D_HEAD));
  a.meta = m;
  if (c.span_steps == 0) {
    hipLaunchKernelGGL(pagedq_plain_form(desc->act_dtype), dim3((unsigned)(batch * c.n_slots * m.n_heads)), dim3(kPagedQThreads), 0, s, a);
    if ((st = launch_ok()) != PALU_OK) return st;
  }
  a.span_steps = c.span_steps;
  a.n_row_blocks = c.n_row_blocks;
  for (int i = 0; i < kDHead / 2 - kPagedQLow; ++i)
    a.w_low[i] = desc->rope_theta > 0.f ? (float)std::pow((double)desc->rope_theta, -2.0 * (kPagedQLow + i) / kDHead) : 0.f;
  for (int k = 0; k < c.n_cls; ++k) {
    const PagedQClass& cl = c.cls[k];
    const PagedQFn fn = pagedq_form(desc->act_dtype, cl.form);
    if ((st = allow_lds(fn, (size_t)cl.lds_bytes)) != PALU_OK) return st;
    a.n_units = cl.n_units;
    std::memcpy(a.units, cl.units, sizeof(PagedUnit) * cl.n_units);
    hipLaunchKernelGGL(fn, dim3((unsigned)((long long)batch * c.n_slots * c.n_row_blocks * cl.n_units)), dim3(kPagedQFoldThreads), (unsigned)cl.lds_bytes, s, a);
    if ((st = launch_ok()) != PALU_OK) return st;
  }

  PagedMergeArgs e;
  std::memset(&e, 0, sizeof(e));
  e.o_part = a.o_part;
  e.ml_part = a.ml_part;
  e.Bv = static_cast<const uint16_t*>(Bv);
  e.seq_lens = seq_lens;
  e.out = static_cast<uint16_t*>(out);
  e.max_len = max_len;
  e.window = window;
  e.n_sink = c.n_sink;
  e.batch = batch;
  e.chunk_tiles = c.chunk_tiles;
  e.n_slots = c.n_slots;
  e.scaled = 1;
  e.o_stride = c.o_stride;
  e.meta = m;
  return launch_paged_merge(e, desc->act_dtype, s);
}

}  // extern "C"
