// Host side of attention over a paged latent cache (part of the translation unit api.hip).

#include "paged.h"

namespace {

// Units that one launch takes: key/value heads of one rank class.
struct PagedClass {
  PagedForm form;
  int n_stages, lds_bytes, max_packed;
  int n_row_blocks[2], block_rows[2];          // of either part
  int n_units;
  PagedUnit units[PALU_MAX_HEADS];
};
constexpr int kPagedMaxClasses = 12;       // steps of key channels 2, 4, 6, 8, 12, 16, value columns up to 256 or above
struct PagedPlanPart {
  int rows, seqs, max_tiles;               // query rows per key/value head, sequences whose tokens are attended one by one, tiles of the longest
  int chunk_tiles, n_slots;                // 0 slots: nothing to attend
  long long o_stride, ml_stride;           // floats per slot
};
enum { kPagedOwn, kPagedShared };          // a sequence's own tokens, those of the prefix
struct PagedPlan {
  PagedMeta meta;
  PagedPlanPart part[2];
  int n_cls;
  PagedClass cls[kPagedMaxClasses];
};

int check_paged_desc(const palu_layer_desc* desc, PagedMeta* pm) {
  Meta m;
  const int st = check_desc(desc, &m);
  if (st != PALU_OK) return st;
  if (latent_bits(desc->k_latent_dtype) || latent_bits(desc->v_latent_dtype)) return PALU_ERR_UNSUPPORTED;
  std::memset(pm, 0, sizeof(*pm));
  pm->n_heads = desc->n_heads;
  pm->n_groups = desc->n_groups;
  pm->qpk = m.qpk;
  int o = 0;
  for (int j = 0; j <= desc->n_groups; ++j) {
    pm->head_off[j] = desc->group_head_off[j];
    pm->k_off[j] = m.k_off[j];
    pm->v_off[j] = m.v_off[j];
    pm->bk_off[j] = m.bk_off[j] / m.qpk;       // Meta counts query heads
    pm->bv_off[j] = m.bv_off[j] / m.qpk;
    if (j == desc->n_groups) break;
    if (m.k_off[j + 1] - m.k_off[j] > PALU_PAGED_MAX_RANK || m.v_off[j + 1] - m.v_off[j] > PALU_PAGED_MAX_RANK) return PALU_ERR_UNSUPPORTED;
    pm->o_off[j] = o;
    o += (desc->group_head_off[j + 1] - desc->group_head_off[j]) * (m.v_off[j + 1] - m.v_off[j]);
    for (int h = desc->group_head_off[j]; h < desc->group_head_off[j + 1]; ++h) pm->group_of_head[h] = (uint8_t)j;
  }
  return PALU_OK;
}

// Time of n0 workgroups of length a followed by n1 of length b <= a on so many compute units, each of which takes the next when it is free
double paged_makespan(long long n0, double a, long long n1, double b, int cus) {
  const long long full = n0 / cus, rest = n0 - full * cus;
  const double least = ((double)n0 * a + (double)n1 * b) / cus;
  double best = 1e300;
  for (int late = 0; late < 2; ++late) {       // it ends with a workgroup of a unit that has had `full` long ones, or one more
    const double base = (full + late) * a;
    const int from = (int)std::max(0.0, std::floor((least - base) / b));
    for (int k = from; k <= from + 8; ++k) {
      const double t = base + k * b;
      if (t < (full + (rest > 0)) * a) continue;
      if (t >= best) break;
      const double fit = (cus - rest) * std::floor((t - full * a) / b + 1e-9) + (rest ? rest * std::floor((t - (full + 1) * a) / b + 1e-9) : 0.0);
      if (fit < (double)n1) continue;
      best = t;
      break;
    }
  }
  return best < 1e300 ? best : least + a;
}

// p->part: rows, seqs and max_tiles are set
int plan_paged(const PagedMeta& m, PagedPlan* p) {
  p->meta = m;
  p->n_cls = 0;
  long long wgs[2] = {0, 0};                   // workgroups per chunk
  int sum_rv = 0;
  auto rk = [&](int j) { return m.k_off[j + 1] - m.k_off[j]; };
  auto rv = [&](int j) { return m.v_off[j + 1] - m.v_off[j]; };
  auto heads = [&](int j) { return m.head_off[j + 1] - m.head_off[j]; };
  for (int j = 0; j < m.n_groups; ++j) sum_rv += heads(j) * rv(j);
  const int kSteps[6] = {2, 4, 6, 8, 12, 16};
  auto steps = [&](int j) {
    int i = 0;
    while (kSteps[i] * 32 < rk(j)) ++i;
    return kSteps[i];
  };
  for (int cls = 0; cls < kPagedMaxClasses; ++cls) {
    const int ks = kSteps[cls % 6], vb = cls / 6 + 1;
    auto in_class = [&](int j) { return steps(j) == ks && (rv(j) > 256) == (vb == 2); };
    int any = 0;
    for (int j = 0; j < m.n_groups; ++j) any += in_class(j);
    if (!any) continue;
    PagedClass& c = p->cls[p->n_cls++];
    c.form = PagedForm{ks, vb, false};
    // Units: whole adjacent groups of equal ranks and size side by side, as far as 256 columns and the heads go (ranks in whole 64s:
    // the staged rows' layout), else parts of one group.  A unit of more heads reads its latents once for all of them.
    const int unit_heads = c.form.unit_heads();
    c.n_units = 0;
    int k_groups = 1, v_cols = 0, most = 1;                  // of a unit: groups, value columns, heads
    for (int first = 0;; first += unit_heads) {              // round robin over the groups: neighbouring workgroups, which go to different
      bool more = false;                                     // L2 caches, take different groups, and the units of one group meet in one
      for (int j = 0; j < m.n_groups; ++j) {
        if (!in_class(j) || first >= heads(j)) continue;
        int n = 1;
        if (rk(j) % 64 == 0)
          while (j + n < m.n_groups && rk(j + n) == rk(j) && rv(j + n) == rv(j) && heads(j + n) == heads(j) && (n + 1) * heads(j) <= unit_heads &&
                 (n + 1) * rk(j) <= 256 && (n + 1) * rv(j) <= 256)
            ++n;
        more = true;
        const int nh = std::min(unit_heads, n * heads(j) - first);
        c.units[c.n_units++].bits = (uint32_t)(m.head_off[j] + first) | (uint32_t)nh << 8 | (uint32_t)j << 16 | (uint32_t)n << 24;
        k_groups = std::max(k_groups, n);
        v_cols = std::max(v_cols, n * rv(j));
        most = std::max(most, nh);
        j += n - 1;
      }
      if (!more) break;
    }
    // Query rows: 16 in all, or 16 per head and as many as accumulators go where there are more; as many blocks of them as it takes.
    // (32 sequences behind 8192 rows, ranks 128 / 384: blocks of 32 packed rows 129 us, of 16 176; 8 sequences: one block 57, two 63.)
    for (const PagedPlanPart& t : p->part) c.form.many = c.form.many || (t.max_tiles > 0 && ks <= 8 && most * t.rows > 16);
    auto lds_bytes = [&](int stages) {
      return paged_lds(k_groups, ks, v_cols, c.max_packed, c.form.row_tiles(), c.form.parts(), stages).total;
    };
    for (int limit = std::min(16, c.form.max_rows() / most); limit > 0; --limit) {   // (fewer where two stages leave no more LDS)
      c.max_packed = 0;
      for (int i = 0; i < 2; ++i) {
        c.n_row_blocks[i] = ceil_div(p->part[i].rows, limit);
        c.block_rows[i] = ceil_div(p->part[i].rows, c.n_row_blocks[i]);
        if (p->part[i].max_tiles > 0) c.max_packed = std::max(c.max_packed, most * c.block_rows[i]);
      }
      if (c.form.many) c.max_packed = c.form.max_rows();
      if (lds_bytes(2) <= kPagedLdsBytes) break;
    }
    if (lds_bytes(2) > kPagedLdsBytes) return PALU_ERR_UNSUPPORTED;
    c.n_stages = 2;
    while (c.n_stages < kPagedMaxStages && lds_bytes(c.n_stages + 1) <= kPagedLdsBytes) ++c.n_stages;
    c.lds_bytes = lds_bytes(c.n_stages);
    for (int i = 0; i < 2; ++i) wgs[i] += (long long)c.n_units * c.n_row_blocks[i] * p->part[i].seqs;
  }
  for (PagedPlanPart& t : p->part) {
    t.o_stride = (long long)t.rows * sum_rv;
    t.ml_stride = (long long)t.rows * m.n_heads * 2;
    t.chunk_tiles = 1;
    t.n_slots = 0;
  }
  // Tiles per workgroup: one workgroup is resident per compute unit, and its start and end cost about as much as four tiles (11 us; 24 sequences
  // with a window of 1024: 100 us, priced at 2.5 tiles 114); a slot more is merged in a twentieth.  The two parts' workgroups run together: of equal
  // length, or one part's halves or quarters of the other's.
  const int cus = device_cu_count();
  double best = 1e300;
  PagedPlanPart& own = p->part[kPagedOwn];
  PagedPlanPart& shared = p->part[kPagedShared];
  auto consider = [&](int tiles_own, int tiles_shared) {
    const int n_own = own.max_tiles > 0 ? ceil_div(own.max_tiles, tiles_own) : 0, n_shared = shared.max_tiles > 0 ? ceil_div(shared.max_tiles, tiles_shared) : 0;
    double a = 4.0 + (n_own ? ceil_div(own.max_tiles, n_own) : 0), b = 4.0 + (n_shared ? ceil_div(shared.max_tiles, n_shared) : 0);
    long long na = wgs[kPagedOwn] * n_own, nb = wgs[kPagedShared] * n_shared;
    if (a < b) {
      std::swap(a, b);
      std::swap(na, nb);
    }
    const double cost = paged_makespan(na, a, nb, b, cus) + 0.05 * (n_own + n_shared);
    if (cost >= best) return;
    best = cost;
    own.n_slots = n_own;
    own.chunk_tiles = std::max(1, n_own ? ceil_div(own.max_tiles, n_own) : 0);
    shared.n_slots = n_shared;
    shared.chunk_tiles = std::max(1, n_shared ? ceil_div(shared.max_tiles, n_shared) : 0);
  };
  const bool both = own.max_tiles > 0 && shared.max_tiles > 0;
  for (const PagedPlanPart* t : {&own, &shared}) {
    // (more than a few workgroups per compute unit would be starts and little else)
    const long long most = std::min<long long>(both ? 64 : 1024, std::max<long long>(16, 4LL * cus / std::max<long long>(1, wgs[t == &own ? kPagedOwn : kPagedShared])));
    for (int n = 1; n <= std::min<long long>(t->max_tiles, most); ++n) {
      const int tiles = ceil_div(t->max_tiles, n);
      consider(tiles, tiles);
      if (!both) continue;
      for (int f = 2; f <= 4; f *= 2) {
        consider(ceil_div(tiles, f), tiles);
        consider(tiles, ceil_div(tiles, f));
      }
    }
  }
  return PALU_OK;
}

// the largest number of tiles that a sequence of up to max_len rows has
int paged_max_tiles(int max_len, int first, int window, int n_sink) {
  const long long all = ceil_div(max_len, kPagedTile) - first / kPagedTile;
  if (window <= 0) return max_len > first ? (int)all : 0;
  return (int)std::min<long long>(all, ((long long)n_sink + kPagedTile - 1) / kPagedTile + ((long long)window + kPagedTile - 2) / kPagedTile + 1);
}

struct PagedCall {
  PagedPlan plan;
  int prefix, max_len, window, n_sink;
  size_t o_at[2], ml_at[2], total;             // partial results in the workspace
};

int plan_paged_call(const palu_layer_desc* desc, int batch, int prefix, int max_len, int window, int n_sink, PagedCall* c) {
  PagedMeta m;
  int st = check_paged_desc(desc, &m);
  if (st != PALU_OK) return st;
  if (batch <= 0 || max_len <= 0 || prefix < 0 || prefix > max_len || window < 0 || n_sink < 0) return PALU_ERR_INVALID_ARG;
  if (batch > 65535) return PALU_ERR_UNSUPPORTED;
  if (max_len > (1 << 30)) return PALU_ERR_UNSUPPORTED;      // positions of the angle table
  c->prefix = prefix;
  c->max_len = max_len;
  c->window = window;
  c->n_sink = window > 0 ? n_sink : 0;
  PagedPlan& p = c->plan;
  p.part[kPagedOwn] = PagedPlanPart{m.qpk, batch, paged_max_tiles(max_len, prefix, window, c->n_sink)};
  p.part[kPagedShared] = PagedPlanPart{batch * m.qpk, 1, ceil_div(prefix, kPagedTile)};
  st = plan_paged(m, &p);
  if (st != PALU_OK) return st;
  c->total = 0;
  for (int i = 0; i < 2; ++i) {
    const PagedPlanPart& t = p.part[i];
    c->o_at[i] = c->total;
    c->ml_at[i] = c->o_at[i] + align_up((size_t)t.seqs * t.n_slots * t.o_stride * sizeof(float));
    c->total = c->ml_at[i] + align_up((size_t)t.seqs * t.n_slots * t.ml_stride * sizeof(float));
  }
  if (c->total < kAlign) c->total = kAlign;
  for (int i = 0; i < p.n_cls; ++i) {
    long long wgs = 0;
    for (int k = 0; k < 2; ++k) wgs += (long long)p.cls[i].n_units * p.cls[i].n_row_blocks[k] * p.part[k].n_slots * p.part[k].seqs;
    if (wgs * kPagedThreads > 0xffffffffLL) return PALU_ERR_UNSUPPORTED;     // (what a launch takes)
  }
  return PALU_OK;
}

// a.part is that of kPagedOwn, kPagedShared, but for what the classes say
int launch_paged(const PagedPlan& p, const PagedArgs& args, int act, hipStream_t s) {
  const int first = p.part[kPagedShared].chunk_tiles > p.part[kPagedOwn].chunk_tiles ? kPagedShared : kPagedOwn;   // (the longer ones)
  for (int i = 0; i < p.n_cls; ++i) {
    const PagedClass& c = p.cls[i];
    PagedArgs a = args;
    a.n_units = c.n_units;
    std::memcpy(a.units, c.units, sizeof(PagedUnit) * c.n_units);
    a.n_stages = c.n_stages;
    a.max_packed = c.max_packed;
    unsigned wgs[2];
    for (int k = 0; k < 2; ++k) {
      const int from = k == 0 ? first : 1 - first;
      a.part[k] = args.part[from];
      a.part[k].n_row_blocks = c.n_row_blocks[from];
      a.part[k].block_rows = c.block_rows[from];
      wgs[k] = (unsigned)(c.n_units * c.n_row_blocks[from] * p.part[from].n_slots * p.part[from].seqs);
    }
    if (wgs[0] + wgs[1] == 0) continue;
    a.n_first = (int)wgs[0];
    const PagedFn fn = act == PALU_F16 ? paged_form<F16>(c.form) : paged_form<BF16>(c.form);
    int st = allow_lds(fn, (size_t)c.lds_bytes);
    if (st != PALU_OK) return st;
    hipLaunchKernelGGL(fn, dim3(wgs[0] + wgs[1]), dim3(kPagedThreads), (unsigned)c.lds_bytes, s, a);
    if ((st = launch_ok()) != PALU_OK) return st;
  }
  return PALU_OK;
}

int paged_impl(const palu_layer_desc* desc, int32_t batch, int32_t prefix, int32_t max_len, int32_t window, int32_t n_sink,
               const void* q, const int32_t* q_pos, const void* hk, const void* hv, int32_t n_pages, int32_t page_rows,
               const int32_t* page_table, int32_t table_stride, const int32_t* seq_lens, const void* Bk, const void* Bv,
               const void* rope_table, int32_t rope_table_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  PagedCall c;
  int st = plan_paged_call(desc, batch, prefix, max_len, window, n_sink, &c);
  if (st != PALU_OK) return st;
  if (!q || !hk || !hv || !page_table || !Bk || !Bv || !rope_table || !out || !workspace) return PALU_ERR_INVALID_ARG;
  if (n_pages <= 0 || page_rows <= 0 || table_stride <= 0) return PALU_ERR_INVALID_ARG;
  if ((long long)table_stride * page_rows < max_len || rope_table_len < max_len) return PALU_ERR_INVALID_ARG;
  for (const void* x : {q, hk, hv, Bk, Bv, rope_table, (const void*)out, (const void*)workspace})
    if (reinterpret_cast<uintptr_t>(x) & 15) return PALU_ERR_INVALID_ARG;
  for (const void* x : {(const void*)q_pos, (const void*)page_table, (const void*)seq_lens})
    if (reinterpret_cast<uintptr_t>(x) & 3) return PALU_ERR_INVALID_ARG;
  if ((page_rows & (page_rows - 1)) != 0 || (long long)n_pages * page_rows > 0x7fffffffLL) return PALU_ERR_UNSUPPORTED;
  if (workspace_bytes < c.total) return PALU_ERR_WORKSPACE_TOO_SMALL;

  unsigned char* ws = static_cast<unsigned char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const PagedPlan& p = c.plan;
  const PagedMeta& m = p.meta;
  PagedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.hk = static_cast<const uint16_t*>(hk);
  a.hv = static_cast<const uint16_t*>(hv);
  a.q = static_cast<const uint16_t*>(q);
  a.Bk = static_cast<const uint16_t*>(Bk);
  a.rope = static_cast<const float*>(rope_table);
  a.q_pos = q_pos;
  a.page_table = page_table;
  a.seq_lens = seq_lens;
  a.R_k = m.k_off[m.n_groups];
  a.R_v = m.v_off[m.n_groups];
  a.n_pages = n_pages;
  a.page_shift = __builtin_ctz((unsigned)page_rows);
  a.table_stride = table_stride;
  a.rope_len = rope_table_len;
  a.pos_len = max_len;
  a.meta = m;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)PALU_D_HEAD));

  for (int i = 0; i < 2; ++i) {
    PagedPart& t = a.part[i];
    t.o_part = reinterpret_cast<float*>(ws + c.o_at[i]);
    t.ml_part = reinterpret_cast<float*>(ws + c.ml_at[i]);
    t.o_stride = p.part[i].o_stride;
    t.rows = p.part[i].rows;
    t.chunk_tiles = p.part[i].chunk_tiles;
    t.n_slots = p.part[i].n_slots;
  }
  a.part[kPagedOwn].max_len = max_len;
  a.part[kPagedOwn].first = prefix;
  a.part[kPagedOwn].window = c.window;
  a.part[kPagedOwn].n_sink = c.n_sink;
  a.part[kPagedShared].max_len = prefix;       // nothing of the shared tokens is before, and no window
  a.part[kPagedShared].shared = 1;
  if ((st = launch_paged(p, a, desc->act_dtype, s)) != PALU_OK) return st;

  PagedMergeArgs e;
  std::memset(&e, 0, sizeof(e));
  e.o_part = a.part[kPagedOwn].o_part;
  e.ml_part = a.part[kPagedOwn].ml_part;
  e.o_shared = a.part[kPagedShared].o_part;
  e.ml_shared = a.part[kPagedShared].ml_part;
  e.Bv = static_cast<const uint16_t*>(Bv);
  e.seq_lens = seq_lens;
  e.out = static_cast<uint16_t*>(out);
  e.max_len = max_len;
  e.first = prefix;
  e.window = c.window;
  e.n_sink = c.n_sink;
  e.batch = batch;
  e.chunk_tiles = p.part[kPagedOwn].chunk_tiles;
  e.n_slots = p.part[kPagedOwn].n_slots;
  e.o_stride = p.part[kPagedOwn].o_stride;
  e.n_shared = p.part[kPagedShared].n_slots;
  e.o_shared_stride = p.part[kPagedShared].o_stride;
  e.meta = m;
  // rows of a head per workgroup: fewer until there are two workgroups per compute unit (48 grouped-query sequences: 118 us a call; until
  // one 126, until four 132)
  int per_wg = 8;
  while (per_wg > 1 && (long long)ceil_div(batch * m.qpk, per_wg) * m.n_heads < 2 * device_cu_count()) per_wg /= 2;
  hipLaunchKernelGGL(desc->act_dtype == PALU_F16 ? paged_merge_form<F16>(per_wg) : paged_merge_form<BF16>(per_wg),
                     dim3((unsigned)ceil_div(batch * m.qpk, per_wg), (unsigned)m.n_heads), dim3(256), 0, s, e);
  return launch_ok();
}

}  // namespace

extern "C" {

int palu_attn_paged_workspace_bytes(const palu_layer_desc* desc, int32_t batch, int32_t max_len, int32_t window, int32_t n_sink,
                                    size_t* out_bytes) {
  PagedCall c;
  const int st = plan_paged_call(desc, batch, 0, max_len, window, n_sink, &c);
  if (st != PALU_OK) return st;
  if (!out_bytes) return PALU_ERR_INVALID_ARG;
  *out_bytes = c.total;
  return PALU_OK;
}

int palu_attn_paged(const palu_layer_desc* desc, int32_t batch, int32_t max_len, int32_t window, int32_t n_sink,
                    const void* q, const int32_t* q_pos, const void* hk, const void* hv, int32_t n_pages, int32_t page_rows,
                    const int32_t* page_table, int32_t table_stride, const int32_t* seq_lens, const void* Bk, const void* Bv,
                    const void* rope_table, int32_t rope_table_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_impl(desc, batch, 0, max_len, window, n_sink, q, q_pos, hk, hv, n_pages, page_rows, page_table, table_stride, seq_lens,
                    Bk, Bv, rope_table, rope_table_len, out, workspace, workspace_bytes, stream);
}

int palu_attn_prefix_workspace_bytes(const palu_layer_desc* desc, int32_t batch, int32_t prefix_len, int32_t max_len, size_t* out_bytes) {
  PagedCall c;
  const int st = plan_paged_call(desc, batch, prefix_len, max_len, 0, 0, &c);
  if (st != PALU_OK) return st;
  if (!out_bytes) return PALU_ERR_INVALID_ARG;
  *out_bytes = c.total;
  return PALU_OK;
}

int palu_attn_prefix(const palu_layer_desc* desc, int32_t batch, int32_t prefix_len, int32_t max_len,
                     const void* q, const int32_t* q_pos, const void* hk, const void* hv, int32_t n_pages, int32_t page_rows,
                     const int32_t* page_table, int32_t table_stride, const int32_t* seq_lens, const void* Bk, const void* Bv,
                     const void* rope_table, int32_t rope_table_len, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_impl(desc, batch, prefix_len, max_len, 0, 0, q, q_pos, hk, hv, n_pages, page_rows, page_table, table_stride, seq_lens,
                    Bk, Bv, rope_table, rope_table_len, out, workspace, workspace_bytes, stream);
}

}  // extern "C"
