// api_kv4.hip -- the extern "C" boundary of the 4-bit cache (append, read, attention) and of eviction: argument
// validation, workspace layout, launch configuration.  Validation happens before any HIP call.
#include <math.h>

#include "kv4.hpp"
#include "validate.hpp"

using namespace dustin;

namespace {

bool pages_ok(const int32_t* table, int page_size, int max_pages, int num_pages, int64_t stride_page, int* shift) {
  if (page_size <= 0 || (page_size & (page_size - 1)) || max_pages <= 0 || num_pages <= 0 || stride_page <= 0 ||
      !aligned(table, 4))
    return false;
  *shift = 0;
  while ((1 << *shift) < page_size) ++*shift;
  return true;
}

// Validates a 4-bit cache view for `need` addressable positions per sequence.
dustin_status kv4_of(const dustin_kv4* kv, int64_t need, Kv4View* out) {
  if (!kv || !kv->data || !kv->scales || kv->num_kv_heads <= 0) return DUSTIN_ERR_INVALID_ARG;
  if (kv->head_dim != 64 && kv->head_dim != 128) return DUSTIN_ERR_UNSUPPORTED;
  const int sb = kv->head_dim / kKv4Block;
  if (!aligned(kv->data, 16) || kv->stride_b % 16 || kv->stride_n % 16 || kv->stride_h % 16 || kv->stride_page % 16 ||
      !aligned(kv->scales, sb) || kv->scale_stride_b % sb || kv->scale_stride_n % sb || kv->scale_stride_h % sb ||
      kv->scale_stride_page % sb)
    return DUSTIN_ERR_INVALID_ARG;
  if (kv->stride_n <= 0 || kv->stride_h < 0 || kv->stride_b < 0 || kv->scale_stride_n <= 0 || kv->scale_stride_h < 0 ||
      kv->scale_stride_b < 0)
    return DUSTIN_ERR_INVALID_ARG;
  memset(out, 0, sizeof *out);
  out->data = static_cast<const uint8_t*>(kv->data);
  out->scales = static_cast<const uint8_t*>(kv->scales);
  out->stride_b = kv->stride_b;
  out->stride_n = kv->stride_n;
  out->stride_h = kv->stride_h;
  out->sstride_b = kv->scale_stride_b;
  out->sstride_n = kv->scale_stride_n;
  out->sstride_h = kv->scale_stride_h;
  if (kv->page_table) {
    if (!pages_ok(kv->page_table, kv->page_size, kv->max_pages, kv->num_pages, kv->stride_page, &out->page_shift) ||
        kv->scale_stride_page <= 0)
      return DUSTIN_ERR_INVALID_ARG;
    out->page_table = kv->page_table;
    out->max_pages = kv->max_pages;
    out->num_pages = kv->num_pages;
    out->stride_page = kv->stride_page;
    out->sstride_page = kv->scale_stride_page;
    out->capacity = (int64_t)kv->max_pages * kv->page_size;
  } else {
    out->capacity = kv->capacity;
  }
  if (out->capacity < need || out->capacity <= 0) return DUSTIN_ERR_INVALID_ARG;
  if (out->capacity > INT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  return DUSTIN_OK;
}

// Positions that the caches of a batch must address.  Where every sequence has nq_max tokens: the longest one's and
// theirs.  Where each has a count of its own, the longest may have the shortest window, which only the device knows:
// max_len (an append writes nothing past a cache, and the attention's positions are clamped into it).
int64_t positions_of(const dustin_batch* bt) { return (int64_t)bt->max_len + (bt->n_query ? 0 : bt->nq_max); }

// K and V of one call: the same heads, channels and pages.
template <class Kv>
bool same_layout(const Kv* k, const Kv* v) {
  return k->num_kv_heads == v->num_kv_heads && k->head_dim == v->head_dim && k->page_table == v->page_table &&
         (!k->page_table ||
          (k->page_size == v->page_size && k->max_pages == v->max_pages && k->num_pages == v->num_pages));
}

// Rows written for several sequences, or heads, have places of their own (with pages, the table says so).
template <class Kv>
bool apart(const Kv* c, int batch) {
  return (c->num_kv_heads <= 1 || c->stride_h > 0) && (batch <= 1 || c->page_table || c->stride_b > 0);
}
bool apart(const dustin_kv4* c, int batch) {
  return apart<dustin_kv4>(c, batch) && (c->num_kv_heads <= 1 || c->scale_stride_h > 0) &&
         (batch <= 1 || c->page_table || c->scale_stride_b > 0);
}

dustin_status kv4_rows(bool append, const void* k_rows, int64_t k_sb, int64_t k_st, int64_t k_sh, const void* v_rows,
                       int64_t v_sb, int64_t v_st, int64_t v_sh, const dustin_kv4* k, const dustin_kv4* v,
                       const dustin_batch* bt, void* stream) {
  if (!batch_ok(bt) || !k || !v) return DUSTIN_ERR_INVALID_ARG;
  const bool none = bt->batch == 0 || bt->nq_max == 0;  // no rows: they may lie nowhere
  if (!none && (!k_rows || !v_rows)) return DUSTIN_ERR_INVALID_ARG;
  if (!rows_aligned(k_rows, k_sb, k_st, k_sh) || !rows_aligned(v_rows, v_sb, v_st, v_sh)) return DUSTIN_ERR_INVALID_ARG;
  if (!same_layout(k, v) || (append && (!apart(k, bt->batch) || !apart(v, bt->batch)))) return DUSTIN_ERR_INVALID_ARG;
  Kv4RowsArgs a;
  memset(&a, 0, sizeof a);
  const int64_t need = positions_of(bt);
  dustin_status st = kv4_of(k, need, &a.k);
  if (st == DUSTIN_OK) st = kv4_of(v, need, &a.v);
  if (st != DUSTIN_OK) return st;
  if ((int64_t)bt->nq_max * k->num_kv_heads * (k->head_dim / 8) > INT32_MAX / 4) return DUSTIN_ERR_UNSUPPORTED;
  if (none) return DUSTIN_OK;
  a.k_in = static_cast<const uint16_t*>(k_rows);
  a.v_in = static_cast<const uint16_t*>(v_rows);
  a.k_out = const_cast<uint16_t*>(a.k_in);
  a.v_out = const_cast<uint16_t*>(a.v_in);
  a.k_sb = k_sb;
  a.k_st = k_st;
  a.k_sh = k_sh;
  a.v_sb = v_sb;
  a.v_st = v_st;
  a.v_sh = v_sh;
  a.dims = dims_of(bt);
  a.batch = bt->batch;
  a.num_kv_heads = k->num_kv_heads;
  a.head_dim = k->head_dim;
  const hipError_t e = append ? launch_kv4_append(a, static_cast<hipStream_t>(stream))
                              : launch_kv4_read(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DUSTIN_OK : DUSTIN_ERR_LAUNCH;
}

// ---- attention

constexpr int64_t kAttn4MaxPairs = 65536;

// Workgroups of a call whose pairs hold up to `tokens` tokens, window included, and `rows` query rows: as many as run
// at once.
int attn4_units(int64_t pairs, int64_t tokens, int64_t rows) {
  const int64_t most = pairs * ((tokens + kAttn4Granule - 1) / kAttn4Granule);
  const int64_t cap = rows <= 16 * kAttn4Two ? 2 * kAttn4Cus : kAttn4Cus;
  const int64_t u = most < cap ? most : cap;
  return (int)((u + 7) / 8 * 8);
}

// Workspace: the plan, then the parts of every run.
struct Attn4Ws {
  size_t ml, acc, total;
};
Attn4Ws attn4_ws(int64_t pairs, int units, int64_t rows_max) {
  Attn4Ws w;
  w.ml = round_up((size_t)(pairs + 1) * sizeof(int32_t), kAlign);
  w.acc = w.ml + round_up((size_t)units * 2 * rows_max * sizeof(float2), kAlign);
  w.total = w.acc + round_up((size_t)units * 2 * rows_max * 128 * sizeof(float), kAlign);
  return w;
}
// What a call asks for: enough for any with fewer rows, too, which may have more runs.
size_t attn4_ws_bytes(int64_t pairs, int64_t tokens, int64_t rows) {
  const size_t own = attn4_ws(pairs, attn4_units(pairs, tokens, rows), rows).total;
  const int64_t two = rows < 16 * kAttn4Two ? rows : 16 * kAttn4Two;
  const size_t fewer = attn4_ws(pairs, attn4_units(pairs, tokens, two), two).total;
  return own > fewer ? own : fewer;
}

dustin_status attn4(bool sparse, const void* q, int64_t q_sb, int64_t q_st, int64_t q_sh, int32_t num_q_heads,
                    const dustin_kv4* k, const dustin_kv4* v, const dustin_batch* bt, const int32_t* idx,
                    int64_t idx_sb, int64_t idx_sg, const int32_t* count, int32_t groups, float scale, void* out,
                    int64_t o_sb, int64_t o_st, int64_t o_sh, void* ws, size_t ws_bytes, void* stream) {
  if (!batch_ok(bt) || !k || !v) return DUSTIN_ERR_INVALID_ARG;
  const bool none = bt->batch == 0 || bt->nq_max == 0;
  if (!none && (!q || !out)) return DUSTIN_ERR_INVALID_ARG;
  if (!isfinite(scale) || !(scale > 0.f)) return DUSTIN_ERR_INVALID_ARG;
  const int H = k->num_kv_heads;
  if (num_q_heads <= 0 || H <= 0 || num_q_heads % H || !same_layout(k, v)) return DUSTIN_ERR_INVALID_ARG;
  if (k->head_dim != 128) return DUSTIN_ERR_UNSUPPORTED;
  if (bt->max_len > INT32_MAX - 4096) return DUSTIN_ERR_UNSUPPORTED;  // int32, with the rounds that are loaded ahead
  if (!rows_aligned(q, q_sb, q_st, q_sh) || !rows_aligned(out, o_sb, o_st, o_sh)) return DUSTIN_ERR_INVALID_ARG;
  const int gs = num_q_heads / H;
  if ((int64_t)bt->nq_max * gs > 128) return DUSTIN_ERR_UNSUPPORTED;
  const int64_t pairs = (int64_t)bt->batch * H;
  if (pairs > kAttn4MaxPairs) return DUSTIN_ERR_UNSUPPORTED;
  if (sparse) {
    if (!none && ((!idx && bt->k_max > 0) || !count)) return DUSTIN_ERR_INVALID_ARG;
    if (groups != 1 && groups != H) return DUSTIN_ERR_INVALID_ARG;
    if (!aligned(idx, 4) || !aligned(count, 4) || idx_sb < 0 || idx_sg < 0) return DUSTIN_ERR_INVALID_ARG;
    if (bt->k_max > INT32_MAX - 4096) return DUSTIN_ERR_UNSUPPORTED;
  }
  Attn4Args a;
  memset(&a, 0, sizeof a);
  const int64_t need = positions_of(bt);
  dustin_status st = kv4_of(k, need, &a.k);
  if (st == DUSTIN_OK) st = kv4_of(v, need, &a.v);
  if (st != DUSTIN_OK) return st;
  a.k.capacity = a.v.capacity = a.k.capacity < a.v.capacity ? a.k.capacity : a.v.capacity;  // a token is a row of both
  // the kernels multiply positions and pages by 32-bit strides, and count granules in 32 bits
  for (const Kv4View* c : {&a.k, &a.v})
    for (const int64_t x : {c->stride_n, c->sstride_n, c->stride_page, c->sstride_page})
      if (x > (int64_t)UINT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  const int64_t tokens = (int64_t)(sparse ? bt->k_max : bt->max_len) + bt->nq_max;
  if (pairs * ((tokens + kAttn4Granule - 1) / kAttn4Granule) > INT32_MAX / 2) return DUSTIN_ERR_UNSUPPORTED;
  if (none) return DUSTIN_OK;
  a.q = static_cast<const uint16_t*>(q);
  a.q_sb = q_sb;
  a.q_st = q_st;
  a.q_sh = q_sh;
  a.out = static_cast<uint16_t*>(out);
  a.o_sb = o_sb;
  a.o_st = o_st;
  a.o_sh = o_sh;
  a.dims = dims_of(bt);
  a.idx = idx;
  a.idx_sb = idx_sb;
  a.idx_sg = idx_sg;
  a.count = count;
  a.groups = sparse ? groups : 1;
  a.num_kv_heads = H;
  a.group_size = gs;
  a.pairs = (int32_t)pairs;
  a.scale_log2 = scale * kLog2e;
  a.rows_max = bt->nq_max * gs;
  a.units = attn4_units(pairs, tokens, a.rows_max);
  const Attn4Ws w = attn4_ws(pairs, a.units, a.rows_max);
  if (!ws || ws_bytes < attn4_ws_bytes(pairs, tokens, a.rows_max) || !aligned(ws, kAlign)) return DUSTIN_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  a.plan = reinterpret_cast<int32_t*>(base);
  a.part_ml = reinterpret_cast<float2*>(base + w.ml);
  a.part = reinterpret_cast<float*>(base + w.acc);
  if (sparse && bt->k_max == 0) a.idx = bt->seq_lens, a.idx_sb = a.idx_sg = 0;  // no entries: read, and not used
  a.idx_last = sparse && bt->k_max > 0 ? bt->k_max - 1 : 0;
  const hipError_t e = launch_attn_kv4(a, (a.rows_max + 15) / 16, sparse, a.k.page_table != nullptr,
                                       static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DUSTIN_OK : DUSTIN_ERR_LAUNCH;
}

// ---- eviction

dustin_status evict_cache(const dustin_kv* kv, int64_t need, EvictCache* out) {
  if (!kv) return DUSTIN_ERR_INVALID_ARG;
  if (kv->head_dim != 64 && kv->head_dim != 128) return DUSTIN_ERR_UNSUPPORTED;
  KvView v;
  const dustin_status st = kv_of(kv, kv->head_dim, need, &v);
  if (st != DUSTIN_OK) return st;
  if (v.capacity > INT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  *out = EvictCache{reinterpret_cast<const uint8_t*>(v.data), nullptr, 2 * v.stride_b, 2 * v.stride_n, 2 * v.stride_h,
                    2 * v.stride_page, 0, 0, 0, 0, v.page_table, v.page_shift, v.max_pages, v.num_pages,
                    (int32_t)(v.capacity - 1)};
  return DUSTIN_OK;
}

dustin_status evict_cache(const dustin_kv4* kv, int64_t need, EvictCache* out) {
  Kv4View v;
  const dustin_status st = kv4_of(kv, need, &v);
  if (st != DUSTIN_OK) return st;
  *out = EvictCache{v.data, v.scales, v.stride_b, v.stride_n, v.stride_h, v.stride_page, v.sstride_b, v.sstride_n,
                    v.sstride_h, v.sstride_page, v.page_table, v.page_shift, v.max_pages, v.num_pages,
                    (int32_t)(v.capacity - 1)};
  return DUSTIN_OK;
}

// Equal caches of a call with `heads` KV heads and `batch` sequences (strides that no row uses aside).
bool same_cache(const EvictCache& x, const EvictCache& y, int heads, int batch) {
  if (x.data != y.data || x.scales != y.scales || x.page_table != y.page_table) return false;
  if (x.stride_n != y.stride_n || x.sstride_n != y.sstride_n) return false;
  if (heads > 1 && (x.stride_h != y.stride_h || x.sstride_h != y.sstride_h)) return false;
  if (x.page_table)
    return x.page_shift == y.page_shift && x.max_pages == y.max_pages && x.num_pages == y.num_pages &&
           x.stride_page == y.stride_page && x.sstride_page == y.sstride_page;
  return batch <= 1 || (x.stride_b == y.stride_b && x.sstride_b == y.sstride_b);
}

template <class Kv>
dustin_status evict(const Kv* k, const Kv* v, const Kv* k_out, const Kv* v_out, int32_t batch, const int32_t* idx,
                    int64_t idx_sb, int64_t idx_sg, const int32_t* count, int32_t groups, int32_t k_max, const float* w,
                    int64_t w_sb, int64_t w_sg, int32_t w_len, float* w_out, int64_t wo_sb, int64_t wo_sg,
                    int32_t* new_lens, int row_bytes_per_dim2, bool four, void* stream) {
  const bool rows = k || v || k_out || v_out;  // else the weights alone
  if ((rows ? !k || !k_out || !v != !v_out : !w) || batch < 0 || k_max < 0) return DUSTIN_ERR_INVALID_ARG;
  if (batch > 0 && ((!idx && k_max > 0) || !count)) return DUSTIN_ERR_INVALID_ARG;
  if (rows && ((v && (!same_layout(k, v) || !same_layout(k_out, v_out))) || k->num_kv_heads != k_out->num_kv_heads ||
               k->head_dim != k_out->head_dim))
    return DUSTIN_ERR_INVALID_ARG;
  if (v && (k->data == v->data || k_out->data == v_out->data)) return DUSTIN_ERR_INVALID_ARG;
  if (rows && (!apart(k_out, batch) || (v_out && !apart(v_out, batch)))) return DUSTIN_ERR_INVALID_ARG;
  if (rows ? groups != 1 && groups != k->num_kv_heads : groups < 1) return DUSTIN_ERR_INVALID_ARG;
  if (!aligned(idx, 4) || !aligned(count, 4) || !aligned(new_lens, 4) || idx_sb < 0 || idx_sg < 0)
    return DUSTIN_ERR_INVALID_ARG;
  if (!w != !w_out || !aligned(w, 4) || !aligned(w_out, 4)) return DUSTIN_ERR_INVALID_ARG;
  if (w && (w_len <= 0 || w_sb < 0 || w_sg < 0 || wo_sb < 0 || wo_sg < 0)) return DUSTIN_ERR_INVALID_ARG;
  if (w && ((groups > 1 && wo_sg == 0) || (batch > 1 && wo_sb == 0))) return DUSTIN_ERR_INVALID_ARG;  // one row for several
  EvictArgs a;
  memset(&a, 0, sizeof a);
  if (rows) {
    dustin_status st = evict_cache(k, 1, &a.src[0]);
    if (st == DUSTIN_OK && v) st = evict_cache(v, 1, &a.src[1]);
    if (st == DUSTIN_OK) st = evict_cache(k_out, k_max, &a.dst[0]);
    if (st == DUSTIN_OK && v) st = evict_cache(v_out, k_max, &a.dst[1]);
    if (st != DUSTIN_OK) return st;
    const bool same_k = same_cache(a.src[0], a.dst[0], k->num_kv_heads, batch);
    const bool same_v = v ? same_cache(a.src[1], a.dst[1], k->num_kv_heads, batch) : same_k;
    if (same_k != same_v || (!same_k && (k->data == k_out->data || (v && v->data == v_out->data))))
      return DUSTIN_ERR_INVALID_ARG;
    a.caches = v ? 2 : 1;
    a.num_kv_heads = k->num_kv_heads;
    a.row_bytes = k->head_dim * row_bytes_per_dim2 / 2;
    a.scale_bytes = four ? k->head_dim / kKv4Block : 0;
    a.in_place = same_k;
    // (32-bit counts of a sequence's pieces)
    if (!same_k && (int64_t)k_max * a.num_kv_heads * a.caches * (a.row_bytes / 16) > INT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  }
  if (batch == 0) return DUSTIN_OK;
  a.idx = idx;
  a.idx_sb = idx_sb;
  a.idx_sg = idx_sg;
  a.count = count;
  a.w = w;
  a.w_out = w_out;
  a.w_sb = w_sb;
  a.w_sg = w_sg;
  a.wo_sb = wo_sb;
  a.wo_sg = wo_sg;
  a.new_lens = new_lens;
  a.batch = batch;
  a.groups = groups;
  a.k_max = k_max;
  a.w_len = w_len;
  return launch_evict(a, static_cast<hipStream_t>(stream)) == hipSuccess ? DUSTIN_OK : DUSTIN_ERR_LAUNCH;
}

}  // namespace

extern "C" {

dustin_status dustin_kv4_append(const void* k_new, int64_t k_sb, int64_t k_st, int64_t k_sh, const void* v_new,
                                int64_t v_sb, int64_t v_st, int64_t v_sh, const dustin_kv4* k, const dustin_kv4* v,
                                const dustin_batch* bt, void* stream) {
  return kv4_rows(true, k_new, k_sb, k_st, k_sh, v_new, v_sb, v_st, v_sh, k, v, bt, stream);
}

dustin_status dustin_kv4_read(void* k_out, int64_t k_sb, int64_t k_st, int64_t k_sh, void* v_out, int64_t v_sb,
                              int64_t v_st, int64_t v_sh, const dustin_kv4* k, const dustin_kv4* v,
                              const dustin_batch* bt, void* stream) {
  return kv4_rows(false, k_out, k_sb, k_st, k_sh, v_out, v_sb, v_st, v_sh, k, v, bt, stream);
}

size_t dustin_attn_kv4_workspace(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t nq_max,
                                 int32_t max_tokens) {
  if (batch <= 0 || num_kv_heads <= 0 || num_q_heads <= 0 || num_q_heads % num_kv_heads || nq_max <= 0 || max_tokens < 0)
    return 0;
  const int64_t pairs = (int64_t)batch * num_kv_heads;
  const int64_t rows = (int64_t)nq_max * (num_q_heads / num_kv_heads);
  return attn4_ws_bytes(pairs, (int64_t)max_tokens + nq_max, rows);
}

dustin_status dustin_sparse_verify_attn_kv4(const void* q, int64_t q_sb, int64_t q_st, int64_t q_sh,
                                            int32_t num_q_heads, const dustin_kv4* k, const dustin_kv4* v,
                                            const dustin_batch* bt, const int32_t* idx, int64_t idx_sb, int64_t idx_sg,
                                            const int32_t* count, int32_t groups, float scale, void* out, int64_t o_sb,
                                            int64_t o_st, int64_t o_sh, void* workspace, size_t workspace_bytes,
                                            void* stream) {
  return attn4(true, q, q_sb, q_st, q_sh, num_q_heads, k, v, bt, idx, idx_sb, idx_sg, count, groups, scale, out, o_sb,
               o_st, o_sh, workspace, workspace_bytes, stream);
}

dustin_status dustin_dense_verify_attn_kv4(const void* q, int64_t q_sb, int64_t q_st, int64_t q_sh,
                                           int32_t num_q_heads, const dustin_kv4* k, const dustin_kv4* v,
                                           const dustin_batch* bt, float scale, void* out, int64_t o_sb, int64_t o_st,
                                           int64_t o_sh, void* workspace, size_t workspace_bytes, void* stream) {
  return attn4(false, q, q_sb, q_st, q_sh, num_q_heads, k, v, bt, nullptr, 0, 0, nullptr, 1, scale, out, o_sb, o_st,
               o_sh, workspace, workspace_bytes, stream);
}

dustin_status dustin_kv_evict(const dustin_kv* k, const dustin_kv* v, const dustin_kv* k_out, const dustin_kv* v_out,
                              int32_t batch, const int32_t* idx, int64_t idx_sb, int64_t idx_sg, const int32_t* count,
                              int32_t groups, int32_t k_max, const float* w, int64_t w_sb, int64_t w_sg, int32_t w_len,
                              float* w_out, int64_t wo_sb, int64_t wo_sg, int32_t* new_lens, void* stream) {
  return evict(k, v, k_out, v_out, batch, idx, idx_sb, idx_sg, count, groups, k_max, w, w_sb, w_sg, w_len, w_out, wo_sb,
               wo_sg, new_lens, 4, false, stream);
}

dustin_status dustin_kv4_evict(const dustin_kv4* k, const dustin_kv4* v, const dustin_kv4* k_out,
                               const dustin_kv4* v_out, int32_t batch, const int32_t* idx, int64_t idx_sb,
                               int64_t idx_sg, const int32_t* count, int32_t groups, int32_t k_max, const float* w,
                               int64_t w_sb, int64_t w_sg, int32_t w_len, float* w_out, int64_t wo_sb, int64_t wo_sg,
                               int32_t* new_lens, void* stream) {
  return evict(k, v, k_out, v_out, batch, idx, idx_sb, idx_sg, count, groups, k_max, w, w_sb, w_sg, w_len, w_out, wo_sb,
               wo_sg, new_lens, 1, true, stream);
}

}  // extern "C"
