// validate.hpp -- host checks of the arguments that the extern "C" entry points share (internal).
#pragma once

#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include "common.hpp"

namespace dustin {

constexpr size_t kAlign = 256;

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline bool rows_aligned(const void* p, int64_t s0, int64_t s1, int64_t s2) {
  // bf16 rows read or written 16 bytes at a time
  return aligned(p, 16) && s0 % 8 == 0 && s1 % 8 == 0 && s2 % 8 == 0;
}

inline int env_int(const char* name, int fallback) {
  const char* v = getenv(name);
  if (!v || !*v) return fallback;
  const int x = atoi(v);
  return x > 0 ? x : fallback;
}

inline bool batch_ok(const dustin_batch* bt) {
  if (!bt || bt->batch < 0 || bt->max_len < 0 || bt->nq_max < 0 || bt->k_max < 0) return false;
  if (bt->batch > 0 && !bt->seq_lens) return false;
  return true;
}

inline SeqDims dims_of(const dustin_batch* bt) {
  SeqDims d;
  d.seq_lens = bt->seq_lens;
  d.n_query = bt->n_query;
  d.budget = bt->budget;
  d.m = bt->m;
  d.max_len = bt->max_len;
  d.nq_max = bt->nq_max;
  d.k_max = bt->k_max;
  d.m_scalar = bt->m_scalar;
  return d;
}

// Validates a cache view for `need` addressable positions per sequence.
inline dustin_status kv_of(const dustin_kv* kv, int head_dim, int64_t need, KvView* out) {
  if (!kv || !kv->data || kv->num_kv_heads <= 0) return DUSTIN_ERR_INVALID_ARG;
  if (kv->head_dim != head_dim) return DUSTIN_ERR_INVALID_ARG;
  if (!aligned(kv->data, 16) || kv->stride_n % 8 || kv->stride_h % 8 || kv->stride_b % 8 ||
      kv->stride_page % 8)
    return DUSTIN_ERR_INVALID_ARG;
  if (kv->stride_n <= 0 || kv->stride_h < 0 || kv->stride_b < 0) return DUSTIN_ERR_INVALID_ARG;
  memset(out, 0, sizeof *out);
  out->data = static_cast<const uint16_t*>(kv->data);
  out->stride_b = kv->stride_b;
  out->stride_n = kv->stride_n;
  out->stride_h = kv->stride_h;
  if (kv->page_table) {
    const int ps = kv->page_size;
    if (ps <= 0 || (ps & (ps - 1)) || kv->max_pages <= 0 || kv->num_pages <= 0 ||
        kv->stride_page <= 0)
      return DUSTIN_ERR_INVALID_ARG;
    if (!aligned(kv->page_table, 4)) return DUSTIN_ERR_INVALID_ARG;
    int shift = 0;
    while ((1 << shift) < ps) ++shift;
    out->page_table = kv->page_table;
    out->page_shift = shift;
    out->max_pages = kv->max_pages;
    out->num_pages = kv->num_pages;
    out->stride_page = kv->stride_page;
    out->capacity = (int64_t)kv->max_pages * ps;
    if (((int64_t)kv->num_pages << shift) > INT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  } else {
    out->capacity = kv->capacity;
  }
  if (out->capacity < need || out->capacity <= 0) return DUSTIN_ERR_INVALID_ARG;
  if (!kv->page_table && out->capacity > INT32_MAX) return DUSTIN_ERR_UNSUPPORTED;
  return DUSTIN_OK;
}

}  // namespace dustin
