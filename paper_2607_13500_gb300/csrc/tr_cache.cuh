// The paged key/value cache as its kernels see it: where a new token's key
// lies, which page holds a key, and the host checks shared by the append and
// the attention.
#pragma once

#include "tr_internal.cuh"

namespace tr {

struct CacheView {
  void *k, *v;
  int pages, heads, page, d;
  const int32_t *table;
  int batch, max_pages;
  const int32_t *lens, *cu_new;
  int total_new;
};

inline CacheView cache_view(const tr_cache *c) {
  return CacheView{c->k,         c->v,    c->pages,  c->heads,    c->page, c->head_dim, c->table,
                   c->batch, c->max_pages, c->lens, c->cu_new, c->total_new};
}

// The keys of sequence b: lens[b], within what its row of the table can hold.
__device__ __forceinline__ int cache_len(const CacheView &c, int b) {
  const long long most = (long long)c.max_pages * c.page;
  const int n = __ldg(c.lens + b);
  return n < 0 ? 0 : n > most ? (int)most : n;
}

struct NewToken {
  int seq;  // -1: no sequence owns the token
  int key;  // its own key; negative or past the table when lens and cu_new disagree
};
__device__ __forceinline__ NewToken find_token(const CacheView &c, int t) {
  if (c.batch == 0) return NewToken{-1, -1};
  int lo = 0, hi = c.batch;  // the last b with cu_new[b] <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(c.cu_new + mid) <= t) lo = mid; else hi = mid;
  }
  const int first = __ldg(c.cu_new + lo), end = __ldg(c.cu_new + lo + 1);
  NewToken r;
  r.seq = first <= t && t < end ? lo : -1;
  r.key = r.seq < 0 ? -1 : max(__ldg(c.lens + lo), 0) - end + t;
  return r;
}

// Page id of key `key` (>= 0) of sequence b, -1 when the table's row does not
// reach it or names a page outside the cache.
__device__ __forceinline__ int page_of(const CacheView &c, int b, int key) {
  const int i = key / c.page;
  if (i >= c.max_pages) return -1;
  const int id = __ldg(c.table + (long long)b * c.max_pages + i);
  return (unsigned)id < (unsigned)c.pages ? id : -1;
}

// ---------------------------------------------------------------- host checks
inline tr_status check_cache(const tr_cache *c) {
  if (!c || !c->k || !c->v) return TR_ERR_ARG;
  if (c->dtype != TR_BF16 && c->dtype != TR_F16) return TR_ERR_DTYPE;
  if (c->pages < 0 || c->heads <= 0 || c->batch < 0 || c->max_pages < 0 || c->total_new < 0) return TR_ERR_ARG;
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1))) return TR_ERR_UNSUPPORTED;
  if (c->head_dim <= 0) return TR_ERR_ARG;
  if (c->head_dim % 16) return TR_ERR_ALIGN;
  if (c->head_dim > 128) return TR_ERR_UNSUPPORTED;
  if ((long long)c->pages * c->heads * c->page > INT32_MAX) return TR_ERR_UNSUPPORTED;  // key rows are int32
  if ((long long)c->max_pages * c->page > INT32_MAX - 65536) return TR_ERR_UNSUPPORTED;  // and keys of a sequence
  if (c->batch > 0 && (!c->lens || !c->cu_new || (c->max_pages > 0 && !c->table))) return TR_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k) & 15u) || (reinterpret_cast<uintptr_t>(c->v) & 15u) ||
      (reinterpret_cast<uintptr_t>(c->lens) & 3u) || (reinterpret_cast<uintptr_t>(c->cu_new) & 3u) ||
      (reinterpret_cast<uintptr_t>(c->table) & 3u))
    return TR_ERR_ALIGN;
  return TR_OK;
}

inline tr_status check_heads(const tr_heads *h, int es) {
  if (!h || !h->p || h->heads <= 0 || h->token_stride < 0 || h->head_stride < 0) return TR_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(h->p) & 15u) || (h->token_stride * es) % 16 || (h->head_stride * es) % 16)
    return TR_ERR_ALIGN;
  if (h->token_stride > INT32_MAX || h->head_stride > INT32_MAX) return TR_ERR_UNSUPPORTED;  // the kernels multiply 32 x 32 bits
  return TR_OK;
}

}  // namespace tr
