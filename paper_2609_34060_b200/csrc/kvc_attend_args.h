// Argument checks shared by the C entry points that work on requests over a cache: extents of what a call reads and
// writes, 8-bit caches, request lists, packed rows.  Host code.
#pragma once
#include <stdint.h>

#include "kvc_attend.h"

namespace kvc {

struct Extent {
  uintptr_t lo, hi;
};
inline Extent extent_of(const void* p, int64_t last_elem, int elem) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)last_elem * elem};
}
inline bool overlap(const Extent& a, const Extent& b) { return a.lo < b.hi && b.lo < a.hi; }

// elements a cache's K (or V) buffer reaches
inline int64_t cache_reach(const kvc_cache* c, const DevCache& d) {
  int64_t last = (int64_t)(c->L - 1) * d.s_layer + (int64_t)(c->H - 1) * d.s_head + c->d;
  last += is_paged(d) ? (int64_t)(c->n_phys_pages - 1) * d.s_page + (int64_t)(c->page_size - 1) * d.s_tok
                      : (int64_t)(c->T > 0 ? c->T - 1 : 0) * d.s_tok;
  return last;
}

// The runs of bytes a cache's codes or exponents take: one of `width` bytes for every (layer, page, head, token).
struct Runs {
  uintptr_t at;
  int64_t n[4], s[4], width;       // counts, distances in bytes
  Extent all() const {
    int64_t last = width;
    for (int i = 0; i < 4; ++i) {
      if (n[i] <= 0) return {at, at};
      last += (n[i] - 1) * s[i];
    }
    return {at, at + (uintptr_t)last};
  }
};
inline Runs runs_of(const void* p, const kvc_cache& c, int64_t s_layer, int64_t s_page, int64_t s_head, int64_t s_tok, int64_t width) {
  const bool paged = c.layout == KVC_PAGED;
  return {reinterpret_cast<uintptr_t>(p), {c.L, paged ? c.n_phys_pages : 1, c.H, paged ? c.page_size : c.T}, {s_layer, paged ? s_page : 0, s_head, s_tok}, width};
}
inline Runs exponent_runs(const uint8_t* p, const kvc_cache& c, const DevScale& e) { return runs_of(p, c, e.s_layer, e.s_page, e.s_head, e.s_tok, 1); }
inline Runs code_runs(const void* p, const kvc_cache& c, const DevCache& d) { return runs_of(p, c, d.s_layer, d.s_page, d.s_head, d.s_tok, c.d); }

// Whether two sets of runs share a byte.  Sets with the same distances may lie inside one another (keys' and values'
// exponents side by side, exponents behind their row of codes): there the question is whether the distance of their
// beginnings is a whole number of steps, level by level, give or take a run; otherwise overlapping extents decide.
inline bool meet(const Runs& a, const Runs& b) {
  if (!overlap(a.all(), b.all())) return false;
  int order[4] = {0, 1, 2, 3}, live = 0;
  for (int i = 0; i < 4; ++i) {
    if (a.n[i] != b.n[i] || (a.n[i] > 1 && a.s[i] != b.s[i])) return true;
    if (a.n[i] > 1) order[live++] = i;
  }
  for (int i = 1; i < live; ++i)                                  // smallest distance first
    for (int j = i; j > 0 && a.s[order[j]] < a.s[order[j - 1]]; --j) {
      const int t = order[j];
      order[j] = order[j - 1];
      order[j - 1] = t;
    }
  int64_t reach[5] = {a.width > b.width ? a.width : b.width};    // of the levels below
  for (int i = 0; i < live; ++i) {
    const int64_t s = a.s[order[i]];
    if (s < reach[i]) return true;                                // levels that are not inside one another
    reach[i + 1] = reach[i] + (a.n[order[i]] - 1) * s;
  }
  struct Search {
    const int64_t *n, *s, *reach;
    const int* order;
    int64_t wa, wb;
    bool at(int level, int64_t delta) const {                     // delta: b's position less a's
      if (level == 0) return delta < wa && -delta < wb;
      const int i = order[level - 1];
      const int64_t q = delta / s[i];
      for (int64_t t = q - 1; t <= q + 1; ++t)
        if (t > -n[i] && t < n[i] && delta - t * s[i] < reach[level - 1] && t * s[i] - delta < reach[level - 1] && at(level - 1, delta - t * s[i])) return true;
      return false;
    }
  };
  return Search{a.n, a.s, reach, order, a.width, b.width}.at(live, (int64_t)(b.at - a.at));
}
// An 8-bit cache that is written: exponents apart from one another and from the codes.
inline bool exponents_apart(const kvc_qcache* q, const DevCache& c, const DevScale& e) {
  const Runs ek = exponent_runs(e.k, q->codes, e), ev = exponent_runs(e.v, q->codes, e);
  const Runs ck = code_runs(q->codes.k, q->codes, c), cv = code_runs(q->codes.v, q->codes, c);
  return !(meet(ek, ev) || meet(ek, ck) || meet(ek, cv) || meet(ev, ck) || meet(ev, cv));
}

inline int resolve_qcache(const kvc_qcache* q, DevCache* c, DevScale* e) {
  if (!q) return KVC_E_INVALID_ARG;
  const int rc = resolve_cache(&q->codes, c);
  if (rc != KVC_OK) return rc;
  if (!q->scale_k || !q->scale_v) return KVC_E_INVALID_ARG;
  if (q->e_layer < 0 || q->e_page < 0 || q->e_head < 0 || q->e_tok < 0) return KVC_E_INVALID_ARG;
  if ((c->s_tok | c->s_head | c->s_layer | c->s_page) & 15) return KVC_E_UNSUPPORTED;   // 16-byte rows of codes
  const kvc_cache& g = q->codes;
  e->k = q->scale_k;
  e->v = q->scale_v;
  e->s_tok = q->e_tok ? q->e_tok : 1;
  if (g.layout == KVC_CONTIG) {
    e->s_head = q->e_head ? q->e_head : (int64_t)g.T * e->s_tok;
    e->s_layer = q->e_layer ? q->e_layer : (int64_t)g.H * e->s_head;
    e->s_page = 0;
  } else {
    e->s_head = q->e_head ? q->e_head : (int64_t)g.page_size * e->s_tok;
    e->s_page = q->e_page ? q->e_page : (int64_t)g.H * e->s_head;
    e->s_layer = q->e_layer ? q->e_layer : (int64_t)g.n_phys_pages * e->s_page;
  }
  return KVC_OK;
}

// Positions are 32-bit integers, and the kernels step up to two tiles past the last one.
constexpr int32_t kMaxTokens = 0x7fffffff - 256;

// the lists alone (c == nullptr), or with the cache the requests live in
inline int resolve_requests(const kvc_requests* r, const kvc_cache* c, int n_rows, DevRequests* out) {
  if (!r || r->n < 0 || r->max_q < 0 || r->max_kv < 0 || r->table_stride < 0 || n_rows < 0) return KVC_E_INVALID_ARG;
  if (r->n > 0 && (!r->q_begin || !r->kv_len)) return KVC_E_INVALID_ARG;
  int64_t cap = c ? c->T : r->max_kv;
  if (!c) {
  } else if (r->page_table) {
    if (c->layout != KVC_PAGED) return KVC_E_INVALID_ARG;
    cap = (int64_t)r->table_stride * c->page_size;
  } else if (c->layout == KVC_PAGED && !c->page_table && r->max_kv > 0) {
    return KVC_E_INVALID_ARG;
  }
  if (r->max_kv > cap) return KVC_E_SHAPE;
  if (r->max_kv > kMaxTokens) return KVC_E_UNSUPPORTED;
  out->q_begin = r->q_begin;
  out->kv_len = r->kv_len;
  out->table = r->page_table;
  out->table_stride = r->table_stride;
  out->n = r->n;
  out->max_q = r->max_q;
  out->max_kv = r->max_kv;
  out->n_rows = n_rows;
  return KVC_OK;
}

inline int resolve_heads(const kvc_heads* h, int d, DevHeads* out, Extent* ext) {
  if (!h || h->n_rows < 0 || h->n_heads <= 0 || h->s_row < 0 || h->s_head < 0) return KVC_E_INVALID_ARG;
  if (!h->data && h->n_rows > 0) return KVC_E_INVALID_ARG;
  out->p = reinterpret_cast<__nv_bfloat16*>(h->data);
  out->s_head = h->s_head ? h->s_head : d;
  out->s_row = h->s_row ? h->s_row : (int64_t)h->n_heads * out->s_head;
  if (((out->s_head | out->s_row) & 7) || (reinterpret_cast<uintptr_t>(h->data) & 15)) return KVC_E_UNSUPPORTED;
  *ext = extent_of(h->data, h->n_rows > 0 ? (int64_t)(h->n_rows - 1) * out->s_row + (int64_t)(h->n_heads - 1) * out->s_head + d : 0, 2);
  return KVC_OK;
}

inline bool overlap_any(const Extent& w, const Extent* r, int n) {
  for (int i = 0; i < n; ++i)
    if (overlap(w, r[i])) return true;
  return false;
}

// What every call on a tree asks of it: room for max_q bits a row.
inline int check_tree(const kvc_tree* t, const kvc_requests* req) {
  if (!t || t->words < 0 || t->n_rows < 0) return KVC_E_INVALID_ARG;
  if (!req || req->max_q < 0) return KVC_E_INVALID_ARG;
  if (req->max_q > KVC_TREE_MAX_Q) return KVC_E_UNSUPPORTED;
  if ((int64_t)t->words * 32 < req->max_q) return KVC_E_SHAPE;
  if ((reinterpret_cast<uintptr_t>(t->parent) | reinterpret_cast<uintptr_t>(t->mask) | reinterpret_cast<uintptr_t>(t->depth)) & 3) return KVC_E_UNSUPPORTED;
  return KVC_OK;
}

// Whether two sets of packed rows share no byte: slices of one projection's output lie in one another's extent, row by row
// side by side.
inline bool rows_apart(const kvc_heads* a, const DevHeads& da, const Extent& ea, const kvc_heads* b, const DevHeads& db, const Extent& eb, int d) {
  if (!overlap(ea, eb)) return true;
  if (da.s_row != db.s_row || da.s_row <= 0) return false;
  const int64_t wa = ((int64_t)(a->n_heads - 1) * da.s_head + d) * 2, wb = ((int64_t)(b->n_heads - 1) * db.s_head + d) * 2, step = da.s_row * 2;
  int64_t off = (int64_t)(eb.lo - ea.lo) % step;                  // of b's rows behind a's
  if (off < 0) off += step;
  return off >= wa && off + wb <= step;
}

}  // namespace kvc
