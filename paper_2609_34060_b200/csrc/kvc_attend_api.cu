// C ABI of kvc_append, kvc_attend, kvc_quantize and kvc_dequantize: argument checks, descriptor resolution, dispatch.
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "kvc_attend.h"
#include "kvc_launch.h"
#include "kvc_tc.h"

namespace kvc {
namespace {

struct Extent {
  uintptr_t lo, hi;
};
Extent extent_of(const void* p, int64_t last_elem, int elem) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)last_elem * elem};
}
bool overlap(const Extent& a, const Extent& b) { return a.lo < b.hi && b.lo < a.hi; }

// elements a cache's K (or V) buffer reaches
int64_t cache_reach(const kvc_cache* c, const DevCache& d) {
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
Runs runs_of(const void* p, const kvc_cache& c, int64_t s_layer, int64_t s_page, int64_t s_head, int64_t s_tok, int64_t width) {
  const bool paged = c.layout == KVC_PAGED;
  return {reinterpret_cast<uintptr_t>(p), {c.L, paged ? c.n_phys_pages : 1, c.H, paged ? c.page_size : c.T}, {s_layer, paged ? s_page : 0, s_head, s_tok}, width};
}
Runs exponent_runs(const uint8_t* p, const kvc_cache& c, const DevScale& e) { return runs_of(p, c, e.s_layer, e.s_page, e.s_head, e.s_tok, 1); }
Runs code_runs(const void* p, const kvc_cache& c, const DevCache& d) { return runs_of(p, c, d.s_layer, d.s_page, d.s_head, d.s_tok, c.d); }

// Whether two sets of runs share a byte.  Sets with the same distances may lie inside one another (keys' and values'
// exponents side by side, exponents behind their row of codes): there the question is whether the distance of their
// beginnings is a whole number of steps, level by level, give or take a run; otherwise overlapping extents decide.
bool meet(const Runs& a, const Runs& b) {
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
bool exponents_apart(const kvc_qcache* q, const DevCache& c, const DevScale& e) {
  const Runs ek = exponent_runs(e.k, q->codes, e), ev = exponent_runs(e.v, q->codes, e);
  const Runs ck = code_runs(q->codes.k, q->codes, c), cv = code_runs(q->codes.v, q->codes, c);
  return !(meet(ek, ev) || meet(ek, ck) || meet(ek, cv) || meet(ev, ck) || meet(ev, cv));
}

int resolve_qcache(const kvc_qcache* q, DevCache* c, DevScale* e) {
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

int resolve_requests(const kvc_requests* r, const kvc_cache* c, int n_rows, DevRequests* out) {
  if (!r || r->n < 0 || r->max_q < 0 || r->max_kv < 0 || r->table_stride < 0 || n_rows < 0) return KVC_E_INVALID_ARG;
  if (r->n > 0 && (!r->q_begin || !r->kv_len)) return KVC_E_INVALID_ARG;
  int64_t cap = c->T;
  if (r->page_table) {
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

int resolve_heads(const kvc_heads* h, int d, DevHeads* out, Extent* ext) {
  if (!h || h->n_rows < 0 || h->n_heads <= 0 || h->s_row < 0 || h->s_head < 0) return KVC_E_INVALID_ARG;
  if (!h->data && h->n_rows > 0) return KVC_E_INVALID_ARG;
  out->p = reinterpret_cast<__nv_bfloat16*>(h->data);
  out->s_head = h->s_head ? h->s_head : d;
  out->s_row = h->s_row ? h->s_row : (int64_t)h->n_heads * out->s_head;
  if (((out->s_head | out->s_row) & 7) || (reinterpret_cast<uintptr_t>(h->data) & 15)) return KVC_E_UNSUPPORTED;
  *ext = extent_of(h->data, h->n_rows > 0 ? (int64_t)(h->n_rows - 1) * out->s_row + (int64_t)(h->n_heads - 1) * out->s_head + d : 0, 2);
  return KVC_OK;
}

int append_common(const kvc_requests* req, const kvc_heads* kn, const kvc_heads* vn, int32_t layer, const kvc_cache* geo, AppendLaunch& a,
                  const kvc_qcache* q8, void* stream) {
  const int elem = q8 ? 1 : 2;
  int rc;
  Extent ek, ev;
  if (layer < 0 || layer >= geo->L) return KVC_E_INVALID_ARG;
  if ((rc = resolve_heads(kn, geo->d, &a.kn, &ek)) != KVC_OK || (rc = resolve_heads(vn, geo->d, &a.vn, &ev)) != KVC_OK) return rc;
  if (kn->n_heads != geo->H || vn->n_heads != geo->H || kn->n_rows != vn->n_rows) return KVC_E_SHAPE;
  if (geo->H > 32767 || (req && (int64_t)req->max_q * geo->H * 2 >= (int64_t)1 << 31)) return KVC_E_UNSUPPORTED;
  if ((rc = resolve_requests(req, geo, kn->n_rows, &a.req)) != KVC_OK) return rc;
  if (!req->page_table && req->n > 1) return KVC_E_INVALID_ARG;
  const int64_t reach = cache_reach(geo, a.dst);
  const Extent ck = extent_of(geo->k, reach, elem), cv = extent_of(geo->v, reach, elem);
  if (overlap(ck, cv) || overlap(ck, ek) || overlap(ck, ev) || overlap(cv, ek) || overlap(cv, ev)) return KVC_E_ALIAS;
  if (q8) {
    const Extent sk = exponent_runs(a.e.k, *geo, a.e).all(), sv = exponent_runs(a.e.v, *geo, a.e).all();
    if (!exponents_apart(q8, a.dst, a.e) || overlap(sk, ek) || overlap(sk, ev) || overlap(sv, ek) || overlap(sv, ev)) return KVC_E_ALIAS;
  }
  a.H = geo->H;
  a.layer = layer;
  if (req->n == 0 || a.req.max_q == 0 || a.req.n_rows == 0) return KVC_OK;
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_append(a, geo->d, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

int convert_common(const kvc_cache* bf, const kvc_qcache* q8, int to8, void* stream) {
  if (!bf || !q8) return KVC_E_INVALID_ARG;
  ConvertLaunch c;
  memset(&c, 0, sizeof(c));
  int rc;
  if ((rc = resolve_cache(bf, &c.bf)) != KVC_OK || (rc = resolve_qcache(q8, &c.q8, &c.e)) != KVC_OK) return rc;
  const kvc_cache& g = q8->codes;
  if (bf->L != g.L || bf->H != g.H || bf->T != g.T || bf->d != g.d) return KVC_E_SHAPE;
  if (g.H > 32767 || g.T > kMaxTokens) return KVC_E_UNSUPPORTED;
  const int64_t rb = cache_reach(bf, c.bf), rq = cache_reach(&g, c.q8);
  const Extent bk = extent_of(bf->k, rb, 2), bv = extent_of(bf->v, rb, 2), qk = extent_of(g.k, rq, 1), qv = extent_of(g.v, rq, 1);
  if (overlap(bk, qk) || overlap(bk, qv) || overlap(bv, qk) || overlap(bv, qv) || (to8 ? overlap(qk, qv) : overlap(bk, bv))) return KVC_E_ALIAS;
  const Extent sk = exponent_runs(c.e.k, g, c.e).all(), sv = exponent_runs(c.e.v, g, c.e).all();
  if (overlap(bk, sk) || overlap(bk, sv) || overlap(bv, sk) || overlap(bv, sv) || (to8 && !exponents_apart(q8, c.q8, c.e))) return KVC_E_ALIAS;
  if (bf->T == 0) return KVC_OK;
  c.L = bf->L;
  c.H = bf->H;
  c.T = bf->T;
  c.to8 = to8;
  if (!(c.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_convert(c, bf->d, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

int attend_common(const kvc_requests* req, const kvc_heads* q, const kvc_cache* geo, int32_t layer, double scale, int32_t causal,
                  kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, AttendLaunch& a, int elem, void* stream) {
  int rc;
  Extent eq, eo;
  if (layer < 0 || layer >= geo->L || !(scale > 0.0) || !isfinite(scale) || !((float)scale > 0.f) || !isfinite((float)scale)) return KVC_E_INVALID_ARG;
  if ((rc = resolve_heads(q, geo->d, &a.q, &eq)) != KVC_OK || (rc = resolve_heads(out, geo->d, &a.out, &eo)) != KVC_OK) return rc;
  if (q->n_heads != out->n_heads || q->n_rows != out->n_rows || q->n_heads % geo->H) return KVC_E_SHAPE;
  if (q->n_heads / geo->H > 64 || geo->H > 65535) return KVC_E_UNSUPPORTED;
  if ((rc = resolve_requests(req, geo, q->n_rows, &a.req)) != KVC_OK) return rc;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return KVC_E_UNSUPPORTED;
  if ((int64_t)req->max_q * (q->n_heads / geo->H) >= (int64_t)1 << 30) return KVC_E_UNSUPPORTED;
  const int64_t reach = cache_reach(geo, a.c);
  const Extent ck = extent_of(geo->k, reach, elem), cv = extent_of(geo->v, reach, elem);
  const Extent el = extent_of(lse, lse ? (int64_t)q->n_rows * q->n_heads : 0, 4);
  // what is read, and what is written: apart from that and from one another
  const Extent none = {0, 0};
  const bool q8 = a.e.k != nullptr;
  const int64_t pages = geo->layout == KVC_PAGED ? ((int64_t)req->max_kv + geo->page_size - 1) / geo->page_size : 0;
  const Extent reads[] = {eq, ck, cv, q8 ? exponent_runs(a.e.k, *geo, a.e).all() : none, q8 ? exponent_runs(a.e.v, *geo, a.e).all() : none,
                          extent_of(req->q_begin, req->n > 0 ? (int64_t)req->n + 1 : 0, 4), extent_of(req->kv_len, req->n, 4),
                          req->page_table && req->n > 0 ? extent_of(req->page_table, (int64_t)(req->n - 1) * req->table_stride + pages, 4)
                                                        : extent_of(geo->page_table, geo->page_table ? pages : 0, 4)};
  auto reads_meet = [&](const Extent& w) {
    for (const Extent& r : reads)
      if (overlap(w, r)) return true;
    return false;
  };
  if (reads_meet(eo) || reads_meet(el) || overlap(el, eo)) return KVC_E_ALIAS;
  if (req->n == 0 || a.req.max_q == 0 || a.req.n_rows == 0) return KVC_OK;
  const size_t need = kvc_attend_workspace_bytes(req, q->n_heads, geo->H, geo->d);
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need)) return KVC_E_WORKSPACE;
  const Extent ew = extent_of(workspace, (int64_t)need, 1);
  if (reads_meet(ew) || overlap(ew, eo) || overlap(ew, el)) return KVC_E_ALIAS;
  a.H = geo->H;
  a.G = q->n_heads / geo->H;
  a.layer = layer;
  a.causal = causal != 0;
  a.scale = (float)scale;
  a.lse = lse;
  a.part = reinterpret_cast<float*>(workspace);
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (path_force() != KVC_PATH_GENERIC) {
    rc = tc_attend(a, geo->L, geo->d, s);
    if (rc == KVC_OK) set_last_path(KVC_PATH_TC);
    if (rc != KVC_E_UNSUPPORTED || path_force() == KVC_PATH_TC) return rc;
  }
  if (launch_attend_generic(a, geo->d, s) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" {

int kvc_quantize(const kvc_cache* src, kvc_qcache* dst, void* stream) { return convert_common(src, dst, 1, stream); }

int kvc_dequantize(const kvc_qcache* src, kvc_cache* dst, void* stream) { return convert_common(dst, src, 0, stream); }

int kvc_append(const kvc_requests* req, const kvc_heads* k_new, const kvc_heads* v_new, int32_t layer, kvc_cache* dst, void* stream) {
  AppendLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_cache(dst, &a.dst);
  return rc != KVC_OK ? rc : append_common(req, k_new, v_new, layer, dst, a, nullptr, stream);
}

int kvc_append_q8(const kvc_requests* req, const kvc_heads* k_new, const kvc_heads* v_new, int32_t layer, kvc_qcache* dst, void* stream) {
  AppendLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_qcache(dst, &a.dst, &a.e);
  return rc != KVC_OK ? rc : append_common(req, k_new, v_new, layer, &dst->codes, a, dst, stream);
}

size_t kvc_attend_workspace_bytes(const kvc_requests* req, int32_t n_heads, int32_t H, int32_t d) {
  if (!req || req->n <= 0 || req->max_q <= 0 || req->max_kv < 0 || req->max_kv > kMaxTokens || H <= 0 || n_heads <= 0 || n_heads % H || (d != 64 && d != 128)) return 0;
  return tc_attend_workspace_bytes(req->n, req->max_q, req->max_kv, n_heads / H, H, d);
}

int kvc_attend(const kvc_requests* req, const kvc_heads* q, const kvc_cache* cache, int32_t layer, double scale, int32_t causal,
               kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttendLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_cache(cache, &a.c);
  return rc != KVC_OK ? rc : attend_common(req, q, cache, layer, scale, causal, out, lse, workspace, workspace_bytes, a, 2, stream);
}

int kvc_attend_q8(const kvc_requests* req, const kvc_heads* q, const kvc_qcache* cache, int32_t layer, double scale, int32_t causal,
                  kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttendLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_qcache(cache, &a.c, &a.e);
  return rc != KVC_OK ? rc : attend_common(req, q, &cache->codes, layer, scale, causal, out, lse, workspace, workspace_bytes, a, 1, stream);
}

}  // extern "C"
