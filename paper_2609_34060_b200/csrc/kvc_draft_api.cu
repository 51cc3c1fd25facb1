// C ABI of kvc_tree_build, kvc_append_rotated, kvc_verify and kvc_keep: argument checks, descriptor resolution, launch.
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "kvc_attend_args.h"
#include "kvc_draft.h"
#include "kvc_launch.h"

namespace kvc {
namespace {

constexpr Extent kNone = {0, 0};
bool off_grid(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }
Extent ints(const void* p, int64_t n) { return extent_of(p, p && n > 0 ? n : 0, 4); }

int32_t pages_of(const kvc_requests* req, const kvc_cache& c) {
  return c.layout == KVC_PAGED ? (int32_t)(((int64_t)req->max_kv + c.page_size - 1) / c.page_size) : 0;
}
Extent table_extent(const kvc_requests* req, const kvc_cache& c) {
  if (req->page_table) return ints(req->page_table, req->n > 0 ? (int64_t)(req->n - 1) * req->table_stride + pages_of(req, c) : 0);
  return ints(c.page_table, pages_of(req, c));
}

// Frequencies in turns a position; false where one is no number.
bool frequencies(const kvc_rope& rope, int rot, double* turns) {
  const double two_pi = 6.283185307179586476925286766559;
  for (int k = 0; k < rot / 2; ++k) {
    const double f = rope.inv_freq ? rope.inv_freq[k] : pow(rope.theta, -2.0 * (double)k / (double)rot);
    if (!isfinite(f)) return false;
    turns[k] = f / two_pi;
  }
  return true;
}

int rotated_common(const kvc_requests* req, const kvc_rotary* rot, const kvc_heads* q, kvc_heads* q_out, const kvc_heads* kn, const kvc_heads* vn,
                   int32_t layer, const kvc_cache* geo, const kvc_qcache* q8, RotateLaunch& a, void* stream) {
  int rc;
  Extent ek, ev, eq = kNone, eo = kNone;
  if (!rot || layer < 0 || layer >= geo->L) return KVC_E_INVALID_ARG;
  if (rot->rope.pairing != KVC_ROPE_HALF && rot->rope.pairing != KVC_ROPE_INTERLEAVED) return KVC_E_INVALID_ARG;
  if (!rot->rope.inv_freq && !(rot->rope.theta > 0.0)) return KVC_E_INVALID_ARG;
  if (!isfinite(rot->amplitude) || !isfinite((float)rot->amplitude) || rot->rot_dim < 0) return KVC_E_INVALID_ARG;
  a.rot = rot->rot_dim ? rot->rot_dim : geo->d;
  if (a.rot > geo->d) return KVC_E_SHAPE;
  if (a.rot % 16 || off_grid(rot->depth) || off_grid(rot->pos_begin)) return KVC_E_UNSUPPORTED;
  if ((q == nullptr) != (q_out == nullptr)) return KVC_E_INVALID_ARG;
  if ((rc = resolve_heads(kn, geo->d, &a.kn, &ek)) != KVC_OK || (rc = resolve_heads(vn, geo->d, &a.vn, &ev)) != KVC_OK) return rc;
  if (q && ((rc = resolve_heads(q, geo->d, &a.q, &eq)) != KVC_OK || (rc = resolve_heads(q_out, geo->d, &a.qo, &eo)) != KVC_OK)) return rc;
  if (kn->n_heads != geo->H || vn->n_heads != geo->H || kn->n_rows != vn->n_rows) return KVC_E_SHAPE;
  if (q && (q->n_rows != kn->n_rows || q_out->n_rows != q->n_rows || q_out->n_heads != q->n_heads)) return KVC_E_SHAPE;
  if (geo->H > 32767 || (q && q->n_heads > 65535)) return KVC_E_UNSUPPORTED;
  if ((rc = resolve_requests(req, geo, kn->n_rows, &a.req)) != KVC_OK) return rc;
  if (!req->page_table && req->n > 1) return KVC_E_INVALID_ARG;
  if (req->max_q > kMaxTokens) return KVC_E_UNSUPPORTED;         // a tile behind the last token is still a 32-bit number
  if (!frequencies(rot->rope, a.rot, a.turns)) return KVC_E_INVALID_ARG;
  // what is written lies apart from what is read, and from one another
  const int64_t reach = cache_reach(geo, a.dst);
  const Extent ck = extent_of(geo->k, reach, q8 ? 1 : 2), cv = extent_of(geo->v, reach, q8 ? 1 : 2);
  const Extent sk = q8 ? exponent_runs(a.e.k, *geo, a.e).all() : kNone, sv = q8 ? exponent_runs(a.e.v, *geo, a.e).all() : kNone;
  const Extent reads[] = {ek, ev, eq, ints(req->q_begin, (int64_t)req->n + 1), ints(req->kv_len, req->n), table_extent(req, *geo), ints(rot->depth, kn->n_rows),
                          ints(rot->pos_begin, req->n)};
  const Extent cache[] = {ck, cv, sk, sv};
  for (const Extent& w : cache)
    if (overlap_any(w, reads, 8) || overlap(w, eo)) return KVC_E_ALIAS;
  if (overlap(ck, cv) || (q8 && !exponents_apart(q8, a.dst, a.e))) return KVC_E_ALIAS;
  if (q) {
    if (overlap_any(eo, reads + 3, 5)) return KVC_E_ALIAS;
    const bool in_place = q->data == q_out->data && a.q.s_row == a.qo.s_row && a.q.s_head == a.qo.s_head;
    // rows written twice would race: heads inside rows, or rows inside heads
    const int64_t wide = (int64_t)(q->n_heads - 1) * a.qo.s_head + geo->d, tall = (int64_t)(q->n_rows - 1) * a.qo.s_row + geo->d;
    if (q->n_rows > 0 && !((a.qo.s_head >= geo->d && a.qo.s_row >= wide) || (a.qo.s_row >= geo->d && a.qo.s_head >= tall) || (q->n_rows == 1 && a.qo.s_head >= geo->d) ||
                           (q->n_heads == 1 && a.qo.s_row >= geo->d)))
      return KVC_E_ALIAS;
    if (!in_place && !rows_apart(q_out, a.qo, eo, q, a.q, eq, geo->d)) return KVC_E_ALIAS;
    if (!rows_apart(q_out, a.qo, eo, kn, a.kn, ek, geo->d) || !rows_apart(q_out, a.qo, eo, vn, a.vn, ev, geo->d)) return KVC_E_ALIAS;
  }
  a.Hq = q ? q->n_heads : 0;
  a.H = geo->H;
  a.layer = layer;
  a.pairing = rot->rope.pairing;
  a.amplitude = rot->amplitude == 0.0 ? 1.f : (float)rot->amplitude;
  a.depth = rot->depth;
  a.pos_begin = rot->pos_begin;
  if (req->n == 0 || a.req.max_q == 0 || a.req.n_rows == 0) return KVC_OK;
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_append_rotated(a, geo->d, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

int resolve_probs(const kvc_probs* p, Extent* ext, int64_t* stride) {
  if (!p || p->n_rows < 0 || p->n < 1 || p->s_row < 0 || (!p->p && p->n_rows > 0)) return KVC_E_INVALID_ARG;
  *stride = p->s_row ? p->s_row : p->n;
  if (off_grid(p->p)) return KVC_E_UNSUPPORTED;
  if (*stride < p->n && p->n_rows > 1) return KVC_E_UNSUPPORTED;
  *ext = extent_of(p->p, p->n_rows > 0 ? (int64_t)(p->n_rows - 1) * *stride + p->n : 0, 4);
  return KVC_OK;
}

int keep_common(const kvc_requests* req, const int32_t* kept, int32_t stride, const int32_t* n_kept, const kvc_cache* geo, const kvc_qcache* q8,
                int32_t* kv_out, KeepLaunch& a, void* stream) {
  int rc;
  if ((rc = resolve_requests(req, geo, 0x7fffffff, &a.req)) != KVC_OK) return rc;
  if (req->max_q > KVC_TREE_MAX_Q) return KVC_E_UNSUPPORTED;
  if (stride < 0 || (req->n > 0 && (!n_kept || (!kept && req->max_q > 0)))) return KVC_E_INVALID_ARG;
  if (stride < req->max_q) return KVC_E_SHAPE;
  if (off_grid(kept) || off_grid(n_kept) || off_grid(kv_out)) return KVC_E_UNSUPPORTED;
  if (!req->page_table && req->n > 1) return KVC_E_INVALID_ARG;
  if ((int64_t)geo->L * geo->H * 2 * 16 >= (int64_t)1 << 31) return KVC_E_UNSUPPORTED;
  const int64_t reach = cache_reach(geo, a.c);
  const Extent ck = extent_of(geo->k, reach, q8 ? 1 : 2), cv = extent_of(geo->v, reach, q8 ? 1 : 2);
  const Extent sk = q8 ? exponent_runs(a.e.k, *geo, a.e).all() : kNone, sv = q8 ? exponent_runs(a.e.v, *geo, a.e).all() : kNone;
  const Extent reads[] = {ints(req->q_begin, (int64_t)req->n + 1), ints(req->kv_len, req->n), table_extent(req, *geo),
                          ints(kept, req->n > 0 ? (int64_t)(req->n - 1) * stride + req->max_q : 0), ints(n_kept, req->n)};
  const Extent writes[] = {ck, cv, sk, sv, ints(kv_out, req->n)};
  for (const Extent& w : writes)
    if (overlap_any(w, reads, 5)) return KVC_E_ALIAS;
  if (overlap_any(writes[4], writes, 4) || overlap(ck, cv) || (q8 && !exponents_apart(q8, a.c, a.e))) return KVC_E_ALIAS;
  if (req->n == 0) return KVC_OK;
  a.L = geo->L;
  a.H = geo->H;
  a.stride = stride;
  a.kept = kept;
  a.n_kept = n_kept;
  a.kv_out = kv_out;
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_keep(a, geo->d, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" {

int kvc_tree_build(const kvc_requests* req, const kvc_tree* tree, void* stream) {
  TreeLaunch a;
  memset(&a, 0, sizeof(a));
  int rc = check_tree(tree, req);
  if (rc != KVC_OK || (rc = resolve_requests(req, nullptr, tree->n_rows, &a.req)) != KVC_OK) return rc;
  if (tree->n_rows > 0 && (!tree->parent || !tree->mask || !tree->depth)) return KVC_E_INVALID_ARG;
  const Extent mask = ints(tree->mask, (int64_t)tree->n_rows * tree->words), depth = ints(tree->depth, tree->n_rows);
  const Extent reads[] = {ints(req->q_begin, (int64_t)req->n + 1), ints(req->kv_len, req->n), ints(tree->parent, tree->n_rows)};
  if (overlap_any(mask, reads, 3) || overlap_any(depth, reads, 3) || overlap(mask, depth)) return KVC_E_ALIAS;
  if (req->n == 0 || req->max_q == 0 || tree->n_rows == 0) return KVC_OK;
  a.parent = tree->parent;
  a.mask = tree->mask;
  a.depth = tree->depth;
  a.words = tree->words;
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_tree_build(a, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

int kvc_append_rotated(const kvc_requests* req, const kvc_rotary* rot, const kvc_heads* q, kvc_heads* q_out, const kvc_heads* k_new,
                       const kvc_heads* v_new, int32_t layer, kvc_cache* dst, void* stream) {
  RotateLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_cache(dst, &a.dst);
  return rc != KVC_OK ? rc : rotated_common(req, rot, q, q_out, k_new, v_new, layer, dst, nullptr, a, stream);
}

int kvc_append_rotated_q8(const kvc_requests* req, const kvc_rotary* rot, const kvc_heads* q, kvc_heads* q_out, const kvc_heads* k_new,
                          const kvc_heads* v_new, int32_t layer, kvc_qcache* dst, void* stream) {
  RotateLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_qcache(dst, &a.dst, &a.e);
  return rc != KVC_OK ? rc : rotated_common(req, rot, q, q_out, k_new, v_new, layer, &dst->codes, dst, a, stream);
}

int kvc_verify(const kvc_requests* req, const int32_t* parent, const int32_t* token, const kvc_probs* target, const kvc_probs* draft,
               const float* u, const float* u_next, int32_t* kept, int32_t kept_stride, int32_t* n_kept, int32_t* next, void* stream) {
  VerifyLaunch a;
  memset(&a, 0, sizeof(a));
  int rc;
  Extent et, ed = kNone;
  if ((rc = resolve_probs(target, &et, &a.s_target)) != KVC_OK || (draft && (rc = resolve_probs(draft, &ed, &a.s_draft)) != KVC_OK)) return rc;
  if (draft && (draft->n != target->n || draft->n_rows != target->n_rows)) return KVC_E_SHAPE;
  if ((rc = resolve_requests(req, nullptr, target->n_rows, &a.req)) != KVC_OK) return rc;
  if (req->max_q > KVC_TREE_MAX_Q || req->n >= 1 << 27) return KVC_E_UNSUPPORTED;
  const bool rows = target->n_rows > 0 && req->max_q > 0;
  if (kept_stride < 0 || (rows && (!parent || !token || !u)) || (req->n > 0 && (!u_next || !n_kept || !next || (!kept && req->max_q > 0)))) return KVC_E_INVALID_ARG;
  if (kept_stride < req->max_q) return KVC_E_SHAPE;
  for (const void* p : {(const void*)parent, (const void*)token, (const void*)u, (const void*)u_next, (const void*)kept, (const void*)n_kept, (const void*)next})
    if (off_grid(p)) return KVC_E_UNSUPPORTED;
  const Extent reads[] = {et, ed, ints(req->q_begin, (int64_t)req->n + 1), ints(req->kv_len, req->n), ints(parent, target->n_rows), ints(token, target->n_rows),
                          ints(u, target->n_rows), ints(u_next, req->n)};
  const Extent writes[] = {ints(kept, req->n > 0 ? (int64_t)(req->n - 1) * kept_stride + req->max_q : 0), ints(n_kept, req->n), ints(next, req->n)};
  for (int i = 0; i < 3; ++i)
    if (overlap_any(writes[i], reads, 8) || overlap_any(writes[i], writes, i)) return KVC_E_ALIAS;
  if (req->n == 0) return KVC_OK;
  a.parent = parent;
  a.token = token;
  a.target = target->p;
  a.draft = draft ? draft->p : nullptr;
  a.vocab = target->n;
  a.stride = kept_stride;
  a.u = u;
  a.u_next = u_next;
  a.kept = kept;
  a.n_kept = n_kept;
  a.next = next;
  if (!(a.status = status_word_ptr())) return KVC_E_CUDA;
  if (launch_verify(a, reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess) return KVC_E_CUDA;
  set_last_path(KVC_PATH_GENERIC);
  return KVC_OK;
}

int kvc_keep(const kvc_requests* req, const int32_t* kept, int32_t kept_stride, const int32_t* n_kept, kvc_cache* cache, int32_t* kv_out, void* stream) {
  KeepLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_cache(cache, &a.c);
  return rc != KVC_OK ? rc : keep_common(req, kept, kept_stride, n_kept, cache, nullptr, kv_out, a, stream);
}

int kvc_keep_q8(const kvc_requests* req, const int32_t* kept, int32_t kept_stride, const int32_t* n_kept, kvc_qcache* cache, int32_t* kv_out,
                void* stream) {
  KeepLaunch a;
  memset(&a, 0, sizeof(a));
  const int rc = resolve_qcache(cache, &a.c, &a.e);
  return rc != KVC_OK ? rc : keep_common(req, kept, kept_stride, n_kept, &cache->codes, cache, kv_out, a, stream);
}

// The same calls from one block of arguments (not part of kvc.h: the Python binding's way in).
int kvc_block_append_rotated(const AppendRotatedCall* c) {
  AppendRotatedCall x = *c;
  if ((x.n_depth >= 0 && x.n_depth < x.k_new.n_rows) || (x.n_pos >= 0 && x.n_pos < x.req->n)) return KVC_E_SHAPE;
  const kvc_heads* q = x.has_q ? &x.q : nullptr;
  kvc_heads* out = x.has_q ? &x.q_out : nullptr;
  return x.q8 ? kvc_append_rotated_q8(x.req, x.rot, q, out, &x.k_new, &x.v_new, x.layer, reinterpret_cast<kvc_qcache*>(x.cache), x.stream)
              : kvc_append_rotated(x.req, x.rot, q, out, &x.k_new, &x.v_new, x.layer, reinterpret_cast<kvc_cache*>(x.cache), x.stream);
}
int kvc_block_attend_tree(const AttendTreeCall* c) {
  AttendTreeCall x = *c;
  if (x.layer != (int32_t)x.layer) return KVC_E_INVALID_ARG;
  return x.q8 ? kvc_attend_tree_q8(x.req, x.tree, &x.q, reinterpret_cast<const kvc_qcache*>(x.cache), (int32_t)x.layer, x.scale, &x.out, x.lse, x.workspace,
                                   (size_t)x.workspace_bytes, x.stream)
              : kvc_attend_tree(x.req, x.tree, &x.q, reinterpret_cast<const kvc_cache*>(x.cache), (int32_t)x.layer, x.scale, &x.out, x.lse, x.workspace,
                                (size_t)x.workspace_bytes, x.stream);
}
int kvc_block_verify(const VerifyCall* c) {
  return kvc_verify(c->req, c->parent, c->token, &c->target, c->has_draft ? &c->draft : nullptr, c->u, c->u_next, c->kept, (int32_t)c->stride, c->n_kept, c->next,
                    c->stream);
}
int kvc_block_keep(const KeepCall* c) {
  return c->q8 ? kvc_keep_q8(c->req, c->kept, (int32_t)c->stride, c->n_kept, reinterpret_cast<kvc_qcache*>(c->cache), c->kv_out, c->stream)
               : kvc_keep(c->req, c->kept, (int32_t)c->stride, c->n_kept, reinterpret_cast<kvc_cache*>(c->cache), c->kv_out, c->stream);
}

}  // extern "C"
