// C ABI of kvc_append, kvc_attend, kvc_attend_tree, kvc_quantize and kvc_dequantize: argument checks, descriptor resolution, dispatch.
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include "kvc_attend_args.h"
#include "kvc_launch.h"
#include "kvc_tc.h"

namespace kvc {
namespace {

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
                  kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, AttendLaunch& a, int elem, void* stream,
                  const kvc_tree* tree = nullptr) {
  int rc;
  Extent eq, eo;
  if (layer < 0 || layer >= geo->L || !(scale > 0.0) || !isfinite(scale) || !((float)scale > 0.f) || !isfinite((float)scale)) return KVC_E_INVALID_ARG;
  if ((rc = resolve_heads(q, geo->d, &a.q, &eq)) != KVC_OK || (rc = resolve_heads(out, geo->d, &a.out, &eo)) != KVC_OK) return rc;
  if (q->n_heads != out->n_heads || q->n_rows != out->n_rows || q->n_heads % geo->H) return KVC_E_SHAPE;
  if (q->n_heads / geo->H > 64 || geo->H > 65535) return KVC_E_UNSUPPORTED;
  if ((rc = resolve_requests(req, geo, q->n_rows, &a.req)) != KVC_OK) return rc;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return KVC_E_UNSUPPORTED;
  if (tree && (rc = check_tree(tree, req)) != KVC_OK) return rc;
  if (tree && tree->n_rows != q->n_rows) return KVC_E_SHAPE;
  if (tree && tree->n_rows > 0 && !tree->mask) return KVC_E_INVALID_ARG;
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
                                                        : extent_of(geo->page_table, geo->page_table ? pages : 0, 4),
                          tree ? extent_of(tree->mask, (int64_t)tree->n_rows * tree->words, 4) : none};
  auto reads_meet = [&](const Extent& w) {
    for (const Extent& r : reads)
      if (overlap(w, r)) return true;
    return false;
  };
  if (reads_meet(eo) || reads_meet(el) || overlap(el, eo)) return KVC_E_ALIAS;
  if (req->n == 0 || a.req.max_q == 0 || a.req.n_rows == 0) return KVC_OK;
  const size_t need = tc_attend_workspace_bytes(req->n, req->max_q, req->max_kv, q->n_heads / geo->H, geo->H, geo->d, tree != nullptr);   // of this call
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
  a.mask = tree ? tree->mask : nullptr;
  a.words = tree ? tree->words : 0;
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
  const size_t plain = tc_attend_workspace_bytes(req->n, req->max_q, req->max_kv, n_heads / H, H, d, false);
  const size_t tree = req->max_q > KVC_TREE_MAX_Q ? 0 : tc_attend_workspace_bytes(req->n, req->max_q, req->max_kv, n_heads / H, H, d, true);
  return plain > tree ? plain : tree;
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

int kvc_attend_tree(const kvc_requests* req, const kvc_tree* tree, const kvc_heads* q, const kvc_cache* cache, int32_t layer, double scale,
                    kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttendLaunch a;
  memset(&a, 0, sizeof(a));
  if (!tree) return KVC_E_INVALID_ARG;
  const int rc = resolve_cache(cache, &a.c);
  return rc != KVC_OK ? rc : attend_common(req, q, cache, layer, scale, 1, out, lse, workspace, workspace_bytes, a, 2, stream, tree);
}

int kvc_attend_tree_q8(const kvc_requests* req, const kvc_tree* tree, const kvc_heads* q, const kvc_qcache* cache, int32_t layer, double scale,
                       kvc_heads* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttendLaunch a;
  memset(&a, 0, sizeof(a));
  if (!tree) return KVC_E_INVALID_ARG;
  const int rc = resolve_qcache(cache, &a.c, &a.e);
  return rc != KVC_OK ? rc : attend_common(req, q, &cache->codes, layer, scale, 1, out, lse, workspace, workspace_bytes, a, 1, stream, tree);
}

}  // extern "C"
