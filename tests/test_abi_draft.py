"""Refusals of the operators on drafted tokens: argument checks before anything touches a device."""
import ctypes as C

import pytest

import paper_2609_34060_b200 as kvc
from paper_2609_34060_b200 import build as kbuild

# addresses far apart, never touched
A, B_, Q, O, T_, K, V, X, Y, Z, W = (0x10000000 * i for i in range(1, 12))
INVALID, SHAPE, UNSUPPORTED, ALIAS, WORKSPACE = -1, -2, -3, -4, -6
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return kvc.load()


def _p(x):
    return None if x is None else C.byref(x)


def _pool(**kw):
    c = kvc.kvc_cache()
    c.k, c.v, c.L, c.H, c.T, c.d, c.layout, c.page_size, c.n_phys_pages = A, B_, 2, 2, 0, 128, kvc.KVC_PAGED, 16, 64
    for a, b in kw.items():
        setattr(c, a, b)
    return c


def _q8(scale_k=0xC0000000, scale_v=0xD0000000, **kw):
    q = kvc.kvc_qcache()
    q.codes, q.scale_k, q.scale_v = _pool(**kw), scale_k, scale_v
    return q


def _req(n=2, max_q=4, max_kv=64, stride=4, q_begin=T_, kv_len=T_ + 64, table=T_ + 4096):
    return kvc.kvc_requests(n, max_q, max_kv, stride, q_begin, kv_len, table)


def _heads(p, rows=8, heads=2, s_row=0, s_head=0):
    return kvc.kvc_heads(p, rows, heads, s_row, s_head)


def _tree(words=1, rows=8, parent=X, mask=Y, depth=Z):
    return kvc.kvc_tree(words, rows, parent, mask, depth)


def _rot(theta=1e4, pairing=0, amplitude=1.0, rot=0, depth=0, begin=0, inv=None):
    r = kvc.kvc_rotary()
    r.rope.theta, r.rope.pairing, r.amplitude, r.rot_dim, r.depth, r.pos_begin = theta, pairing, amplitude, rot, depth, begin
    r.rope.inv_freq = None if inv is None else C.cast(inv, C.c_void_p)
    return r


def _probs(p=Q, rows=8, n=100, s=0):
    return kvc.kvc_probs(p, rows, n, s)


def test_struct_sizes(lib):
    assert C.sizeof(kvc.kvc_tree) == 8 + 24 and C.sizeof(kvc.kvc_rotary) == C.sizeof(kvc.kvc_rope) + 8 + 8 + 16
    assert C.sizeof(kvc.kvc_probs) == 8 + 8 + 8


def test_tree_build_refusals(lib):
    tb = lambda req=None, tree=None: lib.kvc_tree_build(_p(req or _req()), _p(tree or _tree()), None)
    assert lib.kvc_tree_build(None, _p(_tree()), None) == INVALID and lib.kvc_tree_build(_p(_req()), None, None) == INVALID
    assert tb(tree=_tree(words=-1)) == INVALID and tb(tree=_tree(rows=-1)) == INVALID
    for k in ("parent", "mask", "depth"):
        assert tb(tree=_tree(**{k: 0})) == INVALID and tb(tree=_tree(**{k: X + 2})) == UNSUPPORTED
    assert tb(req=_req(max_q=33)) == SHAPE and tb(req=_req(max_q=1025), tree=_tree(words=64)) == UNSUPPORTED
    assert tb(req=_req(n=-1)) == INVALID and tb(req=_req(q_begin=0)) == INVALID and tb(req=_req(max_q=-1)) == INVALID and tb(req=_req(max_kv=-1)) == INVALID
    for bad in (_tree(mask=X + 16), _tree(depth=X), _tree(depth=Y + 28), _tree(mask=T_), _tree(depth=T_ + 64)):
        assert tb(tree=bad) == ALIAS
    assert tb(req=_req(n=0)) == 0 and tb(req=_req(max_q=0)) == 0 and tb(tree=_tree(rows=0, parent=0, mask=0, depth=0)) == 0
    assert tb(req=_req(n=0, table=0)) == 0                                              # the page table is not looked at


def test_attend_tree_refusals(lib):
    def at(req=None, tree=None, q=None, c=None, layer=0, scale=0.1, out=None, lse=0, ws=0, n=0):
        return lib.kvc_attend_tree(_p(req or _req()), _p(tree or _tree()), _p(q or _heads(Q, heads=8)), _p(c or _pool()), layer, scale,
                                   _p(out or _heads(O, heads=8)), lse, ws, n, None)
    assert lib.kvc_attend_tree(_p(_req()), None, _p(_heads(Q, heads=8)), _p(_pool()), 0, 0.1, _p(_heads(O, heads=8)), 0, 0, 0, None) == INVALID
    assert lib.kvc_attend_tree(None, _p(_tree()), _p(_heads(Q, heads=8)), _p(_pool()), 0, 0.1, _p(_heads(O, heads=8)), 0, 0, 0, None) == INVALID
    assert at(tree=_tree(mask=0)) == INVALID and at(tree=_tree(words=0)) == SHAPE and at(tree=_tree(rows=7)) == SHAPE
    assert at(req=_req(max_q=33, max_kv=64)) == SHAPE and at(req=_req(max_q=1025), tree=_tree(words=64)) == UNSUPPORTED
    assert at(tree=_tree(mask=Y + 1)) == UNSUPPORTED
    assert at(layer=2) == INVALID and at(scale=0.0) == INVALID and at(c=_pool(d=96)) == UNSUPPORTED and at(out=_heads(O, heads=4)) == SHAPE
    assert at(out=_heads(Y - 64, heads=8)) == ALIAS and at(lse=Y) == ALIAS and at(out=_heads(A, heads=8)) == ALIAS
    need = lib.kvc_attend_workspace_bytes(_p(_req()), 8, 2, 128)
    if need:
        assert at() == WORKSPACE and at(ws=W, n=need - 1) == WORKSPACE
        assert at(tree=_tree(mask=W + 256), ws=W, n=need) == ALIAS
    assert at(req=_req(n=0)) == 0 and at(req=_req(max_q=0)) == 0 and at(tree=_tree(parent=0, depth=0), req=_req(n=0)) == 0
    q8 = lambda c: lib.kvc_attend_tree_q8(_p(_req()), _p(_tree()), _p(_heads(Q, heads=8)), _p(c), 0, 0.1, _p(_heads(O, heads=8)), 0, 0, 0, None)
    assert q8(None) == INVALID and q8(_q8(scale_k=0)) == INVALID


def test_append_rotated_refusals(lib):
    def ap(req=None, rot=None, q=None, out=None, k=None, v=None, layer=0, c=None):
        return lib.kvc_append_rotated(_p(req or _req()), _p(rot or _rot()), _p(q), _p(out), _p(k or _heads(K)), _p(v or _heads(V)), layer, _p(c or _pool()), None)
    q, o = _heads(Q, heads=8), _heads(O, heads=8)
    assert lib.kvc_append_rotated(_p(_req()), None, None, None, _p(_heads(K)), _p(_heads(V)), 0, _p(_pool()), None) == INVALID
    assert lib.kvc_append_rotated(_p(_req()), _p(_rot()), None, None, None, _p(_heads(V)), 0, _p(_pool()), None) == INVALID
    assert lib.kvc_append_rotated(None, _p(_rot()), None, None, _p(_heads(K)), _p(_heads(V)), 0, _p(_pool()), None) == INVALID
    assert ap(layer=2) == INVALID and ap(layer=-1) == INVALID and ap(c=_pool(v=0)) == INVALID
    assert ap(q=q) == INVALID and ap(out=o) == INVALID                                   # one without the other
    assert ap(rot=_rot(pairing=2)) == INVALID and ap(rot=_rot(theta=0.0)) == INVALID and ap(rot=_rot(theta=NAN)) == INVALID
    for a in (NAN, INF, 1e300):
        assert ap(rot=_rot(amplitude=a)) == INVALID
    assert ap(rot=_rot(rot=-16)) == INVALID and ap(rot=_rot(rot=144)) == SHAPE and ap(rot=_rot(rot=24)) == UNSUPPORTED and ap(rot=_rot(rot=8)) == UNSUPPORTED
    assert ap(rot=_rot(inv=(C.c_double * 64)(*([1.0] * 63 + [NAN])))) == INVALID
    assert ap(rot=_rot(depth=X + 1)) == UNSUPPORTED and ap(rot=_rot(begin=X + 2)) == UNSUPPORTED
    assert ap(k=_heads(K, heads=3)) == SHAPE and ap(v=_heads(V, rows=7)) == SHAPE and ap(q=_heads(Q, rows=7, heads=8), out=o) == SHAPE
    assert ap(q=q, out=_heads(O, heads=7)) == SHAPE and ap(q=q, out=_heads(O, rows=9, heads=8)) == SHAPE
    assert ap(req=_req(max_kv=65)) == SHAPE and ap(c=_pool(layout=kvc.KVC_CONTIG, T=64), req=_req(table=0)) == INVALID
    assert ap(k=_heads(K + 8)) == UNSUPPORTED and ap(c=_pool(d=96)) == UNSUPPORTED
    for bad in (dict(k=_heads(A)), dict(v=_heads(B_)), dict(c=_pool(v=A)), dict(q=q, out=_heads(K, heads=8)), dict(q=q, out=_heads(A, heads=8)),
                dict(q=q, out=_heads(T_, heads=8)), dict(q=q, out=_heads(Q + 256, heads=8)), dict(q=q, out=_heads(Q, heads=8, s_row=2048)),
                dict(rot=_rot(depth=A)), dict(rot=_rot(begin=B_ + 4)), dict(rot=_rot(depth=O), q=q, out=o), dict(req=_req(q_begin=A)),
                dict(q=q, out=_heads(O, heads=8, s_row=128)), dict(q=q, out=_heads(O, heads=8, s_head=64))):
        assert ap(**bad) == ALIAS, bad
    # slices of one projection's output of 12 heads a row, in place: nothing shared but the extents (n = 0: checks alone)
    row, none = 12 * 128, _req(n=0)
    part = lambda at, heads: _heads(Q + at * 256, heads=heads, s_row=row)
    assert ap(req=none, q=part(0, 8), out=part(0, 8), k=part(8, 2), v=part(10, 2)) == 0
    assert ap(req=none, q=part(0, 8), out=part(2, 8), k=part(8, 2), v=part(10, 2)) == ALIAS
    assert ap(req=none, q=part(0, 8), out=part(0, 8), k=part(7, 2), v=part(10, 2)) == ALIAS
    assert ap(req=none, q=part(4, 8), out=part(4, 8), k=part(0, 2), v=part(2, 2)) == 0
    assert ap(req=none, q=part(5, 8), out=part(5, 8), k=part(0, 2), v=part(2, 2)) == ALIAS   # the last head is the next row's first
    assert ap(req=_req(max_q=0)) == 0 and ap(k=_heads(K, rows=0), v=_heads(V, rows=0)) == 0
    q8 = lambda c: lib.kvc_append_rotated_q8(_p(_req()), _p(_rot()), None, None, _p(_heads(K)), _p(_heads(V)), 0, _p(c), None)
    assert q8(None) == INVALID and q8(_q8(scale_v=0)) == INVALID and q8(_q8(scale_v=0xC0000000)) == ALIAS and q8(_q8(scale_k=K)) == ALIAS
    assert q8(_q8(scale_k=A + 64)) == ALIAS


def test_verify_refusals(lib):
    def ve(req=None, parent=X, token=Y, t=None, d=None, u=Z, un=K, kept=O, stride=4, nk=V, nxt=W):
        return lib.kvc_verify(_p(req or _req()), parent, token, _p(t or _probs()), _p(d), u, un, kept, stride, nk, nxt, None)
    assert lib.kvc_verify(_p(_req()), X, Y, None, None, Z, K, O, 4, V, W, None) == INVALID and lib.kvc_verify(None, X, Y, _p(_probs()), None, Z, K, O, 4, V, W, None) == INVALID
    for k in ("parent", "token", "u", "un", "kept", "nk", "nxt"):
        assert ve(**{k: 0}) == INVALID and ve(**{k: 0xE0000002}) == UNSUPPORTED
    assert ve(t=_probs(p=0)) == INVALID and ve(t=_probs(rows=-1)) == INVALID and ve(t=_probs(n=0)) == INVALID and ve(t=_probs(s=-4)) == INVALID
    assert ve(t=_probs(p=Q + 2)) == UNSUPPORTED and ve(t=_probs(s=99)) == UNSUPPORTED
    assert ve(d=_probs(A, n=99)) == SHAPE and ve(d=_probs(A, rows=7)) == SHAPE and ve(d=_probs(p=0)) == INVALID
    assert ve(stride=3) == SHAPE and ve(stride=-1) == INVALID and ve(req=_req(max_q=1025), stride=2000) == UNSUPPORTED
    assert ve(req=_req(n=-1)) == INVALID and ve(req=_req(kv_len=0)) == INVALID
    for bad in (dict(kept=Q), dict(nk=Q + 8 * 100 * 4 - 4), dict(nxt=X), dict(kept=Y + 28), dict(nk=Z), dict(nxt=K + 4), dict(nk=O + 16), dict(nxt=V), dict(kept=T_),
                dict(nxt=T_ + 64), dict(d=_probs(A), kept=A + 3196)):
        assert ve(**bad) == ALIAS, bad
    assert ve(req=_req(n=0)) == 0 and ve(req=_req(n=0), parent=0, token=0, u=0, un=0, kept=0, nk=0, nxt=0, t=_probs(p=0, rows=0)) == 0


def test_keep_refusals(lib):
    def ke(req=None, kept=X, stride=4, nk=Y, c=None, out=Z):
        return lib.kvc_keep(_p(req or _req()), kept, stride, nk, _p(c or _pool()), out, None)
    assert lib.kvc_keep(None, X, 4, Y, _p(_pool()), Z, None) == INVALID and lib.kvc_keep(_p(_req()), X, 4, Y, None, Z, None) == INVALID
    assert ke(kept=0) == INVALID and ke(nk=0) == INVALID and ke(stride=-1) == INVALID and ke(stride=3) == SHAPE
    for k in ("kept", "nk", "out"):
        assert ke(**{k: 0xE0000001}) == UNSUPPORTED
    assert ke(req=_req(max_q=1025), stride=1025) == UNSUPPORTED and ke(req=_req(max_kv=65)) == SHAPE and ke(req=_req(q_begin=0)) == INVALID
    assert ke(c=_pool(layout=kvc.KVC_CONTIG, T=64), req=_req(table=0)) == INVALID and ke(c=_pool(d=96)) == UNSUPPORTED
    for bad in (dict(out=T_ + 64), dict(out=X), dict(out=Y), dict(out=A), dict(out=T_), dict(kept=A), dict(nk=B_), dict(c=_pool(v=A)), dict(out=T_ + 4096 + 4)):
        assert ke(**bad) == ALIAS, bad
    assert ke(req=_req(n=0)) == 0
    q8 = lambda c, out=Z: lib.kvc_keep_q8(_p(_req()), X, 4, Y, _p(c), out, None)
    assert q8(None) == INVALID and q8(_q8(scale_k=0)) == INVALID and q8(_q8(scale_v=0xC0000000)) == ALIAS and q8(_q8(), out=0xC0000000) == ALIAS
