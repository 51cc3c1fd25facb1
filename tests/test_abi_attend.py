"""Refusals of kvc_append, kvc_attend, kvc_quantize and kvc_dequantize: argument checks before anything touches a device."""
import copy
import ctypes as C

import pytest
import torch

import paper_2609_34060_b200 as kvc
from paper_2609_34060_b200 import build as kbuild

A, B_, Q, O, T_ = 0x10000000, 0x20000000, 0x30000000, 0x40000000, 0x50000000     # far apart, never touched
INVALID, SHAPE, UNSUPPORTED, ALIAS, WORKSPACE = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return kvc.load()


def _pool(cls=kvc.kvc_cache, **kw):
    c = kvc.kvc_cache()
    c.k, c.v, c.L, c.H, c.T, c.d, c.layout, c.page_size, c.n_phys_pages = A, B_, 2, 2, 0, 128, kvc.KVC_PAGED, 16, 64
    for a, b in kw.items():
        setattr(c, a, b)
    return c


def _q8(**kw):
    q = kvc.kvc_qcache()
    own = {a: kw.pop(a) for a in list(kw) if a.startswith(("scale", "e_"))}
    q.codes = _pool(**kw)
    q.scale_k, q.scale_v = own.pop("scale_k", 0x60000000), own.pop("scale_v", 0x61000000)
    for a, b in own.items():
        setattr(q, a, b)
    return q


def _req(n=2, max_q=1, max_kv=64, stride=4, q_begin=T_, kv_len=T_ + 64, table=T_ + 4096):
    return kvc.kvc_requests(n, max_q, max_kv, stride, q_begin, kv_len, table)


def _heads(p=Q, rows=8, heads=8, s_row=0, s_head=0):
    return kvc.kvc_heads(p, rows, heads, s_row, s_head)


def _p(x):
    return None if x is None else C.byref(x)


def test_struct_sizes(lib):
    assert C.sizeof(kvc.kvc_requests) == 16 + 24 and C.sizeof(kvc.kvc_heads) == 8 + 8 + 16
    assert C.sizeof(kvc.kvc_qcache) == C.sizeof(kvc.kvc_cache) + 16 + 32


def test_attend_refusals(lib):
    def at(req=None, q=None, c=None, layer=0, scale=0.1, out=None, lse=0, ws=0, n=0):
        return lib.kvc_attend(_p(req or _req()), _p(q or _heads()), _p(c or _pool()), layer, scale, 1, _p(out or _heads(O)), lse, ws, n, None)
    assert lib.kvc_attend(None, _p(_heads()), _p(_pool()), 0, 0.1, 1, _p(_heads(O)), 0, 0, 0, None) == INVALID
    assert lib.kvc_attend(_p(_req()), None, _p(_pool()), 0, 0.1, 1, _p(_heads(O)), 0, 0, 0, None) == INVALID
    assert lib.kvc_attend(_p(_req()), _p(_heads()), None, 0, 0.1, 1, _p(_heads(O)), 0, 0, 0, None) == INVALID
    assert lib.kvc_attend(_p(_req()), _p(_heads()), _p(_pool()), 0, 0.1, 1, None, 0, 0, 0, None) == INVALID
    assert at(layer=2) == INVALID and at(layer=-1) == INVALID
    for s in (0.0, -1.0, float("nan"), float("inf"), 1e300, 1e-60):
        assert at(scale=s) == INVALID
    assert at(c=_pool(d=96)) == UNSUPPORTED and at(c=_pool(page_size=12)) == UNSUPPORTED and at(c=_pool(k=0)) == INVALID
    assert at(q=_heads(heads=9), out=_heads(O, heads=9)) == SHAPE                       # not a multiple of the KV heads
    assert at(out=_heads(O, heads=4)) == SHAPE and at(out=_heads(O, rows=7)) == SHAPE
    assert at(q=_heads(heads=130), out=_heads(O, heads=130)) == UNSUPPORTED             # 65 query heads per KV head
    assert at(q=_heads(s_row=1028)) == UNSUPPORTED and at(q=_heads(p=Q + 8)) == UNSUPPORTED
    assert at(q=_heads(p=0)) == INVALID and at(q=_heads(rows=-1)) == INVALID
    assert at(req=_req(n=-1)) == INVALID and at(req=_req(q_begin=0)) == INVALID and at(req=_req(kv_len=0)) == INVALID
    assert at(req=_req(max_kv=65)) == SHAPE                                             # four pages of 16 hold 64
    assert at(req=_req(table=0)) == INVALID                                             # a pool without a table
    assert at(c=_pool(layout=kvc.KVC_CONTIG, T=64)) == INVALID                          # a table over contiguous rows
    assert at(c=_pool(layout=kvc.KVC_CONTIG, T=63), req=_req(table=0)) == SHAPE
    assert at(out=_heads(Q + 2048)) == ALIAS and at(out=_heads(A)) == ALIAS and at(out=_heads(B_)) == ALIAS
    assert at(lse=O) == ALIAS and at(lse=A + 4) == ALIAS and at(lse=0x70000002) == UNSUPPORTED
    need = lib.kvc_attend_workspace_bytes(_p(_req()), 8, 2, 128)
    if need:
        assert at() == WORKSPACE and at(ws=0x70000000, n=need - 1) == WORKSPACE and at(ws=0x70000010, n=need) == WORKSPACE
    # nothing to do: no launch
    assert at(req=_req(n=0)) == 0 and at(req=_req(max_q=0)) == 0 and at(q=_heads(rows=0), out=_heads(O, rows=0)) == 0
    q8 = lambda c: lib.kvc_attend_q8(_p(_req()), _p(_heads()), _p(c), 0, 0.1, 1, _p(_heads(O)), 0, 0, 0, None)
    assert q8(None) == INVALID and q8(_q8(scale_k=0)) == INVALID and q8(_q8(e_tok=-1)) == INVALID
    assert q8(_q8(s_tok=136)) == UNSUPPORTED                                            # rows of codes off the 16-byte grid


def test_append_refusals(lib):
    def ap(req=None, k=None, v=None, layer=0, c=None):
        return lib.kvc_append(_p(req or _req()), _p(k or _heads(heads=2)), _p(v or _heads(O, heads=2)), layer, _p(c or _pool()), None)
    assert ap(layer=2) == INVALID and ap(c=_pool(v=0)) == INVALID
    assert ap(k=_heads(heads=3)) == SHAPE and ap(v=_heads(O, heads=2, rows=7)) == SHAPE
    assert ap(req=_req(max_kv=65)) == SHAPE
    assert ap(c=_pool(layout=kvc.KVC_CONTIG, T=64), req=_req(table=0)) == INVALID       # two requests, one set of rows
    assert ap(k=_heads(A, heads=2)) == ALIAS and ap(v=_heads(A, heads=2)) == ALIAS and ap(c=_pool(v=A)) == ALIAS
    assert ap(req=_req(n=0)) == 0
    assert lib.kvc_append_q8(_p(_req()), _p(_heads(heads=2)), _p(_heads(O, heads=2)), 0, _p(_q8(scale_v=0)), None) == INVALID
    assert lib.kvc_append(_p(_req()), None, _p(_heads(O, heads=2)), 0, _p(_pool()), None) == INVALID


def test_convert_refusals(lib):
    bf = lambda **kw: _pool(k=Q, v=O, layout=kvc.KVC_CONTIG, T=32, **kw)
    q8 = lambda **kw: _q8(layout=kvc.KVC_CONTIG, **dict(dict(T=32), **kw))
    for f in (lambda b, q: lib.kvc_quantize(_p(b), _p(q), None), lambda b, q: lib.kvc_dequantize(_p(q), _p(b), None)):
        assert f(None, q8()) == INVALID and f(bf(), None) == INVALID
        assert f(bf(), q8(T=33)) == SHAPE and f(bf(), q8(H=3)) == SHAPE and f(bf(), q8(d=64)) == SHAPE
        assert f(bf(), q8(k=Q)) == ALIAS and f(bf(), q8(v=O)) == ALIAS
        assert f(bf(), q8(s_head=32 * 128 + 8)) == UNSUPPORTED
    assert lib.kvc_quantize(_p(bf()), _p(q8(v=A)), None) == ALIAS


def test_binding_refusals():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        kvc.QCache(bf(1, 2, 8, 64), bf(1, 2, 8, 64), torch.zeros(1, 2, 8, dtype=torch.uint8), torch.zeros(1, 2, 8, dtype=torch.uint8))
    with pytest.raises(AssertionError):
        kvc.Requests(torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), 1, 1)
    with pytest.raises(AssertionError):
        kvc.Requests(torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 1, 1)
    with pytest.raises(AssertionError):                     # one table row expanded to all requests has no stride
        kvc.Requests(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 1, 1,
                     page_table=torch.zeros(1, 4, dtype=torch.int32).expand(2, 4))
    with pytest.raises(kvc.KvcError):
        kvc._heads(torch.zeros(2, 2, 64), 64, "q")
    with pytest.raises(kvc.KvcError):
        kvc._heads(bf(2, 2, 64), 128, "q")
    with pytest.raises(kvc.KvcError):
        kvc._heads(bf(1, 2, 64).expand(3, 2, 64), 64, "q")      # a broadcast row
    with pytest.raises(kvc.KvcError):
        kvc._heads(bf(3, 2, 128)[..., ::2], 64, "q")
    with pytest.raises(kvc.KvcError):                       # tensors that are not on the current CUDA device
        kvc.kvc_append(kvc.Requests(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 8), bf(1, 3, 64), bf(1, 3, 64),
                       kvc.Cache(bf(2, 3, 8, 64), bf(2, 3, 8, 64)), 0)
    q = kvc.QCache.like(kvc.Cache(bf(2, 3, 8, 64), bf(2, 3, 8, 64)))
    assert q.struct().codes.T == 8 and q.nbytes() == 2 * (2 * 3 * 8 * 64 + 2 * 3 * 8)


def test_descriptors_follow_the_objects():
    """A cache's tensors may be replaced between calls; a Requests refuses it (its checks ran when it was made)."""
    mk = lambda: torch.zeros(1, 3, 2, 16, 64, dtype=torch.bfloat16)
    c = kvc.Cache.pool(mk(), mk())
    held = lambda c, kind: kind.from_address(kvc._desc(c)[0])
    at = lambda: tuple(getattr(held(c, kvc.kvc_cache), f) for f in ("k", "v", "page_table", "T"))
    assert at() == (c.k.data_ptr(), c.v.data_ptr(), c.page_table.data_ptr() or None, 0)
    c.v, c.page_table, c.T = mk(), torch.zeros(2, dtype=torch.int32), 32
    assert at() == (c.k.data_ptr(), c.v.data_ptr(), c.page_table.data_ptr(), 32)
    q = kvc.QCache.like(c)
    kvc._desc(q)
    q.k, q.scale_v = torch.zeros_like(q.k), torch.zeros_like(q.scale_v)
    s = held(q, kvc.kvc_qcache)
    assert (s.codes.k, s.codes.v, s.scale_k, s.scale_v) == tuple(t.data_ptr() for t in (q.k, q.v, q.scale_k, q.scale_v))
    r = kvc.Requests(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 16)
    with pytest.raises(AttributeError):
        r.kv_len = torch.ones(1, dtype=torch.int32)
    two = copy.deepcopy((c, q, r))                # after calls too: descriptors hold pointers and are not copied
    assert two[0].T == 32 and two[2].max_kv == 16 and two[2].kv_len.data_ptr() != r.kv_len.data_ptr()
    assert held(two[0], kvc.kvc_cache).k == two[0].k.data_ptr() and held(c, kvc.kvc_cache).k == c.k.data_ptr()
    assert two[2].struct().kv_len == two[2].kv_len.data_ptr()
