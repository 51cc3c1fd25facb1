"""Overlapping buffers are refused before anything is launched: exponents of 8-bit caches, scratch, request lists.
(Addresses here are never touched: every call is refused.)"""
import ctypes as C

import pytest

import paper_2609_34060_b200 as kvc
from paper_2609_34060_b200 import build as kbuild

K, V, SK, SV, Q, O, LISTS, LSE, WS = (0x10000000 * i for i in range(1, 10))
ALIAS = kvc.KVC_E_ALIAS


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return kvc.load()


def q8(paged=False, **kw):
    q = kvc.kvc_qcache()
    c = q.codes
    c.k, c.v, c.L, c.H, c.T, c.d = K, V, 2, 2, 0 if paged else 32, 128
    if paged:
        c.layout, c.page_size, c.n_phys_pages = kvc.KVC_PAGED, 16, 8
    q.scale_k, q.scale_v = SK, SV
    for a, b in kw.items():
        setattr(q if a.startswith(("scale", "e_")) else c, a, b)
    return q


def bf(k=Q, v=O):
    c = kvc.kvc_cache()
    c.k, c.v, c.L, c.H, c.T, c.d = k, v, 2, 2, 32, 128
    return c


def heads(p, rows=4, n=2):
    return kvc.kvc_heads(p, rows, n, 0, 0)


def req(max_kv=64, **kw):
    r = kvc.kvc_requests(2, 1, max_kv, 4, LISTS, LISTS + 64, LISTS + 4096)
    for a, b in kw.items():
        setattr(r, a, b)
    return r


ROWS = 2 * 2 * 32                        # bytes of exponents, and rows of codes of 128 bytes


@pytest.mark.parametrize("kw", [dict(scale_v=SK), dict(scale_v=SK + ROWS - 1), dict(scale_k=K), dict(scale_k=V + 5), dict(scale_v=K + ROWS * 128 - 1),
                                dict(scale_v=SK + 1, e_tok=1), dict(scale_v=SK + 2, e_tok=2, e_head=64, e_layer=128),
                                dict(s_tok=144, e_tok=144, s_head=144 * 32, e_head=144 * 32, s_layer=288 * 32, e_layer=288 * 32, scale_k=K + 127),
                                dict(s_tok=144, e_tok=144, s_head=144 * 32, e_head=144 * 32, s_layer=288 * 32, e_layer=288 * 32, scale_k=K + 144)])
def test_exponents_over_one_another_or_the_codes(lib, kw):
    q = q8(**kw)
    assert lib.kvc_quantize(C.byref(bf()), C.byref(q), None) == ALIAS
    r = kvc.kvc_requests(1, 1, 32, 0, LISTS, LISTS + 64, 0)
    assert lib.kvc_append_q8(C.byref(r), C.byref(heads(Q)), C.byref(heads(O)), 0, C.byref(q), None) == ALIAS


def test_exponents_over_what_is_converted_or_appended(lib):
    for kw in (dict(scale_k=Q), dict(scale_k=O + 8), dict(scale_v=Q + 2 * ROWS * 128 - 1), dict(scale_v=O)):
        assert lib.kvc_quantize(C.byref(bf()), C.byref(q8(**kw)), None) == ALIAS
        assert lib.kvc_dequantize(C.byref(q8(**kw)), C.byref(bf()), None) == ALIAS
    for kw in (dict(scale_k=Q), dict(scale_v=O), dict(scale_v=Q + 4 * 2 * 256 - 1)):
        assert lib.kvc_append_q8(C.byref(req()), C.byref(heads(Q)), C.byref(heads(O)), 0, C.byref(q8(paged=True, **kw)), None) == ALIAS


def test_attention_writes_over_what_it_reads(lib):
    def at(out=O, lse=LSE, c=None, r=None):
        return lib.kvc_attend_q8(C.byref(r or req()), C.byref(heads(Q)), C.byref(c or q8(paged=True)), 0, 0.1, 1, C.byref(heads(out)), lse, WS, 1 << 40, None)
    page_rows = 2 * 8 * 2 * 16
    for p in (SK, SV + 16, SK + page_rows - 16, LISTS, LISTS + 4096):
        assert at(out=p) == ALIAS
    for p in (SK, SV + 4, LISTS + 8, LISTS + 64, LISTS + 4096 + 28):
        assert at(lse=p) == ALIAS
    plain = kvc.kvc_cache.from_buffer_copy(q8(paged=True).codes)
    attend = lambda r, out: lib.kvc_attend(C.byref(r), C.byref(heads(Q)), C.byref(plain), 0, 0.1, 1, C.byref(heads(out)), 0, WS, 1 << 40, None)
    assert attend(req(), LISTS) == ALIAS
    plain.T, plain.page_table = 64, LISTS + 8192                  # the cache's own table
    assert attend(req(page_table=0), LISTS + 8192) == ALIAS
