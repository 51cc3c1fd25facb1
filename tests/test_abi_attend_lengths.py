"""Lengths at the end of 32 bits (tables may name a page many times over): refused, not wrapped around.  Nothing is launched:
the addresses are never touched."""
import ctypes as C

import pytest

import paper_2609_34060_b200 as kvc
from paper_2609_34060_b200 import build as kbuild

LONGEST = 2 ** 31 - 257


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return kvc.load()


def pool(T=0):
    c = kvc.kvc_cache()
    c.k, c.v, c.L, c.H, c.T, c.d, c.layout, c.page_size, c.n_phys_pages, c.page_table = 1 << 28, 2 << 28, 1, 2, T, 128, kvc.KVC_PAGED, 16, 64, 3 << 28
    return c


def heads(p):
    return kvc.kvc_heads(p, 4, 2, 0, 0)


@pytest.mark.parametrize("kv", [LONGEST + 1, 2 ** 31 - 100, 2 ** 31 - 1])
def test_lengths_that_would_wrap(lib, kv):
    r = kvc.kvc_requests(1, 1, kv, 1 << 27, 4 << 28, (4 << 28) + 64, 5 << 28)
    assert lib.kvc_attend(C.byref(r), C.byref(heads(6 << 28)), C.byref(pool()), 0, 0.1, 1, C.byref(heads(7 << 28)), None, 8 << 28, 0, None) == kvc.KVC_E_UNSUPPORTED
    assert lib.kvc_append(C.byref(r), C.byref(heads(6 << 28)), C.byref(heads(7 << 28)), 0, C.byref(pool()), None) == kvc.KVC_E_UNSUPPORTED
    assert lib.kvc_attend_workspace_bytes(C.byref(r), 2, 2, 128) == 0
    q = kvc.kvc_qcache()
    q.codes = pool(kv)
    q.codes.k, q.codes.v, q.scale_k, q.scale_v = 9 << 28, 10 << 28, 11 << 28, 12 << 28
    assert lib.kvc_quantize(C.byref(pool(kv)), C.byref(q), None) == kvc.KVC_E_UNSUPPORTED
    assert lib.kvc_dequantize(C.byref(q), C.byref(pool(kv)), None) == kvc.KVC_E_UNSUPPORTED
