"""Tensors that are shorter than their descriptor says are refused before the library sees them.  (A stand-in takes the place
of the library.)"""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from test_binding_classes import fake  # noqa: F401  (fixture)


def bf(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def table(n):
    return torch.zeros(n, dtype=torch.int32)


def refused(call, code):
    with pytest.raises(kvc.KvcError) as e:
        call()
    assert e.value.code == code


def test_page_tables_shorter_than_the_cache(fake):  # noqa: F811
    short = kvc.Cache(bf(1, 4, 2, 16, 64), bf(1, 4, 2, 16, 64), T=49, page_table=table(3))
    dst = kvc.QCache.like(kvc.Cache(bf(1, 2, 49, 64), bf(1, 2, 49, 64)))
    q8 = kvc.QCache.like(short)
    req = kvc.Requests(table(2), table(1), 1, 49)
    q = bf(1, 4, 64)
    refused(lambda: kvc.kvc_quantize(short, dst), kvc.KVC_E_SHAPE)
    refused(lambda: kvc.kvc_dequantize(q8, kvc.Cache(bf(1, 2, 49, 64), bf(1, 2, 49, 64))), kvc.KVC_E_SHAPE)
    refused(lambda: kvc.kvc_append(req, bf(1, 2, 64), bf(1, 2, 64), q8, 0), kvc.KVC_E_SHAPE)
    refused(lambda: kvc.kvc_attend(req, q, short, 0, q.clone()), kvc.KVC_E_SHAPE)
    refused(lambda: kvc.kvc_attend(req, q, q8, 0, q.clone()), kvc.KVC_E_SHAPE)
    assert fake.calls == []
    short.T = 48
    kvc.kvc_attend(req, q, short, 0, q.clone())
    assert fake.calls == ["kvc_attend"]


def test_attributes_that_no_longer_fit(fake):  # noqa: F811
    c = kvc.Cache(bf(1, 2, 32, 64), bf(1, 2, 32, 64))
    q8 = kvc.QCache.like(c)
    kvc.kvc_quantize(c, q8)
    fake.calls.clear()
    for name, t, code in (("scale_v", torch.zeros(1, 2, 31, dtype=torch.uint8), kvc.KVC_E_SHAPE), ("scale_k", torch.zeros(1, 2, 32, dtype=torch.int32), kvc.KVC_E_INVALID_ARG),
                          ("k", torch.zeros(1, 2, 31, 64, dtype=torch.float8_e4m3fn), kvc.KVC_E_SHAPE), ("v", bf(1, 2, 32, 64), kvc.KVC_E_INVALID_ARG)):
        keep = getattr(q8, name)
        setattr(q8, name, t)
        refused(lambda: kvc.kvc_quantize(c, q8), code)
        setattr(q8, name, keep)
    c.T = 33
    refused(lambda: kvc.kvc_quantize(c, q8), kvc.KVC_E_SHAPE)
    c.T = 32
    c.v = bf(1, 2, 64, 64)[:, :, ::2]
    refused(lambda: kvc.kvc_quantize(c, q8), kvc.KVC_E_INVALID_ARG)
    assert fake.calls == []


def test_scratch_that_is_a_view_of_less(fake):  # noqa: F811
    c = kvc.Cache(bf(1, 2, 32, 64), bf(1, 2, 32, 64))
    req, q = kvc.Requests(table(2), table(1), 1, 32), bf(1, 4, 64)
    ws = torch.zeros(1, dtype=torch.uint8).expand(1 << 20)         # one byte of memory
    refused(lambda: kvc.kvc_attend(req, q, c, 0, q.clone(), ws), kvc.KVC_E_INVALID_ARG)
    assert fake.calls == []
