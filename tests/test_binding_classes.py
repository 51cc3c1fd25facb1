"""The calls of a serving step hand descriptors over as addresses: the binding has to see that each is of the right class.
(A stand-in takes the place of the library: nothing is launched, nothing is read through the addresses.)"""
import pytest
import torch

import paper_2609_34060_b200 as kvc


class FakeLibrary:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name == "kvc_strerror":
            return lambda code: b"refused"
        return lambda *a: self.calls.append(name) or 0


@pytest.fixture
def fake(monkeypatch):
    lib = FakeLibrary()
    monkeypatch.setattr(kvc, "load", lambda *a: lib)
    monkeypatch.setattr(kvc, "_here", lambda what, stream, made, *tensors: 0)
    return lib


def objects():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    c = kvc.Cache(z(1, 2, 16, 64), z(1, 2, 16, 64))
    req = kvc.Requests(torch.tensor([0, 1], dtype=torch.int32), torch.ones(1, dtype=torch.int32), 1, 16)
    return c, kvc.QCache.like(c), req, z(1, 2, 64), z(1, 4, 64)


def test_swapped_caches_are_refused(fake):
    c, q8, req, kn, q = objects()
    state = object()
    wrong = [lambda: kvc.kvc_quantize(q8, c), lambda: kvc.kvc_dequantize(c, q8), lambda: kvc.kvc_quantize(c, c), lambda: kvc.kvc_dequantize(q8, q8),
             lambda: kvc.kvc_quantize(q8, q8), lambda: kvc.kvc_dequantize(c, c), lambda: kvc.kvc_quantize(c, None), lambda: kvc.kvc_quantize(c.struct(), q8),
             lambda: kvc.kvc_append(req, kn, kn, state, 0), lambda: kvc.kvc_append(req, kn, kn, c.struct(), 0), lambda: kvc.kvc_attend(req, q, None, 0, q.clone()),
             lambda: kvc.kvc_append(c, kn, kn, req, 0), lambda: kvc.kvc_attend(c, q, q8, 0, q.clone()), lambda: kvc.kvc_attend(req, c, q, 0, q.clone()),
             lambda: kvc.kvc_attend_workspace_bytes(c, c, 4)]
    for call in wrong:
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.code == kvc.KVC_E_INVALID_ARG
    assert fake.calls == []


def test_the_right_classes_reach_the_library(fake):
    c, q8, req, kn, q = objects()
    kvc.kvc_quantize(c, q8)
    kvc.kvc_dequantize(q8, c)
    kvc.kvc_append(req, kn, kn, c, 0)
    kvc.kvc_append(req, kn, kn, q8, 0)
    kvc.kvc_attend(req, q, c, 0, q.clone())
    kvc.kvc_attend(req, q, q8, 0, q.clone())
    assert fake.calls == ["kvc_quantize", "kvc_dequantize", "kvc_append", "kvc_append_q8", "kvc_attend", "kvc_attend_q8"]


def test_subclasses_are_what_they_derive_from(fake):
    class MyQ(kvc.QCache):
        pass

    class MyC(kvc.Cache):
        pass

    c, q8, req, kn, q = objects()
    mq, mc = MyQ(q8.k, q8.v, q8.scale_k, q8.scale_v), MyC(c.k, c.v)
    kvc.kvc_append(req, kn, kn, mq, 0)
    kvc.kvc_attend(req, q, mq, 0, q.clone())
    kvc.kvc_attend(req, q, mc, 0, q.clone())
    kvc.kvc_quantize(mc, mq)
    assert fake.calls == ["kvc_append_q8", "kvc_attend_q8", "kvc_attend", "kvc_quantize"]
    held = kvc.kvc_qcache.from_address(kvc._desc(mq)[0])
    assert (held.codes.k, held.scale_k, held.scale_v) == (mq.k.data_ptr(), mq.scale_k.data_ptr(), mq.scale_v.data_ptr())
