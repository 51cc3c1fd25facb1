"""What the binding checks before it hands addresses on: classes, types, shapes, strides.  (A stand-in for the library.)"""
import copy
import pickle
import struct

import pytest
import torch

import paper_2609_34060_b200 as kvc
from test_binding_classes import FakeLibrary

I32 = torch.int32


@pytest.fixture
def fake(monkeypatch):
    lib = FakeLibrary()
    monkeypatch.setattr(kvc, "load", lambda *a: lib)
    monkeypatch.setattr(kvc, "_here", lambda what, stream, made, *tensors: 0)
    return lib


def z(*s, dtype=torch.bfloat16):
    return torch.zeros(*s, dtype=dtype)


def objects():
    c = kvc.Cache(z(1, 2, 16, 64), z(1, 2, 16, 64))
    req = kvc.Requests(torch.tensor([0, 3], dtype=I32), torch.full((1,), 9, dtype=I32), 3, 16)
    return c, kvc.QCache.like(c), req, kvc.Tree(z(3, dtype=I32), 3), kvc.Rotary(kvc.Rope(1e4))


def refused(code, *calls):
    for i, f in enumerate(calls):
        with pytest.raises(kvc.KvcError) as e:
            f()
        assert e.value.code == code, i


def test_blocks():
    """Argument blocks: what lies where, and what is no argument."""
    q, p, k = z(3, 4, 64), torch.zeros(5, 9), z(2, 6, dtype=I32)
    pack = lambda codes, names, *args: kvc._pack(codes, names, -1, 64, 2, 5, *args)
    b = pack("PHpnKii", ("q", "p", "n", "k"), 7, q[:, 1:3], p[1:3, :6], None, k, -2, 3)
    assert b == struct.pack("@QQiiQQQiiQQQQii", 7, q.data_ptr() + 128, 3, 2, 256, 64, p.data_ptr() + 36, 2, 6, 9, 0, k.data_ptr(), 6, -2, 3)
    assert len(pack("Hp", ("q", "p"), z(1, 1, 64), torch.zeros(1, 1))) == 32 + 24
    c, q8, *_ = objects()
    for x in (c, q8):
        made = kvc._desc(x)
        for name in ("k", "v") + (("scale_k", "scale_v") if x is q8 else ()):
            x.__dict__[name] = getattr(x, name).clone()                 # tensors that moved: the descriptor follows
        assert pack("C", ("c",), x) == struct.pack("@QQ", made[0], x is q8) and made[2].k == x.k.data_ptr() and made[2].v == x.v.data_ptr()
        assert x is c or (made[3].scale_k, made[3].scale_v) == (x.scale_k.data_ptr(), x.scale_v.data_ptr())
    with pytest.raises(OverflowError):
        pack("i", (), 1 << 31)
    with pytest.raises(TypeError):
        pack("PP", (), 1)
    refused(-1, lambda: kvc._pack("H", ("q",), 0, 64, 0, 0, q), lambda: pack("H", ("q",), object()), lambda: pack("A", (), q[:, ::2]), lambda: pack("F", (), z(3)),
            lambda: pack("C", ("c",), q), lambda: pack("K", ("k",), None), lambda: pack("u", ("u",), None))
    refused(-2, lambda: pack("n", ("n",), z(3, dtype=I32)), lambda: pack("K", ("k",), z(2, 4, dtype=I32)), lambda: pack("pr", ("p", "r"), p, z(4, dtype=I32)))


def test_tree(fake):
    refused(-1, lambda: kvc.Tree([0, 1], 3), lambda: kvc.Tree(z(3, dtype=torch.int64), 3), lambda: kvc.Tree(z(6, dtype=I32)[::2], 3),
            lambda: kvc.Tree(z(3, dtype=I32), 3, mask=z(3, 1, dtype=torch.uint8)))
    refused(-2, lambda: kvc.Tree(z(3, dtype=I32), 33, mask=z(3, 1, dtype=I32)), lambda: kvc.Tree(z(3, dtype=I32), 3, depth=z(4, dtype=I32)),
            lambda: kvc.Tree(z(3, 1, dtype=I32), 3), lambda: kvc.Tree(z(3, dtype=I32), 3, mask=z(4, 1, dtype=I32)))
    t = kvc.Tree(z(3, dtype=I32), 70)
    assert t.mask.shape == (3, 3) and t.struct().words == 3 and t.struct().n_rows == 3
    with pytest.raises(AttributeError):
        t.mask = None
    assert copy.deepcopy(t).struct().mask != t.struct().mask and pickle.loads(pickle.dumps(t)).max_q == 70
    c, q8, req, tree, rot = objects()
    refused(-1, lambda: kvc.kvc_tree_build(tree, req), lambda: kvc.kvc_tree_build(req, req), lambda: kvc.kvc_tree_build(req, tree.struct()))
    assert fake.calls == []


def test_rotary():
    refused(-1, lambda: kvc.Rotary(1e4), lambda: kvc.Rotary(kvc.Rope(1e4), amplitude=0.0), lambda: kvc.Rotary(kvc.Rope(1e4), depth=z(3, dtype=torch.int64)))
    r = kvc.Rotary(kvc.Rope(1e4, inv_freq=[1.0] * 16))
    refused(-2, lambda: r._for(64))
    kvc.Rotary(kvc.Rope(1e4, inv_freq=[1.0] * 16), rot_dim=32)._for(64)
    assert copy.deepcopy(kvc.Rotary(kvc.Rope(1e4), rot_dim=32, amplitude=1.5)).struct().amplitude == 1.5
    with pytest.raises(AttributeError):
        r.depth = None


def test_lists_of_positions_that_are_too_short(monkeypatch):
    """The library itself: refused before it looks at a device."""
    monkeypatch.setattr(kvc, "_here", lambda what, stream, made, *tensors: 0)
    c, q8, req, tree, _ = objects()
    k = z(3, 2, 64)
    for cache in (c, q8):
        for rot in (kvc.Rotary(kvc.Rope(1e4), depth=z(2, dtype=I32)), kvc.Rotary(kvc.Rope(1e4), pos_begin=z(0, dtype=I32))):
            refused(-2, lambda: kvc.kvc_append_rotated(req, rot, k, k.clone(), cache, 0))


def test_scaled_frequencies():
    f = kvc.scaled_frequencies(1e4, 64)
    assert f[0] == 1.0 and abs(f[16] - 1e-2) < 1e-15
    assert kvc.scaled_frequencies(1e4, 64, 8.0) == [x / 8.0 for x in f]
    parts = kvc.scaled_frequencies(1e4, 64, 8.0, original=8192)
    turns = [8192 * x / 6.283185307179586 for x in f]
    for a, b, t in zip(parts, f, turns):
        assert (a == b) if t >= 32 else abs(a - b / 8) < 1e-18 if t <= 1 else b / 8 < a < b


def test_append_rotated(fake):
    c, q8, req, tree, rot = objects()
    k, q = z(3, 2, 64), z(3, 4, 64)
    kvc.kvc_append_rotated(req, rot, k, k, c, 0, q=q, q_out=q)
    kvc.kvc_append_rotated(req, rot, k, k, q8, 0)
    assert fake.calls == ["kvc_block_append_rotated"] * 2
    refused(-1, lambda: kvc.kvc_append_rotated(req, kvc.Rope(1e4), k, k, c, 0), lambda: kvc.kvc_append_rotated(rot, req, k, k, c, 0),
            lambda: kvc.kvc_append_rotated(req, rot, k, k, c, 0, q=q), lambda: kvc.kvc_append_rotated(req, rot, k, k, c, 0, q_out=q),
            lambda: kvc.kvc_append_rotated(req, rot, k.float(), k, c, 0), lambda: kvc.kvc_append_rotated(req, rot, k, k, k, 0))
    refused(-2, lambda: kvc.kvc_append_rotated(req, rot, z(3, 2, 128), k, c, 0))
    refused(-3, lambda: kvc.kvc_append_rotated(req, rot, k, z(1, 2, 64).expand(3, 2, 64), c, 0))
    assert len(fake.calls) == 2


def test_attend_tree(fake):
    c, q8, req, tree, rot = objects()
    q = z(3, 4, 64)
    kvc.kvc_attend_tree(req, tree, q, c, 0, q.clone())
    kvc.kvc_attend_tree(req, tree, q, q8, 0, q.clone(), lse=z(3, 4, dtype=torch.float32))
    assert fake.calls == ["kvc_block_attend_tree"] * 2
    refused(-1, lambda: kvc.kvc_attend_tree(req, None, q, c, 0, q.clone()), lambda: kvc.kvc_attend_tree(tree, req, q, c, 0, q.clone()),
            lambda: kvc.kvc_attend_tree(req, tree, q, tree, 0, q.clone()), lambda: kvc.kvc_attend_tree(req, tree, q, c, 0, q.clone(), lse=z(3, 4)),
            lambda: kvc.kvc_attend_tree(req, tree, q, c, 0, q.clone(), workspace=z(8, 8)[:, ::2]))


def test_verify(fake):
    c, q8, req, tree, rot = objects()
    i = lambda *s: z(*s, dtype=I32)
    f = lambda *s: z(*s, dtype=torch.float32)
    good = dict(parent=i(3), token=i(3), target=f(3, 10), u=f(3), u_next=f(1), kept=i(1, 3), n_kept=i(1), next_token=i(1))
    call = lambda **kw: kvc.kvc_verify(req, **{**good, **kw})
    call()
    call(draft=f(3, 16)[:, :10], kept=i(1, 7))
    assert fake.calls == ["kvc_block_verify"] * 2
    refused(-1, lambda: call(target=z(3, 10)), lambda: call(draft=f(3, 10).double()), lambda: call(parent=f(3)), lambda: call(u=f(3).double()),
            lambda: call(token=i(6)[::2]), lambda: call(kept=f(1, 3)), lambda: kvc.kvc_verify(tree, **good), lambda: call(n_kept=f(1)), lambda: call(u_next=i(1)))
    refused(-2, lambda: call(parent=i(4)), lambda: call(token=i(2)), lambda: call(u=f(4)), lambda: call(kept=i(1, 2)), lambda: call(kept=i(2, 3)),
            lambda: call(n_kept=i(2)), lambda: call(next_token=i(2)), lambda: call(u_next=f(3)))
    refused(-3, lambda: call(target=f(3, 20)[:, ::2]), lambda: call(draft=f(1, 10).expand(3, 10)))
    assert len(fake.calls) == 2


def test_keep(fake):
    c, q8, req, tree, rot = objects()
    i = lambda *s: z(*s, dtype=I32)
    kvc.kvc_keep(req, i(1, 3), i(1), c, i(1))
    kvc.kvc_keep(req, i(1, 5), i(1), q8)
    assert fake.calls == ["kvc_block_keep"] * 2
    refused(-1, lambda: kvc.kvc_keep(req, i(1, 3).long(), i(1), c), lambda: kvc.kvc_keep(req, i(1, 3), i(1).long(), c), lambda: kvc.kvc_keep(req, i(1, 3), i(1), req),
            lambda: kvc.kvc_keep(c, i(1, 3), i(1), c), lambda: kvc.kvc_keep(req, i(1, 6)[:, ::2], i(1), c))
    refused(-2, lambda: kvc.kvc_keep(req, i(1, 2), i(1), c), lambda: kvc.kvc_keep(req, i(2, 3), i(1), c), lambda: kvc.kvc_keep(req, i(1, 3), i(2), c),
            lambda: kvc.kvc_keep(req, i(1, 3), i(1), c, i(2)))
