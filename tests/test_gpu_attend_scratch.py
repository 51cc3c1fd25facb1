"""Scratch of kvc_attend: too small, off its alignment or over other buffers is refused; exponents between one another or
behind their rows are served."""
import ctypes as C

import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 50])
def test_scratch_is_checked(nq, q8):
    b = Built(Step([nq, nq], [300, 200], q8=q8))
    need = kvc.kvc_attend_workspace_bytes(b.req, b.cache, 8)
    assert need > 0
    out, big = torch.full_like(b.q, 7.0), torch.empty(need + 512, dtype=torch.uint8, device="cuda")

    def code(ws, **kw):
        with pytest.raises(kvc.KvcError) as e:
            kvc.kvc_attend(b.req, b.q, b.cache, 0, kw.pop("out", out), ws, **kw)
        return e.value.code
    assert code(None) == kvc.KVC_E_WORKSPACE
    assert code(big[: need - 1]) == kvc.KVC_E_WORKSPACE
    assert code(big[16: need + 16]) == kvc.KVC_E_WORKSPACE
    n = b.q.numel() * 2
    arena = torch.empty(n + need + 1024, dtype=torch.uint8, device="cuda")
    inside = arena[:n].view(torch.bfloat16).view(b.q.shape)
    assert code(arena, out=inside) == kvc.KVC_E_ALIAS
    lse = arena[: b.q.shape[0] * 8 * 4].view(torch.float32).view(b.q.shape[:2])
    assert code(arena, lse=lse) == kvc.KVC_E_ALIAS
    inside.copy_(b.q)
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_attend(b.req, inside, b.cache, 0, out, arena)
    assert e.value.code == kvc.KVC_E_ALIAS
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    kvc.kvc_attend(b.req, b.q, b.cache, 0, out, big[:need])
    want, _ = b.run()
    assert torch.equal(out, want)


@pytest.mark.parametrize("layout", ["side_by_side", "behind_the_row"])
@pytest.mark.parametrize("nq", [1, 60])
def test_exponents_among_other_bytes(layout, nq):
    """Exponents of keys and values side by side, or each behind its row of codes: quantised and attended as dense ones."""
    L, H, T, d = 2, 2, 300, 128
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    src = kvc.Cache(rnd(L, H, T, d), rnd(L, H, T, d))
    dense = kvc.QCache.like(src)
    kvc.kvc_quantize(src, dense)
    s = dense.struct()
    if layout == "side_by_side":
        hold = torch.zeros(L, H, T, 2, dtype=torch.uint8, device="cuda")
        codes = [torch.zeros(L, H, T, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
        s.codes.k, s.codes.v = (x.data_ptr() for x in codes)
        s.scale_k, s.scale_v = hold.data_ptr(), hold.data_ptr() + 1
        s.e_tok, s.e_head, s.e_layer = 2, 2 * T, 2 * H * T
        get = lambda: (codes[0], codes[1], hold[..., 0], hold[..., 1])
    else:
        hold = [torch.zeros(L, H, T, d + 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
        s.codes.k, s.codes.v = (x.data_ptr() for x in hold)
        s.scale_k, s.scale_v = (x.data_ptr() + d for x in hold)
        s.codes.s_tok = s.e_tok = d + 16
        s.codes.s_head = s.e_head = T * (d + 16)
        s.codes.s_layer = s.e_layer = H * T * (d + 16)
        get = lambda: (hold[0][..., :d], hold[1][..., :d], hold[0][..., d], hold[1][..., d])
    lib, st = kvc.load(), torch.cuda.current_stream().cuda_stream
    assert lib.kvc_quantize(C.byref(src.struct()), C.byref(s), st) == 0
    for a, b in zip(get(), (dense.k.view(torch.uint8), dense.v.view(torch.uint8), dense.scale_k, dense.scale_v)):
        assert torch.equal(a, b)
    req = kvc.Requests(torch.tensor([0, nq], dtype=torch.int32, device="cuda"), torch.tensor([T], dtype=torch.int32, device="cuda"), nq, T)
    q = rnd(nq, H * 4, d)
    want, got = torch.zeros_like(q), torch.zeros_like(q)
    ws = torch.empty(kvc.kvc_attend_workspace_bytes(req, dense, H * 4), dtype=torch.uint8, device="cuda")
    kvc.kvc_attend(req, q, dense, 1, want, ws)
    rows = lambda t: kvc.kvc_heads(t.data_ptr(), nq, H * 4, 0, 0)
    assert lib.kvc_attend_q8(C.byref(req.struct()), C.byref(rows(q)), C.byref(s), 1, d ** -0.5, 1, C.byref(rows(got)), None, ws.data_ptr(), ws.numel(), st) == 0
    torch.cuda.synchronize()
    assert torch.equal(got, want)
