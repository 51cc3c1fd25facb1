"""Calls with many requests, with bounds far above the lengths, over pools whose keys and values share one buffer, and over
contexts shorter than a tile."""
import ctypes as C
import random

import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("kind", ["tokens", "drafts", "mixed", "mostly_empty"])
def test_hundreds_of_requests(kind, q8):
    r = random.Random(kind)
    n = 333
    nq = {"tokens": [1] * n, "drafts": [r.randint(0, 4) for _ in range(n)], "mixed": [r.choice([1, 1, 1, 0, 20]) for _ in range(n)],
          "mostly_empty": [1 if i % 37 == 5 else 0 for i in range(n)]}[kind]
    kv = [max(q, r.choice([0, 1, r.randint(1, 90), r.randint(100, 400)])) for q in nq]
    b = Built(Step(nq, kv, H=2, G=2, d=64, q8=q8, spare=3, seed=7))
    kvc.kvc_status_reset()
    b.check(*b.run())
    assert kvc.kvc_status_poll() == 0


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("max_q", [1, 8, 64])
def test_bounds_far_above_the_lengths(max_q, q8):
    """A list captured for the longest step: short requests under bounds of many tiles and rows."""
    b = Built(Step([1, 1, 0, 1], [5, 130, 0, 257], H=2, G=4, q8=q8, seed=3))
    tab = torch.full((4, 700), -7, dtype=torch.int32, device="cuda")
    tab[:, : b.req.page_table.shape[1]] = b.req.page_table
    b.req = kvc.Requests(b.req.q_begin, b.req.kv_len, max_q, 700 * 16, page_table=tab)
    kvc.kvc_status_reset()
    b.check(*b.run())
    assert kvc.kvc_status_poll() == 0


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("T", [40, 41, 127, 128])
def test_contiguous_contexts_shorter_than_a_tile(T, nq, q8):
    if nq > T:
        pytest.skip("nothing new")
    b = Built(Step([nq], [T - 2], page=0, H=2, G=2, q8=q8, seed=T))      # the rows hold two tokens more than the length
    b.check(*b.run())


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 40])
@pytest.mark.parametrize("order", ["kv_in_a_page", "kv_in_a_row"])
def test_keys_and_values_in_one_buffer(order, nq, q8):
    """Pools [pages, K | V, heads, tokens, d] and [pages, tokens, heads, K | V, d], described through the strides: the bits of
    separate pools."""
    b = Built(Step([nq, nq], [300, 170], H=2, G=4, q8=q8, seed=11))
    want, wlse = b.run()
    c = b.cache
    byte = lambda t: t.view(torch.uint8) if q8 else t
    k, v = byte(c.k)[0], byte(c.v)[0]                              # [P, H, page, d]
    P, H, page, d = k.shape
    s = kvc.kvc_qcache() if q8 else kvc.kvc_cache()
    geo = s.codes if q8 else s
    if order == "kv_in_a_page":
        hold = torch.stack([k, v], 1).contiguous()                 # [P, 2, H, page, d]
        step, geo.s_tok, geo.s_head, geo.s_page = H * page * d, d, page * d, 2 * H * page * d
    else:
        hold = torch.stack([k.transpose(1, 2), v.transpose(1, 2)], 3).contiguous()      # [P, page, H, 2, d]
        step, geo.s_tok, geo.s_head, geo.s_page = d, H * 2 * d, 2 * d, page * H * 2 * d
    geo.s_layer = P * geo.s_page
    geo.k, geo.v = hold.data_ptr(), hold.data_ptr() + step * hold.element_size()
    geo.L, geo.H, geo.T, geo.d, geo.layout, geo.page_size, geo.n_phys_pages = 1, H, 0, d, kvc.KVC_PAGED, page, P
    if q8:
        s.scale_k, s.scale_v = c.scale_k.data_ptr(), c.scale_v.data_ptr()
    out, lse, ws = torch.zeros_like(b.q), torch.zeros_like(wlse), b.workspace()
    rows = lambda t: kvc.kvc_heads(t.data_ptr(), t.shape[0], t.shape[1], 0, 0)
    lib = kvc.load()
    fn = lib.kvc_attend_q8 if q8 else lib.kvc_attend
    st = torch.cuda.current_stream().cuda_stream
    assert fn(C.byref(b.req.struct()), C.byref(rows(b.q)), C.byref(s), 0, b.scale, 1, C.byref(rows(out)), lse.data_ptr(), ws.data_ptr(), ws.numel(), st) == 0
    torch.cuda.synchronize()
    assert kvc.kvc_last_path() == kvc.KVC_PATH_TC
    assert torch.equal(out, want) and torch.equal(lse, wlse)
