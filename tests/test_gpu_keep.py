"""kvc_keep: accepted rows moved together, bit for bit; everything else left."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from draft_helpers import I32, requests, shuffled_table

pytestmark = pytest.mark.gpu


def make(kv, H, d, page, L, q8, tm, seed, strided=False):
    g = torch.Generator().manual_seed(seed)
    if page:
        table, P = shuffled_table(kv, page, seed)
        shape = (L, P, page, H, d) if tm else (L, P, H, page, d)
    else:
        table, shape = None, (L, max(kv) + 2, H, d) if tm else (L, H, max(kv) + 2, d)
    if q8:
        code = [torch.randint(0, 256, shape, generator=g, dtype=torch.int32).to(torch.uint8).cuda().view(torch.float8_e4m3fn) for _ in range(2)]
        exp = [torch.randint(0, 256, shape[:-1], generator=g, dtype=torch.int32).to(torch.uint8).cuda() for _ in range(2)]
        c = kvc.QCache.pool(*code, *exp, token_major=tm) if page else kvc.QCache(*code, *exp, token_major=tm)
    else:
        x = [torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(2)]
        c = kvc.Cache.pool(*x, token_major=tm) if page else kvc.Cache(*x, token_major=tm)
    return c, table


def parts(c):
    names = ("k", "v") + (("scale_k", "scale_v") if isinstance(c, kvc.QCache) else ())
    return {n: (getattr(c, n).view(torch.uint8) if isinstance(c, kvc.QCache) else getattr(c, n)).cpu().clone() for n in names}


def at(c, table, b, t):
    if c.page_table is None:
        return (slice(None), t) if c.token_major else (slice(None), slice(None), t)
    p, s = int(table[b, t // c.page]), t % c.page
    return (slice(None), p, s) if c.token_major else (slice(None), p, slice(None), s)


def moved(c, table, was, nq, kv, lists):
    want = {n: x.clone() for n, x in was.items()}
    for b, keep in enumerate(lists):
        for j, a in enumerate(keep):
            for n in want:
                want[n][at(c, table, b, kv[b] - nq[b] + j)] = was[n][at(c, table, b, kv[b] - nq[b] + a)]
    return want


def run(c, table, nq, kv, lists, stride=None, out=True, **kw):
    max_q = max(nq)
    stride = max_q if stride is None else stride
    kept = torch.tensor([x + [-1] * (stride - len(x)) for x in lists], dtype=I32, device="cuda").view(len(nq), stride)
    n_kept = torch.tensor([len(x) for x in lists], dtype=I32, device="cuda")
    kv_out = torch.full((len(nq),), 55, dtype=I32, device="cuda") if out else None
    kvc.kvc_status_reset()
    kvc.kvc_keep(requests(nq, kv, table=table, **kw), kept, n_kept, c, kv_out)
    torch.cuda.synchronize()
    flags = kvc.kvc_status_poll()
    kvc.kvc_status_reset()
    return flags, kv_out


def ascending(m, k, rng):
    return sorted(rng.choice(m, size=k, replace=False).tolist())


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq,kv,H,d,page,L,tm", [
    ([1], [1], 1, 64, 8, 1, False), ([6, 0, 9], [40, 3, 9], 2, 128, 16, 3, False), ([24] * 7, [24, 30, 99, 128, 129, 500, 25], 4, 64, 32, 2, True),
    ([150, 90], [200, 90], 1, 128, 64, 2, False), ([33], [60], 3, 128, 0, 2, True), ([12], [12], 2, 64, 0, 1, False), ([1000], [1010], 1, 64, 16, 1, False)])
def test_rows_move(nq, kv, H, d, page, L, tm, q8):
    """Ascending lists of every length; neighbours overlap, so that a place is read before it is written."""
    for seed in range(3):
        rng = np.random.default_rng(seed)
        c, table = make(kv, H, d, page, L, q8, tm, seed)
        lists = [ascending(m, m if seed == 2 else int(rng.integers(0, m + 1)), rng) for m in nq]
        was = parts(c)
        flags, kv_out = run(c, table, nq, kv, lists, stride=max(nq) + seed)
        now, want = parts(c), moved(c, table, was, nq, kv, lists)
        assert flags == 0 and kv_out.tolist() == [t - m + len(x) for m, t, x in zip(nq, kv, lists)]
        for n in want:
            assert torch.equal(now[n].view(torch.int16 if now[n].dtype == torch.bfloat16 else torch.uint8), want[n].view(torch.int16 if want[n].dtype == torch.bfloat16 else torch.uint8)), n


def test_without_new_lengths():
    c, table = make([40], 2, 64, 16, 2, False, False, 1)
    was = parts(c)
    run(c, table, [10], [40], [[0, 4, 5, 9]], out=False)
    want = moved(c, table, was, [10], [40], [[0, 4, 5, 9]])
    assert torch.equal(parts(c)["k"], want["k"]) and torch.equal(parts(c)["v"], want["v"])


@pytest.mark.parametrize("bad", [[0, 3, 3], [0, 5, 2], [0, 1, 8], [-1, 2], [2, 0], [0, 1, 2, 3, 4, 5, 6, -4]])
def test_lists_that_are_not_ascending_move_nothing(bad):
    nq, kv = [8, 8], [20, 30]
    c, table = make(kv, 2, 64, 16, 2, False, False, 2)
    was = parts(c)
    flags, kv_out = run(c, table, nq, kv, [bad, [0, 2]])
    want = moved(c, table, was, nq, kv, [[], [0, 2]])
    assert flags == kvc.KVC_FLAG_BAD_TREE and kv_out.tolist() == [20, 24]
    assert torch.equal(parts(c)["k"], want["k"])


def test_counts_positions_pages_and_bounds():
    c, table = make([20, 30, 40], 2, 64, 16, 2, False, False, 3)
    table[1, 1] = 1 << 20                                               # rows 16 .. 29 of request 1
    was = parts(c)
    nq, kv = [8, 20, 8], [5, 30, 41]                                    # request 0 begins at -3, request 2 passes its bound
    flags, kv_out = run(c, table, nq, kv, [[0, 2], [0, 3, 9], [0, 2]], max_kv=40)
    assert flags == kvc.KVC_FLAG_BAD_TREE | kvc.KVC_FLAG_BAD_PAGE | kvc.KVC_FLAG_BAD_LENGTH
    assert kv_out.tolist() == [5, 13, 55]
    want = {n: x.clone() for n, x in was.items()}
    for n in want:
        want[n][at(c, table, 1, 11)] = was[n][at(c, table, 1, 13)]      # row 19 is on the page without a place
    assert torch.equal(parts(c)["k"], want["k"]) and torch.equal(parts(c)["v"], want["v"])
    kept, n_kept = torch.zeros(1, 8, dtype=I32, device="cuda"), torch.tensor([9], dtype=I32, device="cuda")
    kvc.kvc_keep(requests([8], [20], table=table[:1]), kept, n_kept, c)
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_TREE
    kvc.kvc_status_reset()
    assert torch.equal(parts(c)["k"], want["k"])
