"""kvc_attend against the float64 oracle: both kernel families, bf16 and 8-bit caches, every layout, the odd shapes."""
import random

import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu

CASES = {
    "one_key": Step([1], [1]),
    "token": Step([1], [777], H=2, G=4),
    "token_exact_tile": Step([1], [256]),
    "token_tile_plus_one": Step([1], [257]),
    "tokens_ragged": Step([1] * 9, [1, 16, 17, 127, 128, 129, 700, 33, 1024], spare=3),
    "tokens_no_keys": Step([1, 1, 1], [0, 5, 0], causal=False),
    "longer_than_cache": Step([6, 3], [4, 3]),
    "no_new_tokens": Step([0, 2, 0], [40, 33, 0]),
    "few_rows": Step([3, 1, 5], [300, 64, 131], G=8),
    "g1": Step([5, 130], [200, 400], H=3, G=1),
    "g7": Step([1, 40], [333, 500], G=7),
    "g16": Step([1, 9], [150, 260], H=1, G=16),
    "g64": Step([1, 3], [150, 260], H=1, G=64),
    "chunk": Step([300], [300], G=2),
    "chunk_behind_context": Step([200], [901], G=4, key_scale=3.0),
    "chunk_one_tile_rows": Step([32], [640], G=4),
    "mixed": Step([1, 150, 1, 7, 0, 64], [640, 150, 12, 700, 0, 65], G=4, spare=5),
    "cross": Step([70, 1], [333, 129], causal=False),
    "page8": Step([20, 1], [203, 77], page=8),
    "page32_token_major": Step([20, 1], [203, 77], page=32, token_major=True),
    "page64": Step([20, 1], [203, 77], page=64),
    "page256": Step([20, 1], [603, 277], page=256),
    "second_layer": Step([20, 1], [203, 77], L=3, layer=1),
    "contiguous": Step([33, 1], [300, 300], page=0),
    "contiguous_token_major": Step([33, 1], [300, 300], page=0, token_major=True, L=2, layer=1),
    "d64": Step([50, 1, 130], [300, 129, 131], d=64, G=3),
    "d64_contiguous": Step([5], [300], d=64, page=0),
    "d64_token_major": Step([1, 20], [301, 200], d=64, page=32, token_major=True),
    "peaked": Step([40, 1], [400, 300], key_scale=12.0),
    "flat": Step([40, 1], [400, 300], key_scale=0.0),
    "rising": Step([40, 1, 90], [900, 1000, 700], ramp=60.0),
    "rising_steeply": Step([1, 70], [700, 800], ramp=900.0, G=2),
    "falling": Step([40, 1, 90], [900, 1000, 700], ramp=-60.0),
    "few12": Step([3, 2], [300, 65]),
    "few24": Step([3, 1], [300, 131], G=8),
    "few32_d64": Step([4, 2, 1], [300, 131, 128], G=8, d=64),
    "few16_d64": Step([4, 2, 1], [300, 131, 128], G=4, d=64),
    "many_short": Step([1] * 70, [1 + 13 * (i % 17) for i in range(70)], H=3, G=2),
}


@pytest.mark.parametrize("path", ["generic", "auto"])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("name", sorted(CASES))
def test_attend_matches_the_oracle(name, q8, path):
    import dataclasses
    b = Built(dataclasses.replace(CASES[name], q8=q8))
    kvc.kvc_status_reset()
    kvc.kvc_set_path(kvc.KVC_PATH_GENERIC if path == "generic" else kvc.KVC_PATH_AUTO)
    try:
        out, lse = b.run()
        used = kvc.kvc_last_path()
    finally:
        kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
    b.check(out, lse)
    assert kvc.kvc_status_poll() == 0
    if path == "auto" and b.req.max_q > 0:
        assert used == kvc.KVC_PATH_TC, "these shapes belong to the tensor-core kernels"


@pytest.mark.parametrize("seed", range(24))
def test_attend_drawn(seed):
    r = random.Random(seed)
    n = r.randint(1, 6)
    few = r.random() < 0.4
    nq = [r.choice([0, 1, 1, r.randint(1, 4 if few else 150)]) for _ in range(n)]
    kv = [max(0, q + r.choice([-2, 0, r.randint(0, 500)])) if q else r.randint(0, 50) for q in nq]
    page = r.choice([0, 8, 16, 16, 32, 128])
    if page == 0:
        kv = [max(kv)] * n if max(kv) else [1] * n
    b = Built(Step(nq, kv, H=r.randint(1, 3), G=r.choice([1, 2, 3, 4, 5, 8]), d=r.choice([64, 128]), page=page,
                   token_major=r.random() < 0.4, q8=r.random() < 0.5, causal=r.random() < 0.7, spare=r.choice([0, 2]),
                   key_scale=r.choice([0.5, 1.0, 4.0]), seed=seed, L=r.choice([1, 2]), layer=0))
    kvc.kvc_status_reset()
    out, lse = b.run()
    b.check(out, lse)
    assert kvc.kvc_status_poll() == 0


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_strided_rows_and_other_stream(q8):
    """Queries and outputs as slices of a fused projection, on a stream of their own: bit-identical to dense ones."""
    b = Built(Step([3, 40], [300, 170], q8=q8))
    want, lse = b.run()
    rows, hq, d = b.q.shape
    fused = torch.randn(rows, hq + 6, d, device="cuda").to(torch.bfloat16)
    fused[:, 2:2 + hq] = b.q
    outs = torch.full((rows, hq + 3, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws, s = b.workspace(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        kvc.kvc_attend(b.req, fused[:, 2:2 + hq], b.cache, 0, outs[:, 1:1 + hq], ws)
    torch.cuda.synchronize()
    assert torch.equal(outs[:, 1:1 + hq], want)
    assert (outs[:, 0] == 7).all() and (outs[:, 1 + hq:] == 7).all()


@pytest.mark.parametrize("nq", [1, 60])
def test_replayed_graph_takes_new_lengths(nq):
    """Captured once, replayed with other lengths, pages and queries; each replay equals an eager call."""
    b = Built(Step([nq, nq, nq], [500, 420, 77 + nq], q8=False))
    ws = b.workspace()
    out, lse = torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")
    call = lambda: kvc.kvc_attend(b.req, b.q, b.cache, 0, out, ws, lse=lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for lens in ([500, 420, 77 + nq], [nq, 300, 64 + nq], [499, 1 + nq, 77]):
        b.st.kv[:] = lens
        b.req.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        b.val_k = [x[: n] for x, n in zip(b.val_k, lens)]
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = b.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [[1, 1, 1], [60, 1, 17]])
def test_requests_share_the_caches_own_table(nq, q8):
    """Several requests without a table of their own read one paged context, each as much of it as its length says."""
    lens = [200, 130, 64]
    big = Built(Step([0], [200], q8=q8))
    c, tab = big.cache, big.req.page_table[0].contiguous()
    own = (kvc.QCache(c.k, c.v, c.scale_k, c.scale_v, T=200, page_table=tab) if q8 else kvc.Cache(c.k, c.v, T=200, page_table=tab))
    b = Built(Step(nq, lens, q8=False, seed=5))
    b.cache = own
    b.req = kvc.Requests(b.req.q_begin, b.req.kv_len, max(nq), 200)
    b.st.q8 = q8
    b.val_k, b.val_v = [big.val_k[0][:n] for n in lens], [big.val_v[0][:n] for n in lens]
    out, lse = b.run()
    b.check(out, lse)
    with pytest.raises(kvc.KvcError):                       # more than the cache holds
        kvc.kvc_attend(kvc.Requests(b.req.q_begin, b.req.kv_len, max(nq), 201), b.q, own, 0, out, b.workspace())


def test_two_streams_at_once():
    """Calls on two streams, each with its own scratch, interleaved many times: the results of calls made alone."""
    bs = [Built(Step([1, 60, 1], [900, 400, 33], G=8)), Built(Step([1] * 20, [500 + i for i in range(20)], q8=True, seed=3))]
    want = [b.run() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    outs = [(torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda"), b.workspace()) for b in bs]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s, (out, lse, ws) in zip(bs, streams, outs):
            with torch.cuda.stream(s):
                kvc.kvc_attend(b.req, b.q, b.cache, 0, out, ws, lse=lse)
    torch.cuda.synchronize()
    for (out, lse, _), (o, l) in zip(outs, want):
        assert torch.equal(out, o) and torch.equal(lse, l)
    assert kvc.kvc_status_poll() == 0


def test_calls_in_a_row_share_one_scratch():
    """One stream, one workspace, calls of both kernels one behind the other: each result that of the call alone."""
    bs = [Built(Step([1] * 5, [700, 300, 9, 128, 513], seed=1)), Built(Step([200], [700], G=2, seed=2)), Built(Step([1, 80], [640, 300], seed=3))]
    want = [b.run()[0] for b in bs]
    n = max(b.workspace().numel() for b in bs)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    outs = [[torch.zeros_like(b.q) for b in bs] for _ in range(10)]
    for row in outs:
        for b, out in zip(bs, row):
            kvc.kvc_attend(b.req, b.q, b.cache, 0, out, ws)
    torch.cuda.synchronize()
    for row in outs:
        for out, w in zip(row, want):
            assert torch.equal(out, w)


def test_nan_in_a_seen_key_or_value_shows():
    """A NaN that a row does see is not swallowed: the row's output is not finite (bf16 and 8-bit, both kernels)."""
    for q8 in (False, True):
        for nq in (1, 70):
            b = Built(Step([nq], [300], q8=q8))
            code = b.cache.k.view(torch.uint8) if q8 else b.cache.k
            page = int(b.req.page_table[0, 3])
            code[0, page, 0, 5, 7] = 0x7F if q8 else float("nan")
            out, lse = b.run()
            assert not torch.isfinite(out[:, : b.st.G]).any() and torch.isfinite(out[:, b.st.G:]).all()
            b = Built(Step([nq], [300], q8=q8))
            code = b.cache.v.view(torch.uint8) if q8 else b.cache.v
            code[0, page, 0, 5, 7] = 0x7F if q8 else float("nan")
            out, lse = b.run()
            assert not torch.isfinite(out[:, : b.st.G, 7]).any() and torch.isfinite(out[:, b.st.G:]).all() and torch.isfinite(lse).all()


def test_same_call_twice_is_bit_identical():
    b = Built(Step([1, 90, 1], [900, 400, 33], G=8))
    one, two = b.run(), b.run()
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


@pytest.mark.parametrize("path", [kvc.KVC_PATH_GENERIC, kvc.KVC_PATH_AUTO])
@pytest.mark.parametrize("nq", [1, 70])
def test_bad_pages_and_lengths_are_flagged(nq, path):
    """A page id outside the pool reads as zero keys and values; a length above its bound skips the request.  Other
    requests keep their answers."""
    kvc.kvc_set_path(path)
    try:
        b = Built(Step([nq, nq, nq], [200, 180, 190], page=16))
        want, _ = b.run()
        kvc.kvc_status_reset()
        tab = b.req.page_table
        keep = int(tab[1, 2])
        tab[1, 2] = 10 ** 6
        out, _ = b.run()
        assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE
        kvc.kvc_status_reset()
        lo, hi = nq, 2 * nq
        assert torch.equal(out[:lo], want[:lo]) and torch.equal(out[hi:], want[hi:])
        z = b.val_k[1].copy(), b.val_v[1].copy()
        b.val_k[1][32:48], b.val_v[1][32:48] = 0, 0
        lse = b.run()[1]
        b.check(out, lse)
        b.val_k[1], b.val_v[1] = z
        tab[1, 2] = keep
        kvc.kvc_status_reset()
        b.req.kv_len[1] = 5000
        out, _ = b.run()
        assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_LENGTH
        assert torch.equal(out[:lo], want[:lo]) and torch.equal(out[hi:], want[hi:]) and (out[lo:hi] == 7.0).all()
    finally:
        kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
        kvc.kvc_status_reset()


def test_offsets_past_32_bits():
    """The last pages of a pool whose offsets pass 2^32 elements."""
    page, H, d = 128, 8, 128
    P = (1 << 32) // (page * H * d) + 40
    k = torch.zeros(1, P, H, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    small = Built(Step([1, 30], [250, 200], H=H, G=2, page=page))
    tab = small.req.page_table.clone()
    want = small.run()
    n = small.cache.P
    k[:, P - n:], v[:, P - n:] = small.cache.k, small.cache.v
    tab[tab >= 0] += P - n
    req = kvc.Requests(small.req.q_begin, small.req.kv_len, 30, 250, page_table=tab)
    out, lse = torch.zeros_like(small.q), torch.zeros(small.q.shape[:2], device="cuda")
    for path in (kvc.KVC_PATH_AUTO, kvc.KVC_PATH_GENERIC):
        kvc.kvc_set_path(path)
        try:
            kvc.kvc_attend(req, small.q, kvc.Cache.pool(k, v), 0, out, small.workspace(), lse=lse)
            torch.cuda.synchronize()
        finally:
            kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
        small.check(out, lse)
    assert kvc.kvc_status_poll() == 0


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_unit_in_many_pieces(d, q8, loose):
    """One tile of rows over 79 tiles of keys, a piece a block, the last one out of sight of some rows; with a bound far
    above the request's length the join is sized for many units."""
    b = Built(Step(nq=[40], kv=[10007], H=1, G=4, d=d, q8=q8, seed=71))
    if loose:
        b.req = kvc.Requests(b.req.q_begin, b.req.kv_len, 8192, 10007, page_table=b.req.page_table)
    b.check(*b.run())


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 1), (128, 16)])
def test_a_large_mixed_batch(d, G, q8):
    """Enough key tiles by the call's bounds (40 requests x 2 heads x 28 tiles) that single tokens and chunks are served by
    a kernel each, behind one another in one workspace."""
    rng = random.Random(5)
    nq = [rng.choice([1, 1, 1, 2, 0, 9]) for _ in range(38)] + [40, 1]
    kv = [max(n, rng.randrange(0, 400)) for n in nq[:-2]] + [600, 3500]
    b = Built(Step(nq=nq, kv=kv, H=2, G=G, d=d, q8=q8, spare=2, seed=81))
    b.check(*b.run())
    again = b.run()
    assert all(torch.equal(x, y) for x, y in zip(again, b.run()))
