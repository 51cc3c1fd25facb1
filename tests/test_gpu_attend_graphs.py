"""Attention and append inside captured graphs, among copies, fills and branches; each replay equals eager calls."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 60])
def test_copies_and_fills_between_the_calls(nq, q8):
    """Lengths and queries arrive by copies captured right before the call, the output leaves by one right behind it."""
    b = Built(Step([nq, nq], [500, 300], q8=q8))
    ws, out, lse = b.workspace(), torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")
    q_in, kv_in, got = b.q.clone(), b.req.kv_len.clone(), torch.zeros_like(b.q)
    call = lambda: kvc.kvc_attend(b.req, b.q, b.cache, 0, out, ws, lse=lse)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.q.copy_(q_in)
        b.req.kv_len.copy_(kv_in)
        call()
        got.copy_(out)
        out.zero_()
        call()
    gen = torch.Generator().manual_seed(1)
    for lens in ([500, 300], [77 + nq, 200], [nq, 299]):
        q_new = torch.randn(b.q.shape, generator=gen).to(torch.bfloat16).cuda()
        q_in.copy_(q_new)
        kv_in.copy_(torch.tensor(lens, dtype=torch.int32))
        g.replay()
        g.replay()
        torch.cuda.synchronize()
        first, second = got.clone(), out.clone()
        b.q.copy_(q_new)
        b.req.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        want, _ = b.run()
        assert torch.equal(first, want) and torch.equal(second, want)


def test_branches_of_a_graph():
    """Two branches, a call and a scratch each, joined by an append that writes what the next replay reads."""
    H, d, page, P = 2, 128, 16, 40
    g = torch.Generator().manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    pool = kvc.Cache.pool(rnd(1, P, H, page, d), rnd(1, P, H, page, d))
    tab = torch.randperm(P, generator=g)[:38].to(torch.int32).view(2, 19).cuda()
    kv = torch.tensor([200, 120], dtype=torch.int32, device="cuda")
    begin = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    req = kvc.Requests(begin, kv, 1, 300, page_table=tab)
    q = [rnd(2, H * 4, d) for _ in range(2)]
    new = rnd(2, H, d), rnd(2, H, d)
    outs = [torch.zeros_like(x) for x in q]
    ws = [torch.empty(kvc.kvc_attend_workspace_bytes(req, pool, H * 4), dtype=torch.uint8, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        kvc.kvc_append(req, *new, pool, 0)
        side.wait_stream(main)
        kvc.kvc_attend(req, q[0], pool, 0, outs[0], ws[0])
        with torch.cuda.stream(side):
            kvc.kvc_attend(req, q[1], pool, 0, outs[1], ws[1])
        main.wait_stream(side)
        kv.add_(1)

    keep = pool.k.clone(), pool.v.clone(), kv.clone()
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        step()
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    runs = []
    for go in (step, graph.replay):
        for dst, src in zip((pool.k, pool.v, kv), keep):
            dst.copy_(src)
        seen = []
        for _ in range(30):
            go()
            seen.append([o.clone() for o in outs])
        torch.cuda.synchronize()
        runs.append(seen)
    for a, b in zip(*runs):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert kvc.kvc_status_poll() == 0
