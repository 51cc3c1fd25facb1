"""A step of drafted tokens as a serving program runs it: all operators in a row, eager, captured, on another stream."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import f64
from draft_helpers import I32, flat, random_parents

pytestmark = pytest.mark.gpu


class Program:
    """Two layers, three requests, a pool of pages with room for many steps.  The model's parts are random tensors."""

    def __init__(self, q8, seed=0, n=3, max_q=9, H=2, G=4, d=128, V=500, page=16, L=2, kv=(70, 33, 200)):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)
        self.n, self.max_q, self.H, self.Hq, self.d, self.V, self.L, self.q8 = n, max_q, H, H * G, d, V, L, q8
        self.max_kv, self.page = 320, page
        per = self.max_kv // page
        P = n * per + 2
        self.table = torch.randperm(P, generator=g)[: n * per].view(n, per).to(I32).cuda()
        bf = kvc.Cache.pool(*(rnd(L, P, H, page, d).to(torch.bfloat16).cuda() for _ in range(2)))
        self.cache = bf
        if q8:
            self.cache = kvc.QCache.pool(*(rnd(L, P, H, page, d).clamp(-3, 3).mul(100).to(torch.float8_e4m3fn).cuda() for _ in range(2)),
                                         *(torch.randint(118, 121, (L, P, H, page), generator=g).to(torch.uint8).cuda() for _ in range(2)))
        self.context = torch.tensor(kv, dtype=I32, device="cuda")        # tokens before the step's new ones
        self.begin = torch.arange(0, (n + 1) * max_q, max_q, dtype=I32, device="cuda")
        self.kv = torch.zeros(n, dtype=I32, device="cuda")
        self.req = kvc.Requests(self.begin, self.kv, max_q, self.max_kv, page_table=self.table)
        rows = n * max_q
        self.parent = torch.zeros(rows, dtype=I32, device="cuda")
        self.tree = kvc.Tree(self.parent, max_q)
        self.rotary = kvc.Rotary(kvc.Rope(5e5), depth=self.tree.depth)
        self.qkv = torch.zeros(L, rows, self.Hq + 2 * H, d, dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros(L, rows, self.Hq, d, dtype=torch.bfloat16, device="cuda")
        self.ws = torch.empty(kvc.kvc_attend_workspace_bytes(self.req, self.cache, self.Hq), dtype=torch.uint8, device="cuda")
        self.target, self.draft = (torch.zeros(rows, V, device="cuda") for _ in range(2))
        self.token, self.u = torch.zeros(rows, dtype=I32, device="cuda"), torch.zeros(rows, device="cuda")
        self.u_next = torch.zeros(n, device="cuda")
        self.kept = torch.zeros(n, max_q, dtype=I32, device="cuda")
        self.n_kept, self.next, self.kv_out = (torch.zeros(n, dtype=I32, device="cuda") for _ in range(3))

    def inputs(self, seed):
        g, rows = torch.Generator().manual_seed(seed), self.n * self.max_q
        self.parents = random_parents([self.max_q] * self.n, seed)
        p = torch.softmax(torch.randn(rows, self.V, generator=g) * 3, -1)
        q = torch.softmax(torch.log(p) + torch.randn(rows, self.V, generator=g) * 0.5, -1)
        tok = torch.zeros(rows, dtype=torch.long)
        for b, par in enumerate(self.parents):
            for j, a in enumerate(par):
                if a >= 0:
                    tok[b * self.max_q + j] = torch.multinomial(q[b * self.max_q + a], 1, generator=g)[0]
        for dst, src in ((self.parent, flat(self.parents)), (self.qkv, torch.randn(self.qkv.shape, generator=g).to(torch.bfloat16)), (self.target, p),
                         (self.draft, q), (self.token, tok.to(I32)), (self.u, torch.rand(rows, generator=g)), (self.u_next, torch.rand(self.n, generator=g))):
            dst.copy_(src)

    def step(self):
        self.kv.copy_(self.context).add_(self.max_q)
        kvc.kvc_tree_build(self.req, self.tree)
        for l in range(self.L):
            q, k, v = self.qkv[l, :, : self.Hq], self.qkv[l, :, self.Hq: self.Hq + self.H], self.qkv[l, :, self.Hq + self.H:]
            kvc.kvc_append_rotated(self.req, self.rotary, k, v, self.cache, l, q=q, q_out=q)
            kvc.kvc_attend_tree(self.req, self.tree, q, self.cache, l, self.out[l], self.ws)
        kvc.kvc_verify(self.req, self.parent, self.token, self.target, self.u, self.u_next, self.kept, self.n_kept, self.next, draft=self.draft)
        kvc.kvc_keep(self.req, self.kept, self.n_kept, self.cache, self.kv_out)
        self.context.copy_(self.kv_out)

    def state(self):
        c = self.cache
        t = [c.k, c.v] + ([c.scale_k, c.scale_v] if self.q8 else [])
        return [x.view(torch.uint8).clone() if x.element_size() == 1 else x.clone() for x in t + [self.out, self.kept, self.n_kept, self.next, self.context, self.qkv]]


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_a_step_equals_token_by_token(q8):
    """The deepest kept draft's attention in the tree is the attention of a single token over the cache that kvc_keep left:
    the same keys, so both outputs lie within twice the method's roundings (bf16 outputs and probabilities) of one another;
    the next step goes on from there."""
    p = Program(q8)
    for seed in (1, 2, 3):
        p.inputs(seed)
        before = p.context.clone()
        kvc.kvc_status_reset()
        p.step()
        torch.cuda.synchronize()
        assert kvc.kvc_status_poll() == 0
        n_kept = p.n_kept.tolist()
        assert p.context.tolist() == [a + b for a, b in zip(before.tolist(), n_kept)] and min(n_kept) >= 1
        one = kvc.Requests(torch.arange(p.n + 1, dtype=I32, device="cuda"), p.context, 1, p.max_kv, page_table=p.table)
        ws = torch.empty(kvc.kvc_attend_workspace_bytes(one, p.cache, p.Hq), dtype=torch.uint8, device="cuda")
        last = [b * p.max_q + int(p.kept[b, n_kept[b] - 1]) for b in range(p.n)]
        for l in range(p.L):
            q = p.qkv[l, last, : p.Hq].contiguous()
            out = torch.zeros_like(q)
            kvc.kvc_attend(one, q, p.cache, l, out, ws)
            torch.cuda.synchronize()
            a, b = f64(out), f64(p.out[l, last])
            # |out| <= max |V|: values of the pool and the new tokens are normal draws (times 4 in 8 bits), at most 6
            big = 6.0 * (4.0 if q8 else 1.0)
            assert np.all(np.abs(a - b) <= 2 * (2.0 ** -8 * np.abs(a) + 2.0 ** -8 * big))
        for b in range(p.n):                       # depths ascend by one along the kept rows: positions are the places in the cache
            assert p.tree.depth[[b * p.max_q + int(x) for x in p.kept[b, : n_kept[b]]]].tolist() == list(range(n_kept[b]))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_captured_steps(q8):
    """A graph of a whole step, replayed with other trees, lengths and numbers, equals eager steps on another stream."""
    a, b = Program(q8), Program(q8)
    side = torch.cuda.Stream()
    a.inputs(1)
    start = a.context.clone()
    was = a.state()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    c = a.cache
    for t, x in zip([c.k, c.v] + ([c.scale_k, c.scale_v] if q8 else []), was):
        (t.view(torch.uint8) if t.element_size() == 1 else t).copy_(x)
    a.context.copy_(start)
    for seed in range(5):
        for p in (a, b):
            p.inputs(seed)
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            b.step()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x.view(torch.uint8) if x.dtype == torch.bfloat16 else x, y.view(torch.uint8) if y.dtype == torch.bfloat16 else y)
    assert kvc.kvc_status_poll() == 0


def test_two_steps_at_once_on_two_streams():
    """Two programs, interleaved on two streams, each as it is alone."""
    alone, one, two = Program(False, seed=4), Program(False, seed=4), Program(True, seed=5)
    other = Program(True, seed=5)
    for p, s in ((alone, 1), (one, 1), (two, 2), (other, 2)):
        p.inputs(s)
    torch.cuda.synchronize()
    alone.step(), other.step()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s1):
        one.step()
    with torch.cuda.stream(s2):
        two.step()
    torch.cuda.synchronize()
    for x, y in list(zip(alone.state(), one.state())) + list(zip(other.state(), two.state())):
        assert torch.equal(x.view(torch.uint8) if x.dtype == torch.bfloat16 else x, y.view(torch.uint8) if y.dtype == torch.bfloat16 else y)
