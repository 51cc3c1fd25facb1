"""kvc_verify against the oracle: accepted rows and next tokens are whole numbers and have to be equal."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from draft_helpers import I32, flat, random_parents, requests
from oracle import draft_oracle as orc

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, nq, V, kind="tree", drawn=True, seed=0, spare=0, pad=0, sharp=2.0, near=1.0):
        rng = np.random.default_rng(seed)
        self.nq, self.V, self.drawn = nq, V, drawn
        self.parents = random_parents(nq, seed, kind)
        rows = sum(nq) + spare
        z = rng.normal(size=(rows, V)) * sharp
        soft = lambda z: np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)
        wide = lambda p: torch.cat([torch.from_numpy(p.astype(np.float32)), torch.full((rows, pad), 9.0)], 1).cuda()[:, :V]
        self.target, self.draft = wide(soft(z)), wide(soft(z + near * rng.normal(size=z.shape)))
        d = self.draft.cpu().double().numpy()
        first = np.repeat(np.concatenate([[0], np.cumsum(nq)])[:-1], nq)
        self.token = np.zeros(rows, np.int64)
        for r, a in enumerate(x for p in self.parents for x in p):
            if a >= 0:
                self.token[r] = rng.choice(V, p=d[first[r] + a] / d[first[r] + a].sum())
        self.u, self.u_next = rng.random(rows).astype(np.float32), rng.random(len(nq)).astype(np.float32)
        self.u, self.u_next = np.minimum(self.u, 1 - 2.0 ** -24), np.minimum(self.u_next, 1 - 2.0 ** -24)
        self.rows, self.spare = rows, spare

    def run(self, stride=None, kv=None, **kw):
        n, max_q = len(self.nq), max(self.nq + [0])
        stride = max_q if stride is None else stride
        req = requests(self.nq, [m + 3 for m in self.nq] if kv is None else kv, **kw)
        dev = lambda x, t: torch.from_numpy(np.asarray(x)).to(t).cuda()
        self.kept = torch.full((n, stride), 55, dtype=I32, device="cuda")
        self.n_kept, self.next = (torch.full((n,), 55, dtype=I32, device="cuda") for _ in range(2))
        kvc.kvc_status_reset()
        kvc.kvc_verify(req, flat(self.parents, self.spare, -9).cuda(), dev(self.token, I32), self.target, dev(self.u, torch.float32),
                       dev(self.u_next, torch.float32), self.kept, self.n_kept, self.next, draft=self.draft if self.drawn else None)
        torch.cuda.synchronize()
        self.flags = kvc.kvc_status_poll()
        kvc.kvc_status_reset()
        return self

    def check(self):
        t, d = self.target.cpu().double().numpy(), self.draft.cpu().double().numpy()
        kept, n_kept, nxt = self.kept.cpu().tolist(), self.n_kept.cpu().tolist(), self.next.cpu().tolist()
        r, max_q, lens = 0, max(self.nq + [0]), []
        for b, m in enumerate(self.nq):
            if m == 0:
                want, x = [], -1
            else:
                s = slice(r, r + m)
                want, x = orc.verify(self.parents[b], self.token[s].tolist(), t[s], d[s] if self.drawn else None, self.u[s].astype(np.float64),
                                     float(self.u_next[b]))
            assert n_kept[b] == len(want) and kept[b][:max_q] == want + [-1] * (max_q - len(want)) and kept[b][max_q:] == [55] * (len(kept[b]) - max_q), (b, kept[b], want)
            assert nxt[b] == x, (b, nxt[b], x)
            lens.append(len(want))
            r += m
        return lens


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
@pytest.mark.parametrize("nq,V,kind", [([1], 1, "tree"), ([4], 3, "tree"), ([6], 1000, "chain"), ([5, 0, 9, 1], 127, "tree"), ([12] * 20, 50, "tree"),
                                       ([8, 16], 4096, "tree"), ([8, 3], 4097, "chain"), ([10] * 5, 32000, "tree"), ([7, 7], 50001, "tree"),
                                       ([200, 90], 600, "tree"), ([3], 131072, "tree"), ([5] * 40, 6001, "tree")])
def test_against_the_oracle(nq, V, kind, drawn):
    for seed in range(3):
        c = Case(nq, V, kind, drawn, seed=seed, sharp=1.0 + 2 * seed, near=(1.0, 0.2, 3.0)[seed])
        c.run().check()
        assert c.flags == 0


def test_every_outcome_occurs():
    """Chains that stay whole, end at once, and end inside; second siblings that stay."""
    c = Case([6] * 64, 40, "chain", seed=1)
    assert set(c.run().check()) >= {1, 2, 3, 6}
    c = Case([3] * 64, 40, seed=2, near=4.0)
    c.parents = [[-1, 0, 0]] * 64
    c.run().check()
    assert {int(x) for x in c.kept[:, 1]} == {-1, 1, 2}


@pytest.mark.parametrize("V,pad", [(1000, 24), (1000, 1), (5003, 5), (40001, 3)])
@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_padded_rows_wide_lists(V, pad, drawn):
    """Rows of a wider table (16-byte aligned or not), a wider list of kept rows, padding rows behind the requests."""
    c = Case([5, 8], V, drawn=drawn, seed=V, spare=2, pad=pad)
    c.run(stride=11).check()


def test_equal_distributions_always_accept():
    c = Case([9] * 8, 3000, "chain", seed=5)
    c.draft = c.target.clone()
    assert set(c.run().check()) == {9}


def test_no_residual():
    """P <= q everywhere (rounding can have it so): the node's own distribution, further siblings are rejected."""
    c = Case([4] * 6, 5000, seed=6)
    c.parents = [[-1, 0, 0, 0]] * 6
    c.draft = torch.clamp(c.target * 3.0, max=1.0)
    c.u[:] = 0.9999
    c.run().check()
    assert (c.n_kept == 1).all() and c.flags == 0


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
@pytest.mark.parametrize("V", [100, 9000])
def test_one_hot_targets_and_ends_of_the_random_numbers(V, drawn):
    c = Case([6] * 12, V, seed=7, drawn=drawn)
    top = c.target.argmax(-1)
    c.target = torch.nn.functional.one_hot(top, V).float()
    c.u[::3], c.u[1::3] = 0.0, 1 - 2.0 ** -24
    c.u_next[::2], c.u_next[1::2] = 0.0, 1 - 2.0 ** -24
    c.run().check()
    c = Case([6] * 12, V, seed=8, drawn=drawn)
    c.u_next[::2], c.u_next[1::2] = 0.0, 1 - 2.0 ** -24
    c.target[:, : V // 3] = 0.0
    c.target[:, -V // 3:] = 0.0
    c.run().check()


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
def test_nan_negative_and_empty_distributions(drawn):
    c = Case([5] * 9, 6000, seed=9, drawn=drawn)
    c.target[:, ::7] = float("nan")
    c.target[:, 1::7] = -1.0
    c.draft[:, 2::7] = float("nan")
    c.draft[:, 3::7] = -0.5
    c.run().check()
    assert c.flags == 0
    c.target[:] = 0.0
    c.run().check()
    assert (c.next == -1).all() and c.flags == kvc.KVC_FLAG_BAD_PROB
    c.target[:, 5] = float("inf")
    c.run()
    assert (c.next == -1).all() and c.flags == kvc.KVC_FLAG_BAD_PROB


def test_the_same_token_twice_and_tokens_out_of_range():
    for drawn in (True, False):
        c = Case([6] * 30, 20, seed=10, drawn=drawn, near=2.0)
        c.parents = [[-1, 0, 0, 0, 0, 0]] * 30
        c.token[:] = np.where(np.arange(180) % 6 < 4, c.token, np.roll(c.token, 1))
        c.run().check()
        c.token[2::6], c.token[3::12] = 20, -5
        c.run().check()
        assert c.flags == kvc.KVC_FLAG_BAD_TREE


def test_parents_out_of_range_are_never_reached():
    c = Case([5] * 4, 30, seed=11)
    c.parents = [[-1, 0, 7, 2, -3]] * 4
    c.run()
    assert c.flags == kvc.KVC_FLAG_BAD_TREE
    c.parents = [[-1, 0, -1, -1, -1]] * 4
    c.check()


def test_requests_out_of_bounds_are_answered():
    c = Case([4, 5, 3], 50, seed=12)
    c.run(kv=[7, 99, 6], max_kv=20)
    assert c.flags == kvc.KVC_FLAG_BAD_LENGTH and c.n_kept[1] == 0 and c.next[1] == -1 and (c.kept[1] == -1).all()
    assert c.n_kept[0] >= 1 and c.n_kept[2] >= 1


def test_without_rows():
    c = Case([0, 0], 50, seed=1, spare=1)
    c.run().check()
    c = Case([3], 50, seed=1)
    c.nq, c.parents = [0], [[]]
    c.spare = 3
    c.run(max_q=3, stride=3)
    assert c.kept.tolist() == [[-1] * 3] and c.n_kept.tolist() == [0] and c.next.tolist() == [-1]
