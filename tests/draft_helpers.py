"""Steps of drafted tokens for the tests: trees, ragged request lists, their float64 answers."""
import numpy as np
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step, f64
from oracle import attend_oracle as aorc
from oracle import draft_oracle as orc

I32 = torch.int32


def random_parents(nq, seed, kind="tree"):
    """One list a request: a tree whose rows follow one of the earlier rows, a chain, or a forest."""
    rng = np.random.default_rng(seed)
    out = []
    for m in nq:
        if kind == "chain":
            out.append(list(range(-1, m - 1)))
        else:
            p = [int(rng.integers(max(0, j - 6), j)) if j else -1 for j in range(m)]
            if kind == "forest":
                p = [-1 if rng.random() < 0.3 else a for a in p]
            out.append(p)
    return out


def flat(lists, spare=0, fill=0, dtype=I32):
    return torch.tensor([x for p in lists for x in p] + [fill] * spare, dtype=dtype)


def built_tree(req, parents, rows, words=None, dev="cuda"):
    """A kvc.Tree filled by kvc_tree_build."""
    mask = None if words is None else torch.zeros(rows, words, dtype=I32, device=dev)
    t = kvc.Tree(flat(parents, rows - sum(map(len, parents))).to(dev), req.max_q, mask=mask)
    kvc.kvc_tree_build(req, t)
    return t


class TreeBuilt(Built):
    """A step over a poisoned pool whose new tokens form trees (or see what `seen` says)."""

    def __init__(self, st: Step, kind="tree", seen=None, words=None):
        super().__init__(st)
        self.parents = random_parents(st.nq, st.seed + 7, kind)
        self.seen = [orc.tree_rows(p)[0] for p in self.parents] if seen is None else seen
        self.tree = built_tree(self.req, self.parents, self.rows, words)
        if seen is not None:
            w = int(self.tree.mask.shape[1])
            m = np.concatenate([orc.mask_words(s, w) for s in seen] + [np.zeros((st.spare, w), np.uint32)])
            self.tree.mask.copy_(torch.from_numpy(m.view(np.int32)))

    def run_tree(self, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=self.q.device)
        lse = torch.full(self.q.shape[:2], 7.0, device=self.q.device)
        kvc.kvc_attend_tree(self.req, self.tree, self.q, self.cache, self.st.layer, out, self.workspace(), lse=lse, **kw)
        torch.cuda.synchronize()
        return out, lse

    def check_tree(self, out, lse):
        """Every element against float64, with the tolerances of Built.check (the same kernels, the same roundings)."""
        st = self.st
        o, s = f64(out), lse.detach().cpu().numpy().astype(np.float64)
        for b in range(len(st.nq)):
            first = st.kv[b] - st.nq[b]
            for j in range(st.nq[b]):
                r = int(self.begin[b]) + j
                keys = [t for t in range(max(first, 0))] + [first + a for a in sorted(self.seen[b][j]) if a <= j and first + a >= 0]
                for a in range(st.H * st.G):
                    h = a // st.G
                    k, v = self.val_k[b][keys, h], self.val_v[b][keys, h]
                    ref, l, absv, big = aorc.attend_row(f64(self.q_cpu[r, a]), k, v, self.scale)
                    if not keys:
                        assert np.all(o[r, a] == 0) and s[r, a] == -np.inf
                        continue
                    ds = (st.d + 8) * 2.0 ** -24 * self.scale * big
                    if st.q8:
                        # queries meet the codes as two e4m3 parts of q 2^-b, whose largest channel is above 224: what the
                        # second leaves is at most half its smallest step, 2^-10, in every channel
                        qr = f64(self.q_cpu[r, a])
                        ds += self.scale * 2.0 ** -10 * np.abs(qr).max() / 224.0 * np.abs(k).sum(-1).max()
                    rel = 2.0 ** -8 + 2 * ds + len(keys) * 2.0 ** -23 + 2.0 ** -21
                    tol = 2.0 ** -8 * np.abs(ref) + 1.01 * rel * absv + 1e-30
                    if st.q8:
                        tol = tol + 2.0 ** -23 * np.abs(v).sum(0)
                    err = np.abs(o[r, a] - ref)
                    assert np.all(err <= tol), (b, j, a, float((err / tol).max()))
                    assert abs(s[r, a] - l) <= ds + len(keys) * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * abs(l), (b, j, a, s[r, a], l)
        if st.spare:
            assert (out[self.rows - st.spare:] == 7.0).all() and (lse[self.rows - st.spare:] == 7.0).all(), "padding rows"


def requests(nq, kv, page=0, table=None, max_q=None, max_kv=None, dev="cuda"):
    begin = torch.tensor(np.concatenate([[0], np.cumsum(nq)]), dtype=I32, device=dev)
    return kvc.Requests(begin, torch.tensor(kv, dtype=I32, device=dev), max(list(nq) + [0]) if max_q is None else max_q,
                        max(list(kv) + [0]) if max_kv is None else max_kv, page_table=None if table is None else table.to(dev))


def shuffled_table(kv, page, seed):
    """Pages of every request in no order, and how many the pool has."""
    need = [-(-x // page) for x in kv]
    perm = torch.randperm(sum(need) + 3, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(kv), max(need + [1])), -7, dtype=I32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = perm[at: at + m].to(I32)
        at += m
    return table, sum(need) + 3


def row_of(cache, name, table, b, t, layer):
    """Row t of request b in a cache tensor: [H, ...]."""
    x = getattr(cache, name)[layer]
    if cache.page_table is None:
        return x[t] if cache.token_major else x[:, t]
    p, s = int(table[b, t // cache.page]), t % cache.page
    return x[p, s] if cache.token_major else x[p, :, s]
