"""A serving step for the tests: requests over a poisoned pool (or contiguous rows) and its float64 answer."""
import dataclasses
import math

import numpy as np
import torch

import paper_2609_34060_b200 as kvc
from oracle import attend_oracle as orc

NAN = float("nan")


@dataclasses.dataclass
class Step:
    nq: list
    kv: list
    H: int = 2
    G: int = 4
    d: int = 128
    page: int = 16                 # 0: contiguous rows shared by all requests
    token_major: bool = False
    L: int = 1
    layer: int = 0
    q8: bool = False
    causal: bool = True
    spare: int = 0                 # padding rows behind the last request
    key_scale: float = 1.0
    ramp: float = 0.0              # keys grow (or, negative, shrink) linearly with their position, by up to this factor
    seed: int = 0


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().to(torch.float32).numpy().astype(np.float64)


class Built:
    """Tensors of a step: rows [n][kv, H, d] as the requests see them, the pool that holds them, everything else NaN."""

    def __init__(self, st: Step, dev="cuda"):
        self.st, g = st, torch.Generator().manual_seed(1000 + st.seed)
        n = len(st.nq)
        rnd = lambda *s: torch.randn(*s, generator=g)
        T = max(list(st.kv) + [0])
        if st.page:
            need = [-(-x // st.page) for x in st.kv]
            P = sum(need) + 3
            perm = torch.randperm(P, generator=g)
            table = torch.full((n, max(max(need + [0]), 1)), -7, dtype=torch.int32)      # entries nobody needs name no page
            at = 0
            for b in range(n):
                table[b, : need[b]] = perm[at: at + need[b]].to(torch.int32)
                at += need[b]
            shape = (st.L, P, st.page, st.H, st.d)
        else:
            table, shape = None, (st.L, T + 2, st.H, st.d)
        self.rows_k, self.rows_v = [], []
        pools = []
        for is_v in (0, 1):
            pool = torch.full(shape, NAN)
            shared = rnd(T, st.H, st.d) * (1.0 if is_v else st.key_scale)
            for b in range(n):
                x = (shared[: st.kv[b]] if not st.page else rnd(st.kv[b], st.H, st.d) * (1.0 if is_v else st.key_scale))
                if st.ramp and not is_v and st.kv[b]:
                    at = torch.arange(st.kv[b]) / st.kv[b]
                    x = x * (abs(st.ramp) * (at if st.ramp > 0 else 1 - at))[:, None, None]
                x = x.to(torch.bfloat16)
                (self.rows_v if is_v else self.rows_k).append(x)
                if st.page:
                    for j in range(-(-st.kv[b] // st.page)):
                        m = min(st.page, st.kv[b] - j * st.page)
                        pool[st.layer, int(table[b, j]), :m] = x[j * st.page: j * st.page + m].float()
                elif st.kv[b] == T:
                    pool[st.layer, :T] = x.float()
            if not st.token_major:
                pool = pool.transpose(-3, -2)
            pools.append(pool.contiguous())
        bf = [p.to(torch.bfloat16) for p in pools]
        if st.q8:
            made = [orc.quantize_rows(p.double().numpy()) for p in bf]
            code = [torch.from_numpy(c).view(torch.float8_e4m3fn).to(dev) for c, _ in made]
            exp = [torch.from_numpy(e) for _, e in made]
            for e, p in zip(exp, bf):
                e[torch.isnan(p).all(-1)] = 255                                          # unused rows: NaN codes and exponents
            exp = [e.to(dev) for e in exp]
            q = lambda x: torch.from_numpy(orc.dequantize_rows(*orc.quantize_rows(x.double().numpy())))
            self.val_k, self.val_v = [q(x).numpy() for x in self.rows_k], [q(x).numpy() for x in self.rows_v]
            if st.page:
                self.cache = kvc.QCache.pool(code[0], code[1], exp[0], exp[1], token_major=st.token_major)
            else:
                self.cache = kvc.QCache(code[0], code[1], exp[0], exp[1], token_major=st.token_major)
        else:
            self.val_k, self.val_v = [f64(x) for x in self.rows_k], [f64(x) for x in self.rows_v]
            k, v = (p.to(dev) for p in bf)
            self.cache = (kvc.Cache.pool(k, v, token_major=st.token_major) if st.page
                          else kvc.Cache(k, v, token_major=st.token_major))
        begin = np.concatenate([[0], np.cumsum(st.nq)]).astype(np.int32)
        self.rows = int(begin[-1]) + st.spare
        self.begin = begin
        self.req = kvc.Requests(torch.from_numpy(begin).to(dev), torch.tensor(st.kv, dtype=torch.int32, device=dev),
                                max(list(st.nq) + [0]), T, page_table=None if table is None else table.to(dev))
        self.q_cpu = rnd(max(self.rows, 1), st.H * st.G, st.d).to(torch.bfloat16)[: self.rows]
        self.q = self.q_cpu.to(dev)
        self.scale = 1.0 / math.sqrt(st.d)

    def workspace(self, dev="cuda"):
        n = kvc.kvc_attend_workspace_bytes(self.req, self.cache, self.st.H * self.st.G)
        return torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device=dev)             # NaN patterns: written before read

    def run(self, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device=self.q.device)
        lse = torch.full(self.q.shape[:2], 7.0, device=self.q.device)
        kvc.kvc_attend(self.req, self.q, self.cache, self.st.layer, out, self.workspace(), causal=self.st.causal, lse=lse, **kw)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out, lse):
        """Every element against float64.  Tolerances, before any run, from the rounding steps of the method:
        output to bf16 2^-8 |ref|; probabilities to bf16 2^-8 of each term, sum_t p_t |v_t| in all (an 8-bit cache: three
        e4m3 parts of each, closer than that, with steps no finer than 2^-24 of the row's largest, at most 2^-23 sum |v_t|);
        a float32 logit of d products is off by at most (d + 8) 2^-24 scale sum |q_c k_c|, which moves every probability
        by that much in relative terms and their sum once more; n terms added in float32 cost n 2^-24; the exponential 2^-21."""
        st = self.st
        o, s = f64(out), lse.detach().cpu().numpy().astype(np.float64)
        worst = 0.0
        for b in range(len(st.nq)):
            for j in range(st.nq[b]):
                r = int(self.begin[b]) + j
                end = max(0, min(st.kv[b], st.kv[b] - st.nq[b] + j + 1) if st.causal else st.kv[b])
                for a in range(st.H * st.G):
                    h = a // st.G
                    ref, l, absv, big = orc.attend_row(f64(self.q_cpu[r, a]), self.val_k[b][:end, h], self.val_v[b][:end, h], self.scale)
                    if end == 0:
                        assert np.all(o[r, a] == 0) and s[r, a] == -np.inf
                        continue
                    ds = (st.d + 8) * 2.0 ** -24 * self.scale * big
                    rel = 2.0 ** -8 + 2 * ds + end * 2.0 ** -23 + 2.0 ** -21
                    tol = 2.0 ** -8 * np.abs(ref) + 1.01 * rel * absv + 1e-30
                    if st.q8:
                        tol = tol + 2.0 ** -23 * np.abs(self.val_v[b][:end, h]).sum(0)
                    err = np.abs(o[r, a] - ref)
                    worst = max(worst, float((err / tol).max()))
                    assert np.all(err <= tol), (b, j, a, float((err / tol).max()), np.argmax(err / tol))
                    ltol = ds + end * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * abs(l)
                    assert abs(s[r, a] - l) <= ltol, (b, j, a, s[r, a], l, ltol)
        if st.spare:
            assert (out[self.rows - st.spare:] == 7.0).all() and (lse[self.rows - st.spare:] == 7.0).all(), "padding rows"
        return worst
