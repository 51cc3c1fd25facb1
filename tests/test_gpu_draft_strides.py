"""Caches with gaps between rows, heads, pages and layers, through the C calls: nothing between them is touched."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import f64
from draft_helpers import I32, flat, requests
from oracle import attend_oracle as aorc
from oracle import draft_oracle as orc

pytestmark = pytest.mark.gpu


class Gapped:
    """[L, P, H, page, d] (or [L, H, T, d]) inside a larger buffer full of a fill value."""

    def __init__(self, L, P, H, page, d, paged, q8):
        self.q8, self.d = q8, d
        unit = 16 if q8 else 8
        s_tok, dt = d + unit, torch.uint8 if q8 else torch.bfloat16
        s_head = page * s_tok + 2 * unit
        s_page = H * s_head + 3 * unit
        s_layer = (P if paged else 1) * s_page + unit
        self.fill = 0x2A if q8 else 7.0
        mk = lambda n, t, f: torch.full((n,), f, dtype=t, device="cuda")
        self.buf = [mk(L * s_layer, dt, self.fill) for _ in range(2)]
        shape, strides = ((L, P, H, page, d), (s_layer, s_page, s_head, s_tok, 1)) if paged else ((L, H, page, d), (s_layer, s_head, s_tok, 1))
        self.view = [b.as_strided(shape, strides) for b in self.buf]
        c = kvc.kvc_cache()
        c.k, c.v, c.L, c.H, c.d = self.buf[0].data_ptr(), self.buf[1].data_ptr(), L, H, d
        c.s_layer, c.s_head, c.s_tok = s_layer, s_head, s_tok
        if paged:
            c.layout, c.page_size, c.n_phys_pages, c.s_page, c.T = kvc.KVC_PAGED, page, P, s_page, 0
        else:
            c.layout, c.T = kvc.KVC_CONTIG, page
        self.struct = c
        if q8:
            q = kvc.kvc_qcache()
            q.codes = c
            e_tok, e_head = 3, page * 3 + 1
            e_page = H * e_head + 2
            e_layer = (P if paged else 1) * e_page + 5
            self.ebuf = [mk(L * e_layer, torch.uint8, 0x2B) for _ in range(2)]
            eshape, estr = ((L, P, H, page), (e_layer, e_page, e_head, e_tok)) if paged else ((L, H, page), (e_layer, e_head, e_tok))
            self.eview = [b.as_strided(eshape, estr) for b in self.ebuf]
            q.scale_k, q.scale_v = self.ebuf[0].data_ptr(), self.ebuf[1].data_ptr()
            q.e_layer, q.e_head, q.e_tok = e_layer, e_head, e_tok
            if paged:
                q.e_page = e_page
            self.struct = q

    def value(self, which, *at):
        x = self.view[which][at]
        return aorc.dequantize_rows(x.cpu().numpy(), self.eview[which][at].cpu().numpy()) if self.q8 else f64(x)

    def gaps_untouched(self):
        parts = [(b, v, self.fill) for b, v in zip(self.buf, self.view)]
        if self.q8:
            parts += [(b, v, 0x2B) for b, v in zip(self.ebuf, self.eview)]
        for b, v, fill in parts:
            m = torch.ones_like(b, dtype=torch.bool)
            m.as_strided(v.shape, v.stride()).fill_(False)
            assert (b[m] == fill).all()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("paged", [True, False], ids=["pages", "rows"])
@pytest.mark.parametrize("m,G", [(9, 1), (9, 4)])
def test_gapped_caches(q8, paged, m, G):
    L, P, H, page, d, layer, base = 2, 6, 3, 16, 64, 1, 21
    lib, T = kvc.load(), 40
    c = Gapped(L, P, H, page if paged else T, d, paged, q8)
    table = torch.tensor([[4, 1, 5]], dtype=I32)
    req = requests([m], [base + m], table=table if paged else None, max_kv=T)
    where = (lambda t: (layer, int(table[0, t // page]), slice(None), t % page)) if paged else (lambda t: (layer, slice(None), t))
    g = torch.Generator().manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)
    parents = [[-1, 0, 0, 1, 2, 2, 4, 0, 7]]
    tree = kvc.Tree(flat(parents).cuda(), m)
    kvc.kvc_status_reset()
    kvc.kvc_tree_build(req, tree)
    rot = kvc.Rotary(kvc.Rope(1e4), depth=tree.depth)
    heads = lambda t: kvc.kvc_heads(t.data_ptr(), t.shape[0], t.shape[1], 0, 0)
    ref = lambda x: C.byref(x)
    # the context: a chain of base tokens at their positions, then the drafts
    ctx_k, ctx_v, k, v, q = rnd(base, H, d), rnd(base, H, d), rnd(m, H, d), rnd(m, H, d), rnd(m, H * G, d)
    dev = [x.cuda() for x in (ctx_k, ctx_v, k, v, q)]
    turned, out = torch.zeros_like(dev[4]), torch.zeros_like(dev[4])
    append = lib.kvc_append_rotated_q8 if q8 else lib.kvc_append_rotated
    first = requests([base], [base], table=table if paged else None, max_kv=T)
    plain = kvc.Rotary(kvc.Rope(1e4))
    assert append(first._at, plain._for(d), None, None, ref(heads(dev[0])), ref(heads(dev[1])), layer, ref(c.struct), None) == 0
    assert append(req._at, rot._for(d), ref(heads(dev[4])), ref(heads(turned)), ref(heads(dev[2])), ref(heads(dev[3])), layer, ref(c.struct), None) == 0
    n = lib.kvc_attend_workspace_bytes(req._at, H * G, H, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    attend = lib.kvc_attend_tree_q8 if q8 else lib.kvc_attend_tree
    assert attend(req._at, tree._at, ref(heads(turned)), ref(c.struct), layer, d ** -0.5, ref(heads(out)), None, ws.data_ptr(), n, None) == 0
    torch.cuda.synchronize()
    freq = [1e4 ** (-2.0 * i / d) for i in range(d // 2)]
    seen, depth = orc.tree_rows(parents[0])
    # 8 bits: half a step of e4m3, or half of its least step at a row's scale (values below 8, scale 2^-5 at most: 2^-15)
    for j in range(m):
        want, size = orc.rotate(f64(k[j]), base + depth[j], freq, d, False)
        got = c.value(0, *where(base + j))
        tol = (2.0 ** -4 * np.abs(want) + 2.0 ** -15 if q8 else 2.0 ** -8 * np.abs(want)) + 2.0 ** -20 * size + 2.0 ** -133
        assert np.all(np.abs(got - want) <= tol)
    keys = {t: (c.value(0, *where(t)), c.value(1, *where(t))) for t in range(base + m)}
    for j in (0, 5, 8):
        ts = list(range(base)) + [base + a for a in sorted(seen[j])]
        for a in (0, H * G - 1):
            kk, vv = np.stack([keys[t][0][a // G] for t in ts]), np.stack([keys[t][1][a // G] for t in ts])
            want, _, absv, big = aorc.attend_row(f64(turned[j, a]), kk, vv, d ** -0.5)
            ds = d ** -0.5 * ((d + 8) * 2.0 ** -24 * big + 2.0 ** -10 * np.abs(f64(turned[j, a])).max() / 224.0 * np.abs(kk).sum(-1).max())
            assert np.all(np.abs(f64(out[j, a]) - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * (2.0 ** -8 + 2 * ds + 2.0 ** -17) * absv + 2.0 ** -23 * np.abs(vv).sum(0))
    kept = torch.tensor([[0, 2, 5] + [-1] * (m - 3)], dtype=I32, device="cuda")
    n_kept, kv_out = torch.tensor([3], dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    keep = lib.kvc_keep_q8 if q8 else lib.kvc_keep
    assert keep(req._at, kept.data_ptr(), m, n_kept.data_ptr(), ref(c.struct), kv_out.data_ptr(), None) == 0
    torch.cuda.synchronize()
    for j, a in enumerate((0, 2, 5)):
        for w in (0, 1):
            assert np.array_equal(c.value(w, *where(base + j)), keys[base + a][w])
    assert int(kv_out) == base + 3 and kvc.kvc_status_poll() == 0
    c.gaps_untouched()
    other = c.view[0][0]
    assert (other == c.fill).all(), "the other layer"
