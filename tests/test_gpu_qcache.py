"""8-bit caches on the GPU: kvc_quantize, kvc_dequantize and kvc_append against the float64 oracle, bit for bit; and the
operators together, as a serving program runs them."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step, f64
from helpers import bits_of
from oracle import attend_oracle as orc
from paper_2609_34060_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def _table(T, page, seed):
    n = -(-T // page)
    return torch.randperm(n + 3, generator=torch.Generator().manual_seed(seed))[:n].to(torch.int32), n + 3


def _cache(L, H, T, d, page, token_major, seed, special=False):
    g = torch.Generator().manual_seed(seed)
    if page:
        tab, P = _table(T, page, seed)
        shape = (L, P, page, H, d) if token_major else (L, P, H, page, d)
    else:
        tab, shape = None, ((L, T, H, d) if token_major else (L, H, T, d))
    x = [torch.randn(shape, generator=g) * torch.exp2(torch.randint(-12, 9, shape[:-1], generator=g).float())[..., None] for _ in range(2)]
    x = [t.to(torch.bfloat16) for t in x]
    if special:
        for t in x:
            f = t.view(-1, d)
            f[0] = 0
            f[1] = -0.0
            f[2, 3], f[2, 4], f[2, 5] = float("inf"), float("-inf"), float("nan")
            f[3] = 1e-38                                   # subnormal range of the scale
            f[4] = 3.3e38
            f[5] = 448.0 * 2.0 ** 3
            f[6] = 450.0
            f[7] = torch.tensor([17.0, 0.0087890625, -0.0107421875, 2.0 ** -10, 3 * 2.0 ** -10] * d)[:d] * 16   # ties and subnormal codes
            f[8] = float("nan")
    return kvc.Cache(x[0].cuda(), x[1].cuda(), T=T if page else None, page_table=None if tab is None else tab.cuda(), token_major=token_major)


def _rows(t, c):
    """[L, T, H, ...] in logical order of a cache tensor (codes, exponents or bf16)."""
    tail = t.dim() - 4 - (1 if c.page_table is not None else 0)          # 0: with channels, -1: exponents
    x = t if c.token_major else t.transpose(2, 3) if c.page_table is not None else t.transpose(1, 2)
    assert tail in (0, -1)
    if c.page_table is None:
        return x[:, : c.T]
    x = x[:, c.page_table.long()]
    return x.reshape(x.shape[0], -1, *x.shape[3:])[:, : c.T]


@pytest.mark.parametrize("L,H,T,d,page,tm,special", [
    (1, 1, 1, 64, 0, False, False), (2, 2, 300, 128, 0, False, True), (2, 3, 77, 64, 0, True, True), (3, 2, 131, 128, 16, False, True),
    (1, 4, 33, 64, 8, True, False), (2, 1, 513, 128, 64, False, False), (1, 2, 16, 128, 32, True, True)])
def test_quantize_and_back(L, H, T, d, page, tm, special):
    src = _cache(L, H, T, d, page, tm, seed=T, special=special)
    q = kvc.QCache.like(src)
    for t in (q.k, q.v):
        t.view(torch.uint8).fill_(0x2A)
    for t in (q.scale_k, q.scale_v):
        t.fill_(0x2B)
    kvc.kvc_status_reset()
    kvc.kvc_quantize(src, q)
    back = src.empty_like(fill=7.0)
    kvc.kvc_dequantize(q, back)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == 0
    for name in ("k", "v"):
        x = f64(_rows(getattr(src, name), src))
        code, e = orc.quantize_rows(x)
        got_c = _rows(getattr(q, name).view(torch.uint8), src).cpu().numpy()
        got_e = _rows(getattr(q, "scale_" + name), src).cpu().numpy()
        nan = (code & 127) == 127
        assert np.array_equal(got_e, e)
        assert np.array_equal(got_c[~nan], code[~nan]) and np.all((got_c[nan] & 127) == 127)
        want = torch.from_numpy(orc.dequantize_rows(code, e)).to(torch.bfloat16)
        got = _rows(getattr(back, name), src).cpu()
        same = (bits_of(got) == bits_of(want)) | torch.isnan(want).numpy()
        assert same.all() and torch.equal(torch.isnan(got), torch.isnan(want))
        # half a step of e4m3: 2^-4 of the value, or 2^-10 of the scale
        fin = np.isfinite(x)
        err = np.abs(f64(want) - np.where(fin, x, 0))[fin]
        step = np.broadcast_to(np.ldexp(1.0, e.astype(int) - 127)[..., None], x.shape)[fin]
        assert np.all(err <= np.maximum(2.0 ** -4 * np.abs(x[fin]), 2.0 ** -10 * step) + 2.0 ** -133)
        # what the call does not cover stays
        for t, fill in ((getattr(q, name).view(torch.uint8), 0x2A), (getattr(q, "scale_" + name), 0x2B)):
            if page:
                spare = [p for p in range(src.P) if p not in src.page_table.tolist()]
                assert (t[:, spare] == fill).all()
                if T % page:
                    last = int(src.page_table[-1])
                    assert ((t[:, last, T % page:] if tm else t[:, last, :, T % page:]) == fill).all()


def test_quantize_between_layouts():
    """A contiguous cache put away into pages and read back into token-major rows."""
    src = _cache(2, 2, 203, 128, 0, False, seed=5)
    tab, P = _table(203, 16, 9)
    z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    q = kvc.QCache(z(2, P, 2, 16, 128).view(torch.float8_e4m3fn), z(2, P, 2, 16, 128).view(torch.float8_e4m3fn), z(2, P, 2, 16), z(2, P, 2, 16),
                   T=203, page_table=tab.cuda())
    kvc.kvc_quantize(src, q)
    back = kvc.Cache(*(torch.zeros(2, 203, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)), token_major=True)
    kvc.kvc_dequantize(q, back)
    for a, b in ((src.k, back.k), (src.v, back.v)):
        want = torch.from_numpy(orc.dequantize_rows(*orc.quantize_rows(f64(a)))).to(torch.bfloat16)
        assert torch.equal(b.cpu().transpose(1, 2), want)


def test_bad_page_is_skipped_by_convert_and_append():
    src = _cache(1, 2, 64, 128, 16, False, seed=3)
    q = kvc.QCache.like(src)
    src.page_table[1] = 99
    kvc.kvc_status_reset()
    kvc.kvc_quantize(src, q)
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE
    kvc.kvc_status_reset()
    st = Built(Step([3, 2], [20, 18], page=16))
    before = st.cache.k.clone()
    st.req.page_table[0, 1] = -1
    new = torch.ones(5, 2, 128, dtype=torch.bfloat16, device="cuda")
    kvc.kvc_append(st.req, new, new, st.cache, 0)
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE
    kvc.kvc_status_reset()
    st.req.page_table[0, 1] = 0
    st.req.kv_len[0] = 2                                    # the first of three new tokens has no place
    kvc.kvc_append(st.req, new, new, st.cache, 0)
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_LENGTH
    kvc.kvc_status_reset()
    pg = st.req.page_table
    assert (st.cache.k[0, int(pg[0, 0]), :, :2] == 1).all() and (st.cache.k[0, int(pg[1, 1]), :, :2] == 1).all()
    assert torch.equal(st.cache.k[0, int(pg[0, 0]), :, 2:].nan_to_num(9), before[0, int(pg[0, 0]), :, 2:].nan_to_num(9))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("page,tm,d,L,layer", [(16, False, 128, 1, 0), (8, True, 64, 2, 1), (64, False, 64, 1, 0), (0, False, 128, 2, 1), (0, True, 64, 1, 0)])
def test_append(page, tm, d, L, layer, q8):
    nq, kv = ([33], [50]) if page == 0 else ([1, 0, 33, 7], [1, 5, 50, 40])
    st = Built(Step(nq, kv, H=3, d=d, page=page, token_major=tm, L=L, layer=layer, q8=q8))
    c = st.cache
    g = torch.Generator().manual_seed(4)
    rows = sum(nq) + 2
    fused = torch.randn(rows, 2, 3, d, generator=g).to(torch.bfloat16).cuda()
    kn, vn = fused[:, 0], fused[:, 1]                       # strided rows
    names = ("k", "v", "scale_k", "scale_v") if q8 else ("k", "v")
    byte = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16)
    want = {n: byte(getattr(c, n)).clone() for n in names}
    kvc.kvc_status_reset()
    kvc.kvc_append(st.req, kn, vn, c, layer)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == 0
    at = 0
    for b in range(len(nq)):
        for j in range(nq[b]):
            pos = kv[b] - nq[b] + j
            for name, src in (("k", kn), ("v", vn)):
                x = src[at + j]
                if q8:
                    code, e = orc.quantize_rows(f64(x))
                    put = {name: torch.from_numpy(code), "scale_" + name: torch.from_numpy(e)}
                else:
                    put = {name: x.view(torch.int16)}
                for n, val in put.items():
                    w = want[n][layer]
                    if page:
                        w, slot = w[int(st.req.page_table[b, pos // page])], pos % page
                    else:
                        slot = pos
                    if tm:
                        w[slot] = val.to(w.device)
                    else:
                        w[:, slot] = val.to(w.device)
        at += nq[b]
    for n in names:
        assert torch.equal(byte(getattr(c, n)), want[n]), n


def test_serving_step_after_a_correction():
    """The operators as a program uses them: agent 0's cache corrected for agent 1 (kvc_apply), put away in 8 bits, read
    back, agent 1's prompt and then single tokens appended and attended, over the bf16 pages and over the 8-bit ones."""
    cfg = wl.CONFIGS["llama8b_8k"].scaled(name="serve", L=2, H=2, T=150, n_agents=2)
    k0, v0 = wl.base_cache(cfg, "cuda")
    page, T, H, d, G, extra = 16, 150, 2, 128, 4, 60
    P = -(-(T + extra) // page) + 2
    tab = torch.randperm(P, generator=torch.Generator().manual_seed(1))[: -(-(T + extra) // page)].to(torch.int32).cuda()
    z = lambda: torch.zeros(2, P, H, page, d, dtype=torch.bfloat16, device="cuda")
    pool_k, pool_v = z(), z()
    st = kvc.State(*(wl.hop_state(cfg, 1, "cuda")[x] for x in ("coeff_k", "coeff_v", "basis_k", "basis_v")))
    dst = kvc.Cache(pool_k, pool_v, T=T, page_table=tab)
    kvc.kvc_apply(kvc.Cache(k0, v0), st, 17, kvc.Rope(cfg.theta), dst)
    q8 = kvc.QCache.like(dst)
    kvc.kvc_quantize(dst, q8)
    read = kvc.Cache(z(), z(), T=T, page_table=tab)
    kvc.kvc_dequantize(q8, read)
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    caches = {"bf16": kvc.Cache.pool(pool_k, pool_v), "q8": kvc.QCache.pool(q8.k, q8.v, q8.scale_k, q8.scale_v),
              "read": kvc.Cache.pool(read.k, read.v)}
    hist = {c: [[x[l, tab.long()].transpose(1, 2).reshape(-1, H, d)[:T] for x in kv] for l in range(2)]
            for c, kv in (("bf16", (pool_k, pool_v)), ("read", (read.k, read.v)))}
    length = T
    for step, nq in enumerate((37, 1, 1, 5)):
        length += nq
        req = kvc.Requests(torch.tensor([0, nq], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda"),
                           nq, length, page_table=tab[None])
        for layer in range(2):
            kn, vn, q = rnd(nq, H, d), rnd(nq, H, d), rnd(nq, H * G, d)
            outs = {}
            for c, cache in caches.items():
                if c == "read":                             # the same values as the 8-bit pages hold
                    both = [torch.from_numpy(orc.dequantize_rows(*orc.quantize_rows(f64(x)))).to(torch.bfloat16).cuda() for x in (kn, vn)]
                else:
                    both = [kn, vn]
                kvc.kvc_append(req, *both, cache, layer)
                if c in hist:
                    hist[c][layer] = [torch.cat([a, b]) for a, b in zip(hist[c][layer], both)]
                out = torch.zeros_like(q)
                ws = torch.empty(max(1, kvc.kvc_attend_workspace_bytes(req, cache, H * G)), dtype=torch.uint8, device="cuda")
                kvc.kvc_attend(req, q, cache, layer, out, ws)
                outs[c] = f64(out)
            for c in ("bf16", "read"):
                k, v = (f64(x) for x in hist[c][layer])
                for j in range(nq):
                    for a in range(H * G):
                        ref, _, absv, _ = orc.attend_row(f64(q[j, a]), k[: length - nq + j + 1, a // G], v[: length - nq + j + 1, a // G], d ** -0.5)
                        # output and probabilities to bf16, as in attend_helpers, logits' share 2^-12 at these magnitudes
                        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -12) * absv + 1e-30
                        for name in (("bf16",) if c == "bf16" else ("read", "q8")):
                            extra_tol = 2.0 ** -23 * np.abs(v[:, a // G]).sum(0) if name == "q8" else 0.0
                            assert np.all(np.abs(outs[name][j, a] - ref) <= tol + extra_tol), (step, layer, name, j, a)
    assert kvc.kvc_status_poll() == 0
