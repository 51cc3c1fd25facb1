"""Attention over 8-bit caches whose value rows differ by many powers of two."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_given import Given
from attend_helpers import Built, Step, f64
from oracle import attend_oracle as orc

pytestmark = pytest.mark.gpu

PATTERNS = ["rising", "falling", "random", "unlikely_giant", "hidden_giant", "zeros", "giant_first"]


def scales(pattern, T, g):
    """log2 of a value row's size, by token."""
    t = torch.arange(T) / max(T - 1, 1)
    if pattern == "rising":
        return 40 * t - 20
    if pattern == "falling":
        return 20 - 40 * t
    if pattern == "random":
        return 40 * torch.rand(T, generator=g) - 20
    x = torch.zeros(T)
    if pattern == "unlikely_giant":
        x[T // 3] = 30
    if pattern == "hidden_giant":
        x[T - 1] = 30
    if pattern == "giant_first":
        x[0] = 60
    return x


def build(pattern, T, rows, H, G, d, q8=True, causal=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    k, v, q = torch.randn(T, H, d, generator=g), torch.randn(T, H, d, generator=g), torch.randn(rows, H * G, d, generator=g)
    v = v * torch.exp2(scales(pattern, T, g).round())[:, None, None]
    if pattern == "zeros":                                     # half the value rows are nothing but zeros, at any probability
        v[::2] = 0
    giant = {"unlikely_giant": T // 3, "giant_first": 0}.get(pattern)
    if giant is not None:                                      # every query dislikes it: logits about -40 and -60
        u = torch.sign(torch.randn(d, generator=g))
        q = q + u
        k[giant] = -u * (40 if pattern == "unlikely_giant" else 60) / d ** 0.5
    return Given(k, v, q, q8=q8, causal=causal)


def check(b, out, lse):
    """Against float64, element by element.  Tolerances: as attend_helpers has them for the logits, sums, probabilities and
    the output; the few-rows kernel holds a probability times its value row's scale in three e4m3 parts, 2^-12 of it or,
    for small ones, half a step of the third: 2^-24 of the largest such product w of the row, times the code it meets."""
    st, o, s = b.st, f64(out), lse.cpu().numpy().astype(np.float64)
    for i, (nq, kv) in enumerate(zip(st.nq, st.kv)):
        for j in range(nq):
            r, end = int(b.begin[i]) + j, kv - nq + j + 1 if st.causal else kv
            for a in range(st.H * st.G):
                h = a // st.G
                q, k, v = f64(b.q_cpu[r, a]), b.val_k[i][:end, h], b.val_v[i][:end, h]
                ref, l, absv, big = orc.attend_row(q, k, v, b.scale)
                ds = (st.d + 8) * 2.0 ** -24 * b.scale * big
                rel = 2.0 ** -8 + 2 * ds + end * 2.0 ** -23 + 2.0 ** -21
                w = np.exp(b.scale * (k @ q) - l) * np.exp2(b.exp_v[i][:end, h].astype(np.float64))
                tol = 2.0 ** -8 * np.abs(ref) + 1.01 * rel * absv + 2.0 ** -24 * w.max() * np.abs(b.codes_v[i][:end, h]).sum(0) + 1e-38
                err = np.abs(o[r, a] - ref)
                assert np.all(err <= tol), (i, j, a, float((err / tol).max()), o[r, a][:4], ref[:4])
                assert abs(s[r, a] - l) <= ds + end * 2.0 ** -23 + 2.0 ** -20 + 2.0 ** -22 * abs(l)


@pytest.mark.parametrize("path", ["generic", "auto"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,rows,H,G", [(500, 1, 2, 4), (6000, 1, 1, 8), (700, 2, 2, 8), (3000, 3, 1, 4), (900, 4, 1, 8), (130, 5, 1, 1), (300, 60, 1, 2)])
@pytest.mark.parametrize("pattern", PATTERNS)
def test_spread_value_scales(pattern, T, rows, H, G, d, path):
    b = build(pattern, T, rows, H, G, d, seed=T + d)
    kvc.kvc_status_reset()
    kvc.kvc_set_path(kvc.KVC_PATH_GENERIC if path == "generic" else kvc.KVC_PATH_AUTO)
    try:
        out, lse = b.run()
    finally:
        kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
    check(b, out, lse)
    assert kvc.kvc_status_poll() == 0


@pytest.mark.parametrize("d,G", [(128, 4), (64, 16)])
def test_spread_value_scales_in_a_large_mixed_batch(d, G):
    """Single tokens beside chunks, a kernel each: every value row's exponent moved by up to 25 either way."""
    nq = [1] * 40 + [50]
    kv = [200 + 7 * i for i in range(40)] + [3500]
    b = Built(Step(nq=nq, kv=kv, H=2, G=G, d=d, q8=True, seed=9))
    rng, page = np.random.default_rng(4), b.st.page
    b.codes_v, b.exp_v = [], []
    sv = b.cache.scale_v.cpu()
    for i, n in enumerate(kv):
        code, e = orc.quantize_rows(f64(b.rows_v[i]))
        e = (e.astype(np.int64) + rng.integers(-25, 26, e.shape)).astype(np.uint8)       # [n, H]
        for t in range(n):
            sv[0, int(b.req.page_table[i, t // page]), :, t % page] = torch.from_numpy(e[t])
        b.val_v[i] = orc.dequantize_rows(code, e)
        b.codes_v.append(orc.dequantize_rows(code, np.full_like(e, 127)))
        b.exp_v.append(e.astype(np.int64) - 127)
    b.cache.scale_v.copy_(sv)
    check(b, *b.run())
