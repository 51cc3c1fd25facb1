"""Tree attention over 8-bit caches where a single key has nearly all the weight and next to no value: the answer is made by
thousands of keys whose probabilities lie some twenty-five powers of two below."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Step, f64
from draft_helpers import TreeBuilt
from oracle import attend_oracle as aorc

pytestmark = pytest.mark.gpu


def put(b, name, rows):
    """Rows [kv, d] (quantised here) as request 0's keys or values, the same in every head; what they read as."""
    st = b.st
    codes, exps = aorc.quantize_rows(rows)
    code, exp = getattr(b.cache, name), getattr(b.cache, "scale_" + name)
    page = b.req.page_table[0].cpu().numpy().astype(np.int64)[np.arange(st.kv[0]) // st.page]
    at, row = torch.from_numpy(page).cuda(), torch.arange(st.kv[0], device="cuda") % st.page
    for h in range(st.H):
        code.view(torch.uint8)[0, at, h, row] = torch.from_numpy(codes).cuda()
        exp[0, at, h, row] = torch.from_numpy(exps).cuda()
    return aorc.dequantize_rows(codes, exps), exps


@pytest.mark.parametrize("m,G,d", [(5, 4, 128), (7, 8, 128), (25, 4, 64), (6, 2, 128), (40, 4, 128)])
@pytest.mark.parametrize("kv,place", [(8000, 0), (12000, 11900), (700, 3)])
@pytest.mark.parametrize("gap", [20.0, 24.6, 25.2, 40.0])
def test_a_flat_tail_below_one_key(m, G, d, kv, place, gap):
    """One key whose value is zero but for one channel (2^-6 there: its scale is 2^-15), all others gap powers of two below it
    with values of one sign around 1.

    Queries are ones (signs), keys whole numbers of up to four bits times a power of two (exact in codes): the logits of
    the tensor cores are exact.  Rounding, before any run: the output 2^-8 |ref|; probabilities 2^-8 of each term (an 8-bit
    call of at most 16 or more than 128 rows is closer, or the same); float32 sums of n terms n 2^-24, in the numerator and
    in the denominator; scale, exponent and exponential 2^-15 together (|logit| <= 64 in powers of two, c off by 2^-23)."""
    st = Step([m], [kv], H=1, G=G, d=d, q8=True, seed=m)
    b = TreeBuilt(st, kind="chain")
    rng = np.random.default_rng(int(gap * 10) + kv)
    u = np.sign(rng.standard_normal(d))
    b.q.copy_(torch.from_numpy(np.broadcast_to(u, b.q.shape).copy()).to(torch.bfloat16))
    down = (gap - 12.0) * (1.0 + 0.03 * rng.standard_normal((kv, 1)))             # of a key: the mean of its channels
    step = 2.0 ** (np.floor(np.log2(gap - 12.0)) - 3)
    k = -step * np.floor(down / step + rng.random((kv, d))) * u
    k[place] = 12.0 * u
    v = rng.uniform(0.5, 2.0, (kv, d))
    v[place] = 0.0
    v[place, 0] = 0.0136
    k, _ = put(b, "k", k)
    v, ev = put(b, "v", v)
    assert ev[place] == 112 and 119 <= np.delete(ev, place).min() and ev.max() <= 121
    out = torch.zeros(b.q.shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(b.q.shape[:2], device="cuda")
    scale = np.log(2.0) / d
    kvc.kvc_status_reset()
    kvc.kvc_attend_tree(b.req, b.tree, b.q, b.cache, 0, out, b.workspace(), scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == 0
    o, s = f64(out), lse.cpu().numpy().astype(np.float64)
    for j in (0, m // 2, m - 1):
        n = kv - m + j + 1
        ref, l, absv, _ = aorc.attend_row(u, k[:n], v[:n], scale)
        tol = 2.0 ** -8 * np.abs(ref) + 1.01 * (2.0 ** -8 + n * 2.0 ** -23 + 2.0 ** -15) * absv
        if m * G <= 16:                       # the few-rows kernel: a product of probability and scale is held to 2^-24 of the largest
            tol = tol + 2.0 ** -24 * np.exp2(ev[place] - 127.0) * 448.0 * n
        for a in range(G):
            err = np.abs(o[j, a] - ref)
            assert np.all(err <= tol), (j, a, float((err / tol).max()), float((err / np.abs(ref)).max()))
            assert abs(s[j, a] - l) <= 2.0 ** -14 + n * 2.0 ** -23
