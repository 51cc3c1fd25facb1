"""Tree attention over 8-bit caches whose value rows differ in scale: between tiles, inside a tile, out of float16's reach."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Step, f64
from draft_helpers import TreeBuilt
from oracle import attend_oracle as aorc

pytestmark = pytest.mark.gpu

LOW, HIGH = 112, 126        # biased scale exponents of rows whose values float16 holds exactly and small enough


def shifts(pattern, kv, rng):
    """What is added to the scale exponents of a request's value rows (those of normal numbers: about 119 and 120)."""
    t = np.arange(kv)
    return {"none": lambda: np.zeros(kv, int), "small": lambda: np.full(kv, -30), "large": lambda: np.full(kv, 30),
            "blocks": lambda: np.array([0, 12, -25, 0, 0, 0, 40, 0])[(t // 32) % 8],          # 32 keys each
            "edges": lambda: rng.choice([-9, -8, -7, 5, 6, 7, 8], kv),
            "one": lambda: np.where(t % 97 == 5, 9, 0),
            "rising": lambda: (60 * t // max(kv, 1)) - 30}[pattern]()


def scaled(st, pattern, kind="tree"):
    b = TreeBuilt(st, kind=kind)
    rng = np.random.default_rng(st.seed + 1)
    e = b.cache.scale_v.cpu().numpy()                                 # [L, P, H, page]
    b.in_reach = []
    for i, kv in enumerate(st.kv):
        by, rows = shifts(pattern, kv, rng), np.zeros((kv, st.H), bool)
        for t in range(kv):
            at = (st.layer, int(b.req.page_table[i, t // st.page]), slice(None), t % st.page)
            e[at] += by[t].astype(e.dtype) if by[t] >= 0 else 0
            e[at] -= (-by[t]).astype(e.dtype) if by[t] < 0 else 0
            rows[t] = (e[at] >= LOW) & (e[at] <= HIGH)
        b.val_v[i] = b.val_v[i] * np.exp2(by.astype(np.float64))[:, None, None]
        b.in_reach.append(rows)
    b.cache.scale_v.copy_(torch.from_numpy(e))
    return b


def check(b, out):
    """Against float64.  Probabilities meet values as bf16 (2^-8 of a term, with the running maximum's rounding counted as
    in TreeBuilt.check_tree) or, where the rows' scales are in reach, as float16: 2^-11 of a term, or half a subnormal step,
    2^-25 of what stands for 1, which is below twice the sum; once more where a maximum grows: 2^-23 of the value."""
    st, o = b.st, f64(out)
    for i in range(len(st.nq)):
        first = st.kv[i] - st.nq[i]
        for j in range(st.nq[i]):
            keys = list(range(first)) + [first + a for a in sorted(b.seen[i][j])]
            for a in range(0, st.H * st.G, 3):
                h, qr = a // st.G, f64(b.q_cpu[int(b.begin[i]) + j, a])
                k, v = b.val_k[i][keys, h], b.val_v[i][keys, h]
                ref, _, absv, big = aorc.attend_row(qr, k, v, b.scale)
                ds = b.scale * ((st.d + 8) * 2.0 ** -24 * big + 2.0 ** -10 * np.abs(qr).max() / 224.0 * np.abs(k).sum(-1).max())
                rel = 2.0 ** -8 + 2 * ds + len(keys) * 2.0 ** -23 + 2.0 ** -21
                reach = b.in_reach[i][keys, h][:, None]
                tol = 2.0 ** -8 * np.abs(ref) + 1.01 * rel * absv + 2.0 ** -23 * (np.abs(v) * reach).sum(0) + 1e-38
                err = np.abs(o[int(b.begin[i]) + j, a] - ref)
                assert np.all(err <= tol), (i, j, a, float((err / tol).max()))


@pytest.mark.parametrize("pattern", ["none", "small", "large", "blocks", "edges", "one", "rising"])
@pytest.mark.parametrize("nq,kv,G,d", [([8], [500], 4, 128), ([9, 30], [700, 131], 4, 64), ([9], [1000], 8, 128)])
def test_value_scales(pattern, nq, kv, G, d):
    b = scaled(Step(nq, kv, H=2, G=G, d=d, q8=True, seed=len(pattern)), pattern)
    kvc.kvc_status_reset()
    out, _ = b.run_tree()
    assert kvc.kvc_status_poll() == 0
    check(b, out)


@pytest.mark.parametrize("pattern", ["none", "blocks", "edges"])
@pytest.mark.parametrize("ramp", [60.0, 400.0])
@pytest.mark.parametrize("m", [10, 30])
def test_growing_maxima_over_both_types(m, ramp, pattern):
    """Probabilities already written, of either type, are scaled when a later key's logit is far above."""
    b = scaled(Step([m], [700], G=4, q8=True, ramp=ramp, seed=m), pattern)
    check(b, b.run_tree()[0])


@pytest.mark.parametrize("m,kv", [(20, 148), (30, 158)])
def test_what_a_jump_leaves_of_a_probability(m, kv):
    """Logits, in powers of two: nothing; 7.2 in the second 32 keys (less than what makes the maximum follow); 26 in the
    third.  In one channel only the second part's key has a value: 2^-18.8 of it is the output, held to 2^-23."""
    st = Step([m], [kv], H=1, G=4, d=64, q8=True, seed=2)
    b = TreeBuilt(st, kind="chain")
    u = np.sign(np.random.default_rng(3).standard_normal(st.d))
    b.q_cpu = torch.from_numpy(np.broadcast_to(u, b.q_cpu.shape).copy()).to(torch.bfloat16)
    b.q.copy_(b.q_cpu)
    k, v = np.zeros((kv, st.d)), b.val_v[0][:, 0].copy()
    k[40], k[70] = 0.625 * u, 2.25 * u
    v[:, 0] = 0.0
    v[40, 0] = 1.0
    for x, code, exp, val in ((k, b.cache.k, b.cache.scale_k, b.val_k), (v, b.cache.v, b.cache.scale_v, b.val_v)):
        c, e = aorc.quantize_rows(x)
        val[0] = aorc.dequantize_rows(c, e)[:, None]
        for t in range(kv):
            p, at = int(b.req.page_table[0, t // st.page]), t % st.page
            code.view(torch.uint8)[0, p, 0, at] = torch.from_numpy(c[t])
            exp[0, p, 0, at] = int(e[t])
    b.in_reach = [np.ones((kv, 1), bool)]
    out, _ = b.run_tree()
    assert np.all(f64(out)[:, :, 0] > 2.0 ** -19)
    check(b, out)


@pytest.mark.parametrize("m", [10, 30])
def test_values_that_are_no_numbers(m):
    """A NaN code, or a NaN scale, in a key that everybody sees: its channel, or all of them, and nothing of the others."""
    for what in ("code", "scale"):
        st = Step([m], [300], H=2, G=4, q8=True, seed=m)
        b = TreeBuilt(st)
        clean, _ = b.run_tree()
        p, s = int(b.req.page_table[0, 70 // st.page]), 70 % st.page
        if what == "code":
            b.cache.v.view(torch.uint8)[0, p, 1, s, 5] = 0xFF
        else:
            b.cache.scale_v[0, p, 1, s] = 255
        out, _ = b.run_tree()
        nan = torch.isnan(out.float())
        want = torch.zeros_like(nan)
        want[:, st.G:, 5 if what == "code" else slice(None)] = True
        assert torch.equal(nan, want)
        # the other head's numbers are those of the clean run; the row's 32 keys may have changed type in the NaN's head
        assert torch.equal(out[:, : st.G], clean[:, : st.G])
