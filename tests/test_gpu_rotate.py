"""kvc_append_rotated against float64: positions, pairings, parts of heads, scaled frequencies, bf16 and 8-bit caches."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import f64
from draft_helpers import I32, requests, row_of, shuffled_table
from oracle import attend_oracle as aorc
from oracle import draft_oracle as orc

pytestmark = pytest.mark.gpu


def pool(P, page, H, d, L, q8, tm, dev="cuda"):
    shape = (L, P, page, H, d) if tm else (L, P, H, page, d)
    if not q8:
        return kvc.Cache.pool(*(torch.full(shape, 7.0, dtype=torch.bfloat16, device=dev) for _ in range(2)), token_major=tm)
    code = lambda: torch.full(shape, 0x2A, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
    return kvc.QCache.pool(code(), code(), *(torch.full(shape[:-1], 0x2B, dtype=torch.uint8, device=dev) for _ in range(2)), token_major=tm)


def check_rows(got, ref, size, what):
    """bf16 rows.  Before any run: the output's rounding 2^-8 |ref|; cos and sin from an angle of at most half a turn in
    float32 (its rounding moves them by pi 2^-25), the functions' own error (2^-23) and the amplitude's rounding: 3 2^-23
    together; two products and a sum of float32 add 2^-22: less than 2^-21 of a (|x| + |y|) in all."""
    tol = 2.0 ** -8 * np.abs(ref) + 1.01 * 2.0 ** -21 * size + 2.0 ** -133
    err = np.abs(got - ref)
    assert np.all(err <= tol), (what, float((err / tol).max()))


def check_codes(code, e, ref, size, what):
    """8-bit rows: the exponent is the smallest that holds the row's maximum, as far as float32 can tell; values are off by
    half a step (2^-4 of the value, or 2^-10 of the scale) and by what the float32 products are off before."""
    val = aorc.dequantize_rows(code, e)
    delta = 1.01 * 2.0 ** -21 * size
    scale = np.ldexp(1.0, e.astype(np.int64) - 127)
    top, slack = np.abs(ref).max(-1), delta.max(-1)
    assert np.all(top <= 448 * scale + slack) and np.all((top >= 224 * scale - slack) | (e == 0)), what
    tol = np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * scale[..., None]) + 1.07 * delta
    err = np.abs(val - ref)
    assert np.all(err <= tol), (what, float((err / tol).max()))


CASES = [
    # nq, kv, H, Hq, d, page, q8, token-major, rot, interleaved, theta, amplitude, far, depths
    ([1], [1], 1, 1, 64, 8, False, False, 64, False, 1e4, 1.0, 0, False),
    ([1, 1, 1], [1, 17, 300], 2, 8, 128, 16, False, False, 128, False, 5e5, 1.0, 0, False),
    ([1, 1, 1], [5, 16, 301], 8, 32, 128, 16, True, False, 128, False, 5e5, 1.0, 0, False),
    ([5, 0, 33], [40, 9, 33], 2, 2, 64, 32, False, True, 32, True, 1e4, 1.0, 0, True),
    ([7, 13], [100, 13], 3, 21, 128, 16, True, True, 64, False, 1e6, 1.2, 0, True),
    ([3, 40], [3, 77], 4, 4, 128, 64, True, False, 16, True, 1e4, 0.7, 1000000, True),
    ([130], [200], 1, 7, 64, 128, False, False, 48, False, 1e4, 1.0, 100000000, False),
    ([9], [9], 8, 64, 128, 16, False, False, 128, True, 5e5, 1.0, -500, False),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_against_float64(case):
    nq, kv, H, Hq, d, page, q8, tm, rot, inter, theta, amp, far, trees = case
    g = torch.Generator().manual_seed(sum(kv) + d)
    rows, spare, L, layer = sum(nq), 2, 2, 1
    table, P = shuffled_table(kv, page, 5)
    req = requests(nq, kv, table=table)
    rnd = lambda h: torch.randn(rows + spare, h, d, generator=g).to(torch.bfloat16)
    q, k, v = rnd(Hq), rnd(H) * 10, rnd(H)
    depth = torch.randint(0, 30, (rows + spare,), generator=g, dtype=I32) if trees else None
    begin = torch.tensor([far - 3 * b for b in range(len(nq))], dtype=I32) if far else None
    f = kvc.scaled_frequencies(theta, rot, 4.0, original=4096) if amp != 1.0 else kvc.scaled_frequencies(theta, rot)
    rope = kvc.Rope(theta, kvc.KVC_ROPE_INTERLEAVED if inter else kvc.KVC_ROPE_HALF, inv_freq=f if amp != 1.0 else None)
    dev = lambda t: None if t is None else t.cuda()
    rotary = kvc.Rotary(rope, rot_dim=rot, amplitude=amp, depth=dev(depth), pos_begin=dev(begin))
    cache, out = pool(P, page, H, d, L, q8, tm), torch.full((rows + spare, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kvc.kvc_status_reset()
    kvc.kvc_append_rotated(req, rotary, k.cuda(), v.cuda(), cache, layer, q=q.cuda(), q_out=out)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == 0
    f = [float(theta) ** (-2.0 * i / rot) for i in range(rot // 2)] if amp == 1.0 else f
    written = torch.zeros(cache.k.shape[:-1], dtype=torch.bool)
    r = 0
    for b, m in enumerate(nq):
        for j in range(m):
            pos = (int(begin[b]) if far else 0) + kv[b] - m + (int(depth[r]) if trees else j)
            ref, size = orc.rotate(f64(q[r]), pos, f, rot, inter, amp)
            check_rows(f64(out[r]), ref, size, ("q", b, j))
            assert torch.equal(out[r, :, rot:].cpu(), q[r, :, rot:])
            t = kv[b] - m + j
            p, s = int(table[b, t // page]), t % page
            written[(layer, p, s) if tm else (layer, p, slice(None), s)] = True
            ref, size = orc.rotate(f64(k[r]), pos, f, rot, inter, amp)
            here = lambda name: row_of(cache, name, table, b, t, layer).cpu()
            if q8:
                check_codes(here("k").view(torch.uint8).numpy(), here("scale_k").numpy(), ref, size, ("k", b, j))
                code, e = aorc.quantize_rows(f64(v[r]))
                assert np.array_equal(here("v").view(torch.uint8).numpy(), code) and np.array_equal(here("scale_v").numpy(), e)
            else:
                check_rows(f64(here("k")), ref, size, ("k", b, j))
                assert torch.equal(here("v"), v[r])
            r += 1
    assert (out[rows:] == 7.0).all()
    for x, was in ((cache.k, 0x2A if q8 else 7.0), (cache.v, 0x2A if q8 else 7.0)) + (((cache.scale_k, 0x2B), (cache.scale_v, 0x2B)) if q8 else ()):
        x = (x.view(torch.uint8) if x.element_size() == 1 else x).cpu()
        assert (x[~written] == was).all(), "other rows are left"


def test_slices_of_one_projection_in_place():
    """q, k and v side by side in one row; the queries are rotated where they lie."""
    nq, kv, H, Hq, d, page = [9, 4], [30, 4], 2, 6, 128, 16
    table, P = shuffled_table(kv, page, 1)
    req = requests(nq, kv, table=table)
    fused = torch.randn(13, Hq + 2 * H, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    was = fused.clone()
    rotary = kvc.Rotary(kvc.Rope(1e4))
    a, b = pool(P, page, H, d, 1, False, False), pool(P, page, H, d, 1, False, False)
    apart = torch.empty(13, Hq, d, dtype=torch.bfloat16, device="cuda")
    kvc.kvc_append_rotated(req, rotary, was[:, Hq: Hq + H].contiguous(), was[:, Hq + H:].contiguous(), a, 0, q=was[:, :Hq].contiguous(), q_out=apart)
    kvc.kvc_append_rotated(req, rotary, fused[:, Hq: Hq + H], fused[:, Hq + H:], b, 0, q=fused[:, :Hq], q_out=fused[:, :Hq])
    torch.cuda.synchronize()
    assert torch.equal(fused[:, :Hq], apart) and torch.equal(fused[:, Hq:], was[:, Hq:])
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    kvc.kvc_append_rotated(req, rotary, was[:, Hq: Hq + H], was[:, Hq + H:], b, 0)              # keys alone
    assert torch.equal(a.k, b.k)


def test_contiguous_rows_and_long_strides():
    """One request over contiguous rows (token-major), query heads as the outer axis."""
    H, d, T, m = 2, 64, 50, 20
    g = torch.Generator().manual_seed(8)
    c = kvc.Cache(*(torch.full((1, T, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)), token_major=True)
    req = requests([m], [45])
    k, v = (torch.randn(m, H, d, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q = torch.randn(5, m, d, generator=g).to(torch.bfloat16).cuda().transpose(0, 1)
    out = torch.zeros(5, m, d, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    kvc.kvc_append_rotated(req, kvc.Rotary(kvc.Rope(1e4)), k, v, c, 0, q=q, q_out=out)
    torch.cuda.synchronize()
    f = [1e4 ** (-2.0 * i / d) for i in range(d // 2)]
    for j in range(m):
        ref, size = orc.rotate(f64(q[j]), 25 + j, f, d, False)
        check_rows(f64(out[j]), ref, size, j)
        ref, size = orc.rotate(f64(k[j]), 25 + j, f, d, False)
        check_rows(f64(c.k[0, 25 + j]), ref, size, j)
    assert (c.k[0, :25] == 7.0).all() and (c.k[0, 45:] == 7.0).all()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_no_rotation_is_append(q8):
    """At positions 0 the cache is kvc_append's, bit for bit."""
    nq, kv, H, d, page = [6, 3], [6, 3], 4, 128, 16
    table, P = shuffled_table(kv, page, 2)
    req = requests(nq, kv, table=table)
    k, v = (torch.randn(9, H, d, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in (1, 2))
    a, b = pool(P, page, H, d, 1, q8, False), pool(P, page, H, d, 1, q8, False)
    kvc.kvc_append(req, k, v, a, 0)
    kvc.kvc_append_rotated(req, kvc.Rotary(kvc.Rope(1e4), depth=torch.zeros(9, dtype=I32, device="cuda")), k, v, b, 0)
    torch.cuda.synchronize()
    for name in ("k", "v") + (("scale_k", "scale_v") if q8 else ()):
        x, y = getattr(a, name), getattr(b, name)
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)) if q8 else torch.equal(x, y)


def test_agrees_with_realignment():
    """Keys written at positions p and re-aligned by s are the keys written at p + s, but for two roundings to bf16 and what
    the first one carries through the rotation: 2^-8 of both channels of a pair, once more 2^-8 of the result, 2^-20 in all
    for the float32 angles."""
    H, d, T, s = 2, 128, 64, 777
    k, v = (torch.randn(T, H, d, generator=torch.Generator().manual_seed(x)).to(torch.bfloat16).cuda() for x in (1, 2))
    mk = lambda: kvc.Cache(*(torch.zeros(1, H, T, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    req, rope = requests([T], [T]), kvc.Rope(5e5)
    a, b, moved = mk(), mk(), mk()
    kvc.kvc_append_rotated(req, kvc.Rotary(rope), k, v, a, 0)
    kvc.kvc_append_rotated(req, kvc.Rotary(rope, pos_begin=torch.tensor([s], dtype=I32, device="cuda")), k, v, b, 0)
    kvc.kvc_apply(a, kvc.State.empty(), s, rope, moved)
    torch.cuda.synchronize()
    x = f64(k).transpose(1, 0, 2)
    size = np.abs(x[..., :64]) + np.abs(x[..., 64:])
    tol = (2 * 2.0 ** -8 + 2 * 2.0 ** -8 + 2.0 ** -20) * np.concatenate([size, size], -1)
    assert np.all(np.abs(f64(moved.k[0]) - f64(b.k[0])) <= tol) and torch.equal(moved.v, b.v)


def test_special_values_and_skipped_rows():
    """Infinities and NaN stay in their pairs; a negative position and a bad page skip the key, not the query."""
    H, d, page = 1, 64, 8
    table = torch.tensor([[0], [99], [1]], dtype=I32)
    req = requests([3, 1, 1], [1, 4, 4], table=table, max_kv=8)                    # request 0 begins at position -2
    k = torch.ones(5, H, d, dtype=torch.bfloat16)
    k[4, 0, 5], k[4, 0, 40] = float("inf"), float("nan")
    q = k.clone().cuda()
    for q8 in (False, True):
        c, out = pool(2, page, H, d, 1, q8, False), torch.zeros_like(q)
        kvc.kvc_status_reset()
        kvc.kvc_append_rotated(req, kvc.Rotary(kvc.Rope(1e4)), k.cuda(), k.cuda(), c, 0, q=q, q_out=out)
        torch.cuda.synchronize()
        assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE | kvc.KVC_FLAG_BAD_LENGTH
        kvc.kvc_status_reset()
        bad = ~torch.isfinite(out.float())
        assert bad[4, 0].nonzero().flatten().tolist() == [5, 8, 37, 40] and not bad[:4].any() and (out[:4].float().abs().sum(-1) > 0).all()
        held = c.k.view(torch.uint8) if q8 else c.k
        untouched = (held == (0x2A if q8 else 7.0)).all(-1)[0, :, 0]               # [page, row]
        assert untouched.tolist() == [[False] + [True] * 7, [True] * 3 + [False] + [True] * 4]
        if q8:
            assert (c.k[0, 1, 0, 3].float().isnan().nonzero().flatten().tolist()) == [5, 8, 37, 40]
            ref = k.float()[4, 0].clone()
            assert torch.isfinite(c.v[0, 1, 0, 3].float()).sum() == 62 and int(c.scale_v[0, 1, 0, 3]) == int(c.scale_v[0, 0, 0, 0])
