"""Drafted tokens where offsets pass 32 bits, at far strides, and with values that are no numbers."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Step, f64
from draft_helpers import I32, TreeBuilt, flat, requests
from oracle import attend_oracle as aorc
from oracle import draft_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_pages_behind_two_billion_elements(q8):
    """A pool of 140000 pages (2.3e9 elements), drafts in its last ones: append, attention of the drafts alone, move."""
    P, H, page, d, m, G = 140000, 8, 16, 128, 12, 2
    if q8:
        c = kvc.QCache.pool(*(torch.zeros(1, P, H, page, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)),
                            *(torch.zeros(1, P, H, page, dtype=torch.uint8, device="cuda") for _ in range(2)))
    else:
        c = kvc.Cache.pool(*(torch.zeros(1, P, H, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table = torch.tensor([[P - 1, 0], [P - 3, P - 2]], dtype=I32)
    nq, kv = [m, 5], [m, 20]
    req = requests(nq, kv, table=table)
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)
    k, v, q = rnd(17, H, d), rnd(17, H, d), rnd(17, H * G, d)
    parents = [[-1, 0, 0, 1, 1, 2, 3, 3, 5, 6, 8, 9], [-1, 0, 1, 0, 2]]
    tree = kvc.Tree(flat(parents).cuda(), m)
    kvc.kvc_status_reset()
    kvc.kvc_tree_build(req, tree)
    kvc.kvc_append_rotated(req, kvc.Rotary(kvc.Rope(1e4), depth=torch.zeros(17, dtype=I32, device="cuda"), pos_begin=torch.tensor([0, -15], dtype=I32, device="cuda")),
                           k.cuda(), v.cuda(), c, 0)                         # every position is 0: keys as they are
    out = torch.zeros(17, H * G, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(kvc.kvc_attend_workspace_bytes(req, c, H * G), dtype=torch.uint8, device="cuda")
    kvc.kvc_attend_tree(req, tree, q.cuda(), c, 0, out, ws)
    kept = torch.tensor([[0, 2, 5, 8] + [-1] * 8, [0, 3] + [-1] * 10], dtype=I32, device="cuda")
    kvc.kvc_keep(req, kept, torch.tensor([4, 2], dtype=I32, device="cuda"), c)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == 0
    seen = orc.tree_rows(parents[0])[0]
    val = (lambda x: aorc.dequantize_rows(*aorc.quantize_rows(f64(x)))) if q8 else f64
    for j in (0, 7, 11):
        keys = sorted(seen[j])
        for a in (0, H * G - 1):
            ref, _, absv, big = aorc.attend_row(f64(q[j, a]), val(k)[keys, a // G], val(v)[keys, a // G], d ** -0.5)
            # roundings of outputs and probabilities 2^-8 each; logits as in draft_helpers
            ds = d ** -0.5 * ((d + 8) * 2.0 ** -24 * big + 2.0 ** -10 * np.abs(f64(q[j, a])).max() / 224.0 * np.abs(val(k)[keys, a // G]).sum(-1).max())
            assert np.all(np.abs(f64(out[j, a]) - ref) <= 2.0 ** -8 * np.abs(ref) + 1.01 * (2.0 ** -8 + 2 * ds + 2.0 ** -19) * absv + 2.0 ** -23 * np.abs(val(v)[keys, a // G]).sum(0))
    held = (lambda x, e: aorc.dequantize_rows(x.view(torch.uint8).cpu().numpy(), e.cpu().numpy())) if q8 else (lambda x, e: f64(x))
    for name, new in (("k", k), ("v", v)):
        e = getattr(c, "scale_" + name) if q8 else getattr(c, name)
        x = getattr(c, name)
        assert np.array_equal(held(x[0, P - 1, :, :4], e[0, P - 1, :, :4]), val(new[[0, 2, 5, 8]]).transpose(1, 0, 2))
        assert np.array_equal(held(x[0, P - 3, :, 15], e[0, P - 3, :, 15]), val(new[12])) and np.array_equal(held(x[0, P - 2, :, 0], e[0, P - 2, :, 0]), val(new[15]))


def test_distributions_behind_two_billion_entries():
    """The rows of the one request are the last of 17000 by 131072."""
    V, rows, m = 131072, 17000, 6
    target = torch.zeros(rows, V, device="cuda")
    g = torch.Generator().manual_seed(3)
    p = torch.softmax(torch.randn(m, V, generator=g) * 3, -1)
    target[-m:] = p.cuda()
    parents, token, u = [-1, 0, 0, 2, 2, 4], [0, 5, int(p[0].argmax()), 9, int(p[2].argmax()), 77], [0.0, 0.9, 0.0, 0.9, 0.0, 0.9]
    req = kvc.Requests(torch.tensor([rows - m, rows], dtype=I32, device="cuda"), torch.tensor([m], dtype=I32, device="cuda"), m, m)
    full = lambda x, t: torch.cat([torch.zeros(rows - m, dtype=t), torch.tensor(x, dtype=t)]).cuda()
    kept, n_kept, nxt = torch.zeros(1, m, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    kvc.kvc_verify(req, full(parents, I32), full(token, I32), target, full(u, torch.float32), torch.tensor([0.6], device="cuda"), kept, n_kept, nxt)
    torch.cuda.synchronize()
    want = orc.verify(parents, token, p.double().numpy(), None, [float(np.float32(x)) for x in u], float(np.float32(0.6)))
    assert want[0] == [0, 2, 4] and (kept[0, : int(n_kept)].tolist(), int(nxt)) == want


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("m,G", [(4, 4), (10, 4), (25, 4), (60, 4)])
def test_queries_and_keys_that_are_no_numbers(m, G, q8):
    """A NaN or infinite query makes its own row NaN and no other; a key of the context that is NaN, every row."""
    b = TreeBuilt(Step([m, 3], [300, 150], G=G, q8=q8, seed=5))
    clean, _ = b.run_tree()
    b.q[2, 1, 7], b.q[m - 1, 2, 0] = float("nan"), float("inf")
    out, lse = b.run_tree()
    odd = [(2, 1), (m - 1, 2)]
    same = torch.ones(out.shape[:2], dtype=torch.bool)
    for r, a in odd:
        assert out[r, a].isnan().all() and not torch.isfinite(lse[r, a])
        same[r, a] = False
    assert torch.equal(out[same.cuda()], clean[same.cuda()])
    b = TreeBuilt(Step([m, 3], [300, 150], G=G, q8=q8, seed=5))
    p, s = int(b.req.page_table[0, 3]), 5                                       # key 53 of request 0
    if q8:
        b.cache.scale_k[0, p, :, s] = 255
    else:
        b.cache.k[0, p, :, s, 3] = float("nan")
    out, _ = b.run_tree()
    assert out[:m].isnan().all() and torch.equal(out[m:], clean[m:])
