"""kvc_append_rotated by blocks of eight tokens (bounds that allow thousands): 8-bit caches, borders, odd head counts."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
import test_gpu_rotate as base
from draft_helpers import I32, requests, shuffled_table

pytestmark = pytest.mark.gpu

CASES = [
    # nq, kv, H, Hq, d, page, q8, token-major, rot, interleaved, theta, amplitude, far, depths
    ([64], [64], 1, 1, 128, 16, True, False, 128, False, 1e4, 1.0, 0, False),
    ([130, 64, 3, 0, 65], [300, 64, 90, 8, 70], 2, 6, 128, 16, True, False, 128, False, 5e5, 1.0, 0, False),
    ([71, 9], [100, 13], 3, 21, 64, 32, True, True, 32, True, 1e4, 1.0, 0, True),
    ([100, 1, 66], [150, 1, 67], 1, 5, 128, 128, True, True, 64, False, 1e6, 1.2, 1000000, True),
    ([67], [333], 4, 28, 128, 16, True, False, 16, True, 1e4, 0.7, -500, False),
    ([64, 63], [90, 63], 8, 64, 64, 8, True, False, 64, False, 5e5, 1.0, 0, True),
    ([65, 7], [80, 300], 3, 13, 64, 16, False, True, 64, True, 1e4, 1.0, 0, True),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
@pytest.mark.parametrize("loose", [False, True], ids=["one", "eight"])
def test_against_float64(case, loose, monkeypatch):
    if loose:
        monkeypatch.setattr(base, "requests", lambda nq, kv, **kw: requests(nq, kv, max_q=9000 // len(nq) + 3, **kw))
    base.test_against_float64(case)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_eight_tokens_a_block_and_one_agree(q8):
    """The bound decides how many tokens share a block, not what they become: the same bits, queries in place among them."""
    nq, kv, H, Hq, d, page = [37, 5, 63], [200, 5, 100], 2, 6, 128, 16
    table, P = shuffled_table(kv, page, 1)
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(sum(nq), Hq + 2 * H, d, generator=g).to(torch.bfloat16).cuda()
    depth = torch.randint(0, 20, (sum(nq),), generator=g, dtype=I32).cuda()
    rotary = kvc.Rotary(kvc.Rope(5e5), depth=depth)
    held = []
    for max_q in (63, 2333, 2334, 5000):                                          # 3 * 2334 > 7000
        x = fused.clone()
        c = base.pool(P, page, H, d, 1, q8, False)
        kvc.kvc_append_rotated(requests(nq, kv, table=table, max_q=max_q), rotary, x[:, Hq: Hq + H], x[:, Hq + H:], c, 0, q=x[:, :Hq], q_out=x[:, :Hq])
        torch.cuda.synchronize()
        assert torch.equal(x[:, Hq:], fused[:, Hq:])
        held.append([x] + [getattr(c, n).view(torch.uint8) for n in ("k", "v") + (("scale_k", "scale_v") if q8 else ())])
    for other in held[1:]:
        assert all(torch.equal(a, b) for a, b in zip(held[0], other))


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_special_values_and_skipped_rows(q8):
    """In a block of eight tokens: negative positions and a bad page skip keys, not queries; infinities stay in their pair."""
    H, d, page, m = 1, 64, 8, 70
    table = torch.tensor([[0, 1, 99, 2, 3, 4, 5, 6, 7]], dtype=I32)
    req = requests([m], [m - 3], table=table, max_kv=72, max_q=8000)                         # the first three have no place
    k = torch.ones(m, H, d, dtype=torch.bfloat16)
    k[12, 0, 5] = float("inf")
    q = k.clone().cuda()
    c, out = base.pool(8, page, H, d, 1, q8, False), torch.zeros_like(q)
    kvc.kvc_status_reset()
    kvc.kvc_append_rotated(req, kvc.Rotary(kvc.Rope(1e4)), k.cuda(), k.cuda(), c, 0, q=q, q_out=out)
    torch.cuda.synchronize()
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE | kvc.KVC_FLAG_BAD_LENGTH
    kvc.kvc_status_reset()
    bad = ~torch.isfinite(out.float())
    assert bad[12, 0].nonzero().flatten().tolist() == [5, 37] and bad.sum() == 2 and (out.float().nan_to_num(1).abs().sum(-1) > 0).all()
    untouched = ((c.k.view(torch.uint8) if q8 else c.k) == (0x2A if q8 else 7.0)).all(-1)[0, :, 0]
    assert untouched.flatten().nonzero().flatten().tolist() == [59, 60, 61, 62, 63]  # behind position 66
    row = c.k[0, 1, 0, 1].float()                                            # token 12 is at position 9
    assert (~torch.isfinite(row)).nonzero().flatten().tolist() == [5, 37]
