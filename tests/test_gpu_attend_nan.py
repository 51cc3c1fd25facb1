"""A NaN among the logits of a row makes the row NaN, its log-sum-exp too, also where nothing but NaN is seen: in every
kernel, bf16 and 8 bits, whole rows and rows whose keys are shared out over many blocks."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(params=["generic", "auto"])
def path(request):
    kvc.kvc_set_path(kvc.KVC_PATH_GENERIC if request.param == "generic" else kvc.KVC_PATH_AUTO)
    kvc.kvc_status_reset()
    yield request.param
    kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
    assert kvc.kvc_status_poll() == 0


def poison_keys(b, lo, hi, head):
    """Keys lo .. hi - 1 of request 0: every channel NaN (8-bit caches: by their exponent)."""
    page = b.st.page
    for t in range(lo, hi):
        p = int(b.req.page_table[0, t // page])
        if b.st.q8:
            b.cache.scale_k[0, p, head, t % page] = 255
        else:
            b.cache.k[0, p, head, t % page] = NAN


def all_nan(x):
    return bool(torch.isnan(x).all())


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq,kv", [(1, 300), (3, 300), (70, 300), (300, 700), (1, 9000), (40, 10007)])
def test_a_query_of_nan(nq, kv, q8, path):
    """One query row of one head: that row is NaN, every other is what it is without it being there."""
    b = Built(Step([nq], [kv], H=1, G=4, q8=q8))
    row, head = nq // 2, 2
    b.q[row, head, 5] = NAN
    out, lse = b.run()
    assert all_nan(out[row, head]) and all_nan(lse[row, head])
    out[row, head], lse[row, head] = 0, 0
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 6, 70, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_the_first_key_of_a_prompt_is_nan(nq, q8, d, path):
    """Row 0 sees that key alone; every row sees it."""
    b = Built(Step([nq], [nq], H=2, G=2, d=d, q8=q8))
    poison_keys(b, 0, 1, 0)
    out, lse = b.run()
    assert all_nan(out[:, :2]) and all_nan(lse[:, :2])
    assert torch.isfinite(out[:, 2:]).all() and torch.isfinite(lse[:, 2:]).all()


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq", [1, 40, 150])
@pytest.mark.parametrize("lo,hi", [(1280, 1408), (0, 128), (0, 5000), (0, 10007)])
def test_whole_tiles_of_nan(nq, lo, hi, q8, path):
    """Tiles of keys that are nothing but NaN, each a block's whole share of a long context (79 tiles, one or two units)."""
    b = Built(Step([nq], [10007], H=1, G=4, q8=q8))
    poison_keys(b, lo, hi, 0)
    out, lse = b.run()
    assert all_nan(out) and all_nan(lse)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_a_nan_that_only_later_rows_see(q8, path):
    """Keys from 250 on are NaN: rows before them are as good as without, rows behind are NaN."""
    b = Built(Step([300], [300], H=1, G=2, q8=q8))
    want, wlse = b.run()
    poison_keys(b, 250, 300, 0)
    out, lse = b.run()
    assert torch.equal(out[:250], want[:250]) and torch.equal(lse[:250], wlse[:250])
    assert all_nan(out[250:]) and all_nan(lse[250:])


def test_rows_that_see_nothing_stay_zero(path):
    for q8 in (False, True):
        for nq, kv in ((300, 5), (40, 0), (2, 0)):
            b = Built(Step([nq], [kv], H=1, G=2, q8=q8))
            out, lse = b.run()
            n = nq - kv
            assert (out[:n] == 0).all() and (lse[:n] == -float("inf")).all() and torch.isfinite(lse[n:]).all()
