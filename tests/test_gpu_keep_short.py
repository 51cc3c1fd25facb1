"""kvc_keep where a request has more new tokens than its cache holds: no length below zero, whatever is kept."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from test_gpu_keep import make, parts, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("keep", [[], [0], [3, 7]])
def test_a_first_position_below_zero(keep, q8):
    c, table = make([16, 30], 2, 64, 16, 2, q8, False, 4)
    was = parts(c)
    flags, kv_out = run(c, table, [8, 8], [5, 30], [keep, []])
    assert flags == kvc.KVC_FLAG_BAD_TREE and kv_out.tolist() == [5, 22]
    assert all(torch.equal(parts(c)[n].view(torch.uint8), was[n].view(torch.uint8)) for n in was)


@pytest.mark.parametrize("nq,kv", [([0, 4], [0, 4]), ([4, 0], [4, 9])])
def test_nothing_kept_of_what_the_cache_holds(nq, kv):
    """An empty list is no fault by itself: the length falls back to the context's."""
    c, table = make(kv, 1, 64, 16, 1, False, False, 5)
    flags, kv_out = run(c, table, nq, kv, [[], []])
    assert flags == 0 and kv_out.tolist() == [t - m for m, t in zip(nq, kv)]
