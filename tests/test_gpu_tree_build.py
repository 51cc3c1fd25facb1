"""kvc_tree_build against the oracle, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from draft_helpers import I32, built_tree, flat, random_parents, requests
from oracle import draft_oracle as orc

pytestmark = pytest.mark.gpu


def expect(tree, nq, parents):
    mask, depth = tree.mask.cpu().numpy().view(np.uint32), tree.depth.cpu().numpy()
    r = 0
    for m, p in zip(nq, parents):
        seen, d = orc.tree_rows(p)
        assert np.array_equal(mask[r: r + m], orc.mask_words(seen, mask.shape[1]))
        assert depth[r: r + m].tolist() == d
        r += m
    return r


@pytest.mark.parametrize("nq,kind", [([1], "tree"), ([13], "tree"), ([32, 33, 31], "tree"), ([0, 5, 0, 200], "forest"), ([64] * 40, "tree"),
                                     ([1024], "chain"), ([1024, 1000], "tree"), ([257, 3], "chain")])
def test_against_the_oracle(nq, kind):
    parents = random_parents(nq, sum(nq), kind)
    kvc.kvc_status_reset()
    expect(built_tree(requests(nq, nq), parents, sum(nq)), nq, parents)
    assert kvc.kvc_status_poll() == 0


def test_wider_masks_and_padding_rows():
    nq, spare = [40, 7], 5
    parents = random_parents(nq, 3)
    req = requests(nq, nq, max_q=70)
    t = kvc.Tree(flat(parents, spare, -9).cuda(), 70, mask=torch.full((sum(nq) + spare, 5), 0x5A5A, dtype=I32, device="cuda"),
                 depth=torch.full((sum(nq) + spare,), 77, dtype=I32, device="cuda"))
    kvc.kvc_status_reset()
    kvc.kvc_tree_build(req, t)
    end = expect(t, nq, parents)
    assert (t.mask[end:] == 0x5A5A).all() and (t.depth[end:] == 77).all() and kvc.kvc_status_poll() == 0


def test_parents_out_of_range_count_as_none():
    parents = [[-1, 0, 2, 7, -2, 1, 4], [0, -1, 1]]
    nq = [7, 3]
    kvc.kvc_status_reset()
    expect(built_tree(requests(nq, nq), parents, 10), nq, parents)
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_TREE
    kvc.kvc_status_reset()


def test_a_request_out_of_bounds_is_left():
    nq = [4, 6]
    parents = random_parents(nq, 2)
    req = requests(nq, [4, 99], max_kv=50)
    t = kvc.Tree(flat(parents).cuda(), 6)
    t.mask.fill_(-3)
    kvc.kvc_status_reset()
    kvc.kvc_tree_build(req, t)
    expect(t, nq[:1], parents[:1])
    assert (t.mask[4:] == -3).all() and kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_LENGTH
    kvc.kvc_status_reset()
