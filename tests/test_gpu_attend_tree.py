"""kvc_attend_tree against float64: trees, chains, forests and masks of the caller's own; both kernels, bf16 and 8 bits."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Step
from draft_helpers import TreeBuilt

pytestmark = pytest.mark.gpu

STEPS = [
    Step([1], [1], H=1, G=1, d=64, page=8),
    Step([5], [5], H=2, G=2, d=128),                                   # nothing but drafts
    Step([7], [130], H=2, G=4, d=128),                                 # few rows, drafts across a tile's border
    Step([8], [128], H=1, G=4, d=64),                                  # drafts end with the tile
    Step([13, 1, 0, 6], [777, 40, 9, 129], H=2, G=4, d=128, spare=3),
    Step([32], [161], H=2, G=1, d=128, page=32),
    Step([33, 20], [500, 148], H=2, G=4, d=128),                       # the other kernel
    Step([64], [1100], H=1, G=8, d=64, page=64, token_major=True),
    Step([200], [333], H=2, G=2, d=128, page=16),                      # masks of seven words, drafts over three tiles
    Step([300, 17], [300, 290], H=1, G=1, d=64, page=8, token_major=True),
    Step([40], [90], H=2, G=3, d=128, page=0, token_major=True),       # contiguous rows
    Step([9], [250], H=3, G=7, d=128, page=0),
    Step([16] * 6, [400, 16, 129, 128, 127, 1000], H=2, G=2, d=128, key_scale=3.0),
    Step([3, 90, 1, 40], [500, 700, 300, 260], H=2, G=4, d=128, L=2, layer=1, spare=2),
]


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("i", range(len(STEPS)))
def test_trees(i, q8):
    st = Step(**{**STEPS[i].__dict__, "q8": q8, "seed": i})
    b = TreeBuilt(st)
    kvc.kvc_status_reset()
    out, lse = b.run_tree()
    assert kvc.kvc_status_poll() == 0 and kvc.kvc_last_path() == kvc.KVC_PATH_TC
    b.check_tree(out, lse)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,kv,G", [([12], [3000], 4), ([16, 9, 2], [2500, 64, 1900], 4), ([25, 32, 7], [1800, 140, 2200], 4), ([128], [1000], 1), ([5, 5], [129, 63], 13)])
def test_one_row_tile(nq, kv, G, d, q8):
    """33 to 128 rows, units cut into pieces and whole ones, lengths on and off the tiles' halves."""
    b = TreeBuilt(Step(nq, kv, G=G, d=d, q8=q8, seed=sum(kv)))
    out, lse = b.run_tree()
    b.check_tree(out, lse)
    again, lse2 = b.run_tree()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("ramp", [60.0, -60.0, 400.0])
@pytest.mark.parametrize("m", [10, 30])
def test_rising_and_falling_logits(m, ramp, q8):
    """Keys that grow or shrink with their position: maxima move inside tiles, far above what came before."""
    b = TreeBuilt(Step([m], [700], G=4, q8=q8, ramp=ramp, seed=m))
    b.check_tree(*b.run_tree())


@pytest.mark.parametrize("nq,kv,G,same", [([4, 3], [90, 200], 4, True), ([70], [300], 2, True), ([6, 3], [90, 200], 4, False), ([30], [900], 4, False)])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_a_chain_is_causal_attention(nq, kv, G, same, q8):
    """A chain's mask hides what the causal rule hides: the same bits where both calls take the same kernel (up to 16 and
    beyond 128 rows), otherwise the same numbers (both are checked against float64)."""
    b = TreeBuilt(Step(nq, kv, G=G, q8=q8), kind="chain")
    out, lse = b.run_tree()
    want, want_lse = b.run()
    assert not same or (torch.equal(out, want) and torch.equal(lse, want_lse))
    b.check_tree(out, lse)
    b.check_tree(want, want_lse)


@pytest.mark.parametrize("nq,kv,G", [([8], [300], 4), ([45, 20], [45, 300], 4)])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_forests_and_wide_masks(nq, kv, G, q8):
    b = TreeBuilt(Step(nq, kv, G=G, q8=q8, seed=3), kind="forest", words=6)
    b.check_tree(*b.run_tree())


@pytest.mark.parametrize("nq,kv,G", [([12], [12], 2), ([50], [50], 4), ([20, 50], [300, 140], 2)])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_masks_of_the_callers_own(nq, kv, G, q8):
    """Rows that see nothing (not even themselves, without a context), any bits, bits beyond the row's own place."""
    rng = np.random.default_rng(5)
    seen = [[set() if j % 5 == 3 else set(np.nonzero(rng.random(m) < 0.3)[0].tolist()) for j in range(m)] for m in nq]
    b = TreeBuilt(Step(nq, kv, G=G, q8=q8, seed=9), seen=seen)
    b.check_tree(*b.run_tree())


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("m", [6, 60])
def test_more_new_tokens_than_the_cache_holds(m, q8):
    """Rows at negative positions see nothing; the others the drafts that the cache holds."""
    b = TreeBuilt(Step([m], [m - 4], q8=q8, seed=2))
    b.check_tree(*b.run_tree())


@pytest.mark.parametrize("m,G", [(7, 4), (60, 2)])
def test_hidden_drafts_may_hold_anything(m, G):
    """Keys of drafts that nobody's mask names: infinities and NaN do not reach the others (their values are finite)."""
    st = Step([m], [200], G=G, seed=4)
    seen = [[{a for a in (0, j) if a != 3} for j in range(m)]]
    b = TreeBuilt(st, seen=seen)
    t = 200 - m + 3
    p, s = int(b.req.page_table[0, t // 16]), t % 16
    b.cache.k[0, p, :, s] = float("nan")
    b.cache.k[0, p, :, s, ::3] = float("inf")
    out, lse = b.run_tree()
    keep = [j for j in range(m) if j != 3]
    assert torch.isfinite(out[keep].float()).all()
    b.check_tree(out, lse)


@pytest.mark.parametrize("path", [kvc.KVC_PATH_GENERIC, kvc.KVC_PATH_TC])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
def test_both_families(path, q8):
    b = TreeBuilt(Step([21, 5], [250, 60], H=2, G=3, q8=q8, seed=6), kind="forest")
    kvc.kvc_set_path(path)
    try:
        b.check_tree(*b.run_tree())
        assert kvc.kvc_last_path() == path
    finally:
        kvc.kvc_set_path(kvc.KVC_PATH_AUTO)


def test_bad_pages_and_lengths_are_flagged():
    b = TreeBuilt(Step([5, 5], [100, 60], seed=1))
    b.req.page_table[0, 1] = 1 << 20
    kvc.kvc_status_reset()
    out, _ = b.run_tree()
    assert kvc.kvc_status_poll() == kvc.KVC_FLAG_BAD_PAGE and torch.isfinite(out[5:].float()).all()
    kvc.kvc_status_reset()
    b.req.kv_len[1] = 101
    out, _ = b.run_tree()
    assert kvc.kvc_status_poll() & kvc.KVC_FLAG_BAD_LENGTH and (out[5:] == 7.0).all()
    kvc.kvc_status_reset()


def test_large_mixed_batch_by_both_kernels():
    """Enough tiles that single tokens go to the few-rows kernel and the trees to the other."""
    nq = [1] * 30 + [70, 33, 100]
    kv = [1500 + 37 * i for i in range(30)] + [3000, 2100, 2700]
    b = TreeBuilt(Step(nq, kv, H=4, G=2, d=64, seed=8))
    out, lse = b.run_tree()
    b.check_tree(out, lse)
    again, lse2 = b.run_tree()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
