"""kvc_verify where probabilities are subnormal float32 numbers (what is left after a rejection, whole distributions) or far
above 1."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from test_gpu_verify import Case

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -149


def rows_of(c, make):
    return torch.from_numpy(np.stack([make() for _ in range(c.rows)])).to(torch.float32).cuda()


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
@pytest.mark.parametrize("V", [5, 1000, 6001, 20000])
def test_subnormal_residuals(V, drawn):
    """Drafts that are rejected take all normal numbers with them; the next token comes from entries of a few times 2^-149,
    whose sums and quotients float64 holds exactly or to its rounding."""
    c = Case([3] * 24, V, drawn=drawn, seed=V)
    rng = np.random.default_rng(V)
    c.parents = [[-1, 0, 0]] * 24

    def target():
        p = rng.integers(0, 9, V) * LEAST
        p[:2] = 0.25, 0.125
        return p

    c.target = rows_of(c, target)
    q = np.zeros(V)
    q[:2] = 0.5, 0.5
    c.draft = rows_of(c, lambda: q)
    c.token = np.tile([0, 0, 1], 24)
    c.u[:] = 0.75 if drawn else 0.5               # chosen: 0.5 * 1 >= 0.25, then 0.5 * 0.75 >= 0.125
    c.u_next[:] = (np.arange(24) + 0.37) / 24
    c.run().check()
    assert (c.n_kept == 1).all() and (c.next >= 2).all() and c.flags == 0
    assert len(set(c.next.tolist())) > 2 or V == 5


@pytest.mark.parametrize("V", [7, 4500])
def test_subnormal_distributions(V):
    """Nothing but subnormal numbers, up to the largest one, beside the smallest normal one: acceptance and draw."""
    for drawn in (True, False):
        c = Case([4] * 16, V, seed=V, drawn=drawn)
        rng = np.random.default_rng(V + 1)
        c.target = rows_of(c, lambda: rng.integers(1, 1 << 23, V) * LEAST)
        c.target[:, 3] = 2.0 ** -126
        c.draft = rows_of(c, lambda: rng.integers(1, 1 << 23, V) * LEAST)
        c.run().check()
        assert c.flags == 0


@pytest.mark.parametrize("drawn", [True, False], ids=["drawn", "chosen"])
@pytest.mark.parametrize("V", [7, 4500])
def test_entries_far_above_one(V, drawn):
    """Up to 2^104 - 1 step a distribution is a distribution; from there on it has no finite sum."""
    c = Case([3] * 16, V, seed=V, drawn=drawn)
    c.target *= 2.0 ** 100
    c.draft *= 2.0 ** 100
    c.target[:, 2] = float(np.nextafter(np.float32(2.0 ** 104), np.float32(0)))
    c.u *= 2.0 ** -10 if drawn else 1.0
    c.run().check()
    assert c.flags == 0
    c.target[:, 2] = 2.0 ** 104
    c.run()
    assert c.flags == kvc.KVC_FLAG_BAD_PROB and (c.next == -1).all()
