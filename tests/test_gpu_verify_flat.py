"""kvc_verify where most of the vocabulary is left after every rejection: passes over whole distributions, again and again."""
import numpy as np
import pytest
import torch

from test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,V,sharp", [(1, 131072, 1.0), (40, 60000, 1.0), (3, 100003, 3.0), (2, 3000, 0.5)])
def test_rejections_that_leave_the_vocabulary(n, V, sharp):
    """q = 0.75 p with the rest on the drafted tokens: a rejection leaves about p, so that the next one finds it again.  Four
    siblings are rejected, the fifth stays, and the same follows at its children; sums of 131072 float64 terms agree with the
    oracle's to far less than what the random numbers are away from any border."""
    c = Case([12] * n, V, seed=V, sharp=sharp)
    c.parents = [[-1, 0, 0, 0, 0, 0] + [5] * 6] * n
    rng = np.random.default_rng(V)
    p = c.target.cpu().numpy().astype(np.float64)
    q = 0.75 * p
    c.token = np.zeros(12 * n, np.int64)
    for b in range(n):
        for node, first in ((0, 1), (5, 6)):
            bad = rng.choice(V, 4, replace=False)
            q[12 * b + node, bad] += 0.0625
            c.token[12 * b + first: 12 * b + first + 4] = bad
            c.token[12 * b + first + 4] = rng.choice(np.setdiff1d(np.arange(min(V, 5000)), bad))
    c.draft = torch.from_numpy(q.astype(np.float32)).cuda()
    c.u[:] = 0.9999
    c.u[5::12] = c.u[10::12] = 0.5
    c.run().check()
    assert (c.n_kept == 3).all() and c.flags == 0
