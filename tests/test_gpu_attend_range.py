"""Values far from 1 under logits that keep rising: the sums stay within float32's range, so finite answers come out finite."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_given import Given

pytestmark = pytest.mark.gpu


def rising(T, H, rows, G, d, step, size, q8, seed=0):
    """Logits that climb by `step` powers of two from one tile of 128 keys to the next, values of magnitude 2^size."""
    g = torch.Generator().manual_seed(seed)
    u = torch.ones(d)
    per = step * 0.6931471805599453 / 128 * d ** 0.5 / d          # of u . u = d, after the scale 1 / sqrt(d)
    k = (torch.arange(T) * per)[:, None, None] * u + 0.01 * torch.randn(T, H, d, generator=g)
    v = torch.randn(T, H, d, generator=g) * 2.0 ** size
    q = u.expand(rows, H * G, d).clone()
    return Given(k, v, q, q8=q8)


@pytest.mark.parametrize("path", ["generic", "auto"])
@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("rows,T,H,G", [(1, 700, 1, 4), (70, 700, 1, 4), (1, 9000, 8, 4), (17, 9000, 8, 2)])   # the last two: several tiles a block
@pytest.mark.parametrize("step", [6.0, 30.0, 58.0])
@pytest.mark.parametrize("size", [100, -60])
def test_large_and_small_values_under_rising_logits(size, step, rows, T, H, G, q8, path):
    b = rising(T, H, rows, G, 128, step, size, q8)
    kvc.kvc_status_reset()
    kvc.kvc_set_path(kvc.KVC_PATH_GENERIC if path == "generic" else kvc.KVC_PATH_AUTO)
    try:
        out, lse = b.run()
    finally:
        kvc.kvc_set_path(kvc.KVC_PATH_AUTO)
    assert torch.isfinite(out).all()
    b.check(out, lse)
    assert kvc.kvc_status_poll() == 0
