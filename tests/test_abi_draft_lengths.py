"""kvc_append_rotated with bounds on the new tokens near 2^31: refused before a grid is made of them."""
import pytest

import paper_2609_34060_b200 as kvc
from paper_2609_34060_b200 import build as kbuild
from test_abi_draft import K, UNSUPPORTED, V, _heads, _p, _pool, _q8, _req, _rot

MOST = 2 ** 31 - 1 - 256


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return kvc.load()


@pytest.mark.parametrize("max_q", [MOST + 1, 2 ** 31 - 8, 2 ** 31 - 7, 2 ** 31 - 1])
def test_bounds_past_the_last_tile_are_refused(lib, max_q):
    args = (_p(_rot()), None, None, _p(_heads(K)), _p(_heads(V)), 0)
    assert lib.kvc_append_rotated(_p(_req(max_q=max_q)), *args, _p(_pool()), None) == UNSUPPORTED
    assert lib.kvc_append_rotated_q8(_p(_req(max_q=max_q)), *args, _p(_q8()), None) == UNSUPPORTED


def test_the_largest_bound_passes_the_checks(lib):
    """n = 0: checks alone."""
    args = (_p(_rot()), None, None, _p(_heads(K)), _p(_heads(V)), 0)
    assert lib.kvc_append_rotated(_p(_req(n=0, max_q=MOST)), *args, _p(_pool()), None) == 0
