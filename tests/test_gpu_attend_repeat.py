"""Many calls with few tiles a block, where the halves of a row that two groups of warps hold are put together all the time:
every call gives the first one's bits, and those are right."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq,G,d", [(1, 4, 128), (2, 8, 128), (4, 8, 64)])
def test_repeated_calls_give_the_same_bits(nq, G, d, q8):
    b = Built(Step([nq] * 90, [130 + 3 * i for i in range(90)], H=3, G=G, d=d, q8=q8, seed=nq))
    want, wlse = b.run()
    b.check(want, wlse)
    ws = b.workspace()
    outs = [(torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")) for _ in range(50)]
    for out, lse in outs:
        kvc.kvc_attend(b.req, b.q, b.cache, 0, out, ws, lse=lse)
    torch.cuda.synchronize()
    for out, lse in outs:
        assert torch.equal(out, want) and torch.equal(lse, wlse)
    assert kvc.kvc_status_poll() == 0
