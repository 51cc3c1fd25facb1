"""Scratch of kvc_attend and kvc_attend_tree for 17 to 128 rows a KV head: what either call needs, and nothing behind it."""
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step
from draft_helpers import TreeBuilt

pytestmark = pytest.mark.gpu


def few_rows_bytes(st, capacity):
    """What the kernel for up to `capacity` rows a KV head writes: for every block two units' sums, maxima and totals."""
    tiles = len(st.nq) * st.H * -(-max(st.kv) // 128)
    blocks = min(tiles, torch.cuda.get_device_properties(0).multi_processor_count)
    return blocks * 2 * capacity * (st.d + 2) * 4


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("nq,kv,G,H,d", [([5, 2], [1000, 700], 4, 2, 128), ([8], [30000], 4, 8, 128), ([17], [400], 1, 1, 64)])
def test_a_call_without_a_tree_takes_what_it_needs(nq, kv, G, H, d, q8):
    st = Step(nq, kv, H=H, G=G, d=d, q8=q8)
    assert 17 <= max(nq) * G <= 32
    b = Built(st)
    out, lse = torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")
    need = few_rows_bytes(st, 32)
    assert kvc.kvc_attend_workspace_bytes(b.req, b.cache, H * G) <= need + 4096           # with a tree the blocks' starts as well
    arena = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    kvc.kvc_attend(b.req, b.q, b.cache, 0, out, arena[:need], lse=lse)
    torch.cuda.synchronize()
    assert (arena[need:] == 0xAB).all()
    want, want_lse = b.run()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    with pytest.raises(kvc.KvcError) as e:
        kvc.kvc_attend(b.req, b.q, b.cache, 0, out, arena[: need - 1024])
    assert e.value.code == kvc.KVC_E_WORKSPACE


@pytest.mark.parametrize("q8", [False, True], ids=["bf16", "q8"])
@pytest.mark.parametrize("m,G", [(17, 1), (20, 1), (8, 4), (33, 1), (13, 4), (32, 2), (24, 4), (13, 8), (32, 4), (129, 1)])
def test_a_tree_stays_inside_its_scratch(m, G, q8):
    """A long context in many pieces: every block leaves partial results, also the last one."""
    b = TreeBuilt(Step([m, 3], [9000, 7000], H=8, G=G, d=64, q8=q8, seed=m))
    need = kvc.kvc_attend_workspace_bytes(b.req, b.cache, 8 * G)
    arena = torch.full((need + 8192,), 0xAB, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")
    kvc.kvc_attend_tree(b.req, b.tree, b.q, b.cache, 0, out, arena[:need], lse=lse)
    torch.cuda.synchronize()
    assert (arena[need:] == 0xAB).all()
    want, want_lse = b.run_tree()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.isfinite(out.float()).all()
