"""Tree attention over 8-bit caches whose keys are huge and whose queries are tiny: logits fit float32 although the products
of codes and key scales would not."""
import numpy as np
import pytest
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Step
from draft_helpers import TreeBuilt

pytestmark = pytest.mark.gpu


def moved(st, key, query, which):
    """Keys (those of `which`) up by powers of two, queries down."""
    b = TreeBuilt(st)
    b.q_cpu = (b.q_cpu.float() * 2.0 ** -query).to(torch.bfloat16)
    b.q.copy_(b.q_cpu)
    e = b.cache.scale_k.cpu().numpy()                                 # [L, P, H, page]
    for i, kv in enumerate(st.kv):
        for t in np.arange(kv)[which(np.arange(kv))]:
            at = (st.layer, int(b.req.page_table[i, t // st.page]), slice(None), t % st.page)
            e[at] += np.uint8(key)
            b.val_k[i][t] = b.val_k[i][t] * 2.0 ** key
    b.cache.scale_k.copy_(torch.from_numpy(e))
    return b


EVERY, SOME, LAST = (lambda t: t >= 0), (lambda t: t % 97 == 5), (lambda t: t >= len(t) - 40)


@pytest.mark.parametrize("m,G,d", [(4, 4, 128), (10, 4, 128), (30, 4, 64), (7, 8, 64), (40, 4, 128)])
@pytest.mark.parametrize("key,query,which", [(118, 118, EVERY), (118, 119, SOME), (112, 112, LAST), (70, 70, EVERY), (100, 95, EVERY), (64, 66, SOME)],
                         ids=["every", "some", "last", "at_the_border", "strong", "half"])
def test_huge_keys_and_tiny_queries(key, query, which, m, G, d):
    b = moved(Step([m, 5], [400, 150], G=G, d=d, q8=True, seed=m), key, query, which)
    kvc.kvc_status_reset()
    out, lse = b.run_tree()
    assert kvc.kvc_status_poll() == 0 and torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
    b.check_tree(out, lse)
