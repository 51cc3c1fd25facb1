"""A serving step over given keys, values and queries (one request, contiguous rows) and its float64 answer."""
import numpy as np
import torch

import paper_2609_34060_b200 as kvc
from attend_helpers import Built, Step, f64
from oracle import attend_oracle as orc


class Given(Built):
    """k, v float [T, H, d] and q float [rows, H G, d] on the CPU, rounded to bf16 (8-bit caches: then to codes); the last
    `rows` of the T tokens are the new ones."""

    def __init__(self, k, v, q, q8=False, causal=True, dev="cuda"):
        (T, H, d), rows = k.shape, q.shape[0]
        self.st = Step([rows], [T], H=H, G=q.shape[1] // H, d=d, page=0, q8=q8, causal=causal)
        k, v, self.q_cpu = (x.to(torch.bfloat16) for x in (k, v, q))
        lay = lambda x: x.transpose(0, 1)[None].contiguous()                 # [1, H, T, d]
        if q8:
            (ck, ek), (cv, ev) = (orc.quantize_rows(f64(lay(x))) for x in (k, v))
            code = lambda c: torch.from_numpy(c).view(torch.float8_e4m3fn).to(dev)
            self.cache = kvc.QCache(code(ck), code(cv), torch.from_numpy(ek).to(dev), torch.from_numpy(ev).to(dev))
            val = lambda c, e: orc.dequantize_rows(c, e)[0].transpose(1, 0, 2)
            self.val_k, self.val_v = [val(ck, ek)], [val(cv, ev)]
            self.codes_v = [orc.dequantize_rows(cv, np.full_like(ev, 127))[0].transpose(1, 0, 2)]
            self.exp_v = [ev[0].astype(np.int64).T - 127]                    # [T, H]
        else:
            self.cache = kvc.Cache(lay(k).to(dev), lay(v).to(dev))
            self.val_k, self.val_v = [f64(k)], [f64(v)]
        self.begin, self.rows = np.array([0, rows], np.int32), rows
        self.req = kvc.Requests(torch.tensor([0, rows], dtype=torch.int32, device=dev), torch.tensor([T], dtype=torch.int32, device=dev), rows, T)
        self.q, self.scale = self.q_cpu.to(dev), d ** -0.5
