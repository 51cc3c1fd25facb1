"""Operators that keep a cache in 8 bits, write new tokens into it and attend over it: measured cases and plain forms.

``kvc_attend`` / ``kvc_append`` / ``kvc_quantize`` / ``kvc_dequantize`` on the caches this library serves (bf16, or e4m3
codes with one power-of-two scale per token and head; contiguous, or pages and a page table).  ``run`` computes a case
with elementary torch operations in float32, or, where ``own`` is true, with the calls a user makes of the library.
"""
import math
import random

import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ cases


def listed():
    return [
        # one request generates its next token over a short context: latency
        dict(name="attend_token_short", op="attend", n=1, hq=32, h=8, d=128, page=16, q_lo=1, q_hi=1, kv=777, spread=0.0,
             kv_max=777, q8=False, causal=True, lse=False, token_major=False, spare=0),
        # the serving batch: 64 requests, lognormal context lengths, one new token each
        dict(name="attend_tokens_batch", op="attend", n=64, hq=32, h=8, d=128, page=16, q_lo=1, q_hi=1, kv=4096, spread=0.6,
             kv_max=32768, q8=False, causal=True, lse=False, token_major=False, spare=0),
        # eight agents of the long-context shape, each at its next token over a 32K cache held in 8 bits
        dict(name="attend_tokens_long_q8", op="attend", n=8, hq=64, h=8, d=128, page=16, q_lo=1, q_hi=1, kv=32000, spread=0.02,
             kv_max=32768, q8=True, causal=True, lse=False, token_major=False, spare=0),
        # an agent's own 2K of new tokens behind a shared context, 8K in all
        dict(name="attend_chunk_8k", op="attend", n=1, hq=32, h=8, d=128, page=16, q_lo=2048, q_hi=2048, kv=8192, spread=0.0,
             kv_max=8192, q8=False, causal=True, lse=False, token_major=False, spare=0),
        # a question behind an image context held in 8 bits, seven query heads per KV head, lengths off every grid
        dict(name="attend_chunk_vlm_q8", op="attend", n=1, hq=28, h=4, d=128, page=16, q_lo=777, q_hi=777, kv=16651, spread=0.0,
             kv_max=16651, q8=True, causal=True, lse=True, token_major=False, spare=0),
        # prompts and single tokens in one batch, head dim 64, pages of 32 tokens in token order, padding rows at the end
        dict(name="attend_mixed_d64", op="attend", n=9, hq=8, h=2, d=64, page=32, q_lo=1, q_hi=400, kv=1500, spread=0.5,
             kv_max=4096, q8=False, causal=True, lse=True, token_major=True, spare=13),
        # the 64 new tokens of a decode step written into an 8-bit pool: latency
        dict(name="append_tokens_q8", op="append", n=64, h=8, d=128, page=16, q_lo=1, q_hi=1, kv=1024, spread=0.3,
             kv_max=2048, q8=True, token_major=False),
        # prompts written into a bf16 pool
        dict(name="append_prompts", op="append", n=5, h=8, d=128, page=16, q_lo=1500, q_hi=2500, kv=2900, spread=0.1,
             kv_max=4096, q8=False, token_major=False),
        # an agent's finished 8K cache put away in 8 bits, all layers
        dict(name="quantize_8k", op="quantize", layers=32, h=8, d=128, tokens=8192, page=0, token_major=False),
        # the parity-sized cache, in pages, a partial last page
        dict(name="quantize_tiny", op="quantize", layers=2, h=2, d=64, tokens=251, page=16, token_major=False),
        # the image context read back for the next agent's correction, in pages
        dict(name="dequantize_vlm_16k", op="dequantize", layers=28, h=4, d=128, tokens=16384, page=16, token_major=False),
        # the parity-sized cache read back
        dict(name="dequantize_tiny", op="dequantize", layers=2, h=2, d=64, tokens=256, page=0, token_major=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "quantize", "dequantize"])
    d = rng.choice([64, 128, 128])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "attend":
        h = rng.choice([1, 2, 4, 8])
        g = rng.choice([1, 2, 3, 4, 7, 8])
        kind = rng.choice(["tokens", "few", "chunk", "mixed"])
        if kind == "tokens":
            n, q_lo, q_hi, kv = _log_int(rng, 1, 96), 1, 1, _log_int(rng, 1, 24000)
        elif kind == "few":
            n, q_lo, q_hi, kv = _log_int(rng, 1, 16), 2, rng.randint(2, 24), _log_int(rng, 32, 16000)
        elif kind == "chunk":
            n, q_hi = 1, _log_int(rng, 32, 1500)
            q_lo, kv = q_hi, _log_int(rng, q_hi, 12000)
        else:
            n, q_lo, q_hi, kv = rng.randint(2, 10), 1, rng.randint(2, 500), _log_int(rng, 500, 3500)
        kv_max = max(kv, q_hi) if n == 1 else max(q_hi, min(2 * kv, 32768))
        while n * kv_max * h > 3000000:
            n = max(1, n // 2)
        while g > 1 and n * q_hi * h * g * kv_max > 400000000:
            g -= 1
        return dict(op=op, n=n, hq=h * g, h=h, d=d, page=page, q_lo=q_lo, q_hi=q_hi, kv=kv, spread=0.0 if n == 1 else 0.4,
                    kv_max=kv_max, q8=rng.random() < 0.5, causal=rng.random() < 0.8, lse=rng.random() < 0.5,
                    token_major=rng.random() < 0.3, spare=rng.choice([0, 0, 5]))
    if op == "append":
        n = _log_int(rng, 1, 64)
        q_hi = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4000 // n + 2)
        kv = q_hi + _log_int(rng, 1, 1500)
        return dict(op=op, n=n, h=rng.choice([1, 2, 4, 8]), d=d, page=page, q_lo=1 if n > 1 else q_hi, q_hi=q_hi, kv=kv,
                    spread=0.2, kv_max=2 * kv, q8=rng.random() < 0.6, token_major=rng.random() < 0.3)
    layers, h, tokens = rng.randint(1, 24), rng.choice([1, 2, 4, 8]), _log_int(rng, 1, 9000)
    return dict(op=op, layers=layers, h=h, d=d, tokens=tokens, page=rng.choice([0, page]), token_major=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(shape, g, outlier_axis_heads=None):
    """bf16 normal draws; keys have four channels of every head ten times larger, as the caches of this library do."""
    x = torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g)
    if outlier_axis_heads is not None:
        h, d = shape[outlier_axis_heads], shape[-1]
        pick = torch.rand(h, d, device=DEV, generator=g).argsort(dim=1) < 4
        view = [1] * len(shape)
        view[outlier_axis_heads], view[-1] = h, d
        x = x * (1.0 + 9.0 * pick.float()).view(view)
    return x.to(torch.bfloat16)


def _pool_shape(c, pages, layers=1):
    return (layers, pages, c["page"], c["h"], c["d"]) if c["token_major"] else (layers, pages, c["h"], c["page"], c["d"])


def _head_axis(c):
    return 3 if c["token_major"] else 2


def _codes(shape, g):
    """Codes as a quantised cache holds them (normal rows under their power-of-two scale) and exponents near 1."""
    x = torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g) * 110.0
    x = x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    e = torch.randint(118, 121, shape[:-1], device=DEV, generator=g, dtype=torch.int32).to(torch.uint8)
    return x, e


def _lengths(c):
    """New tokens and cache lengths of the requests: the case's own, whatever the seed (buffers keep their shapes)."""
    rng = random.Random("%(n)d %(q_lo)d %(q_hi)d %(kv)d %(kv_max)d" % c)
    nq = [rng.randint(c["q_lo"], c["q_hi"]) for _ in range(c["n"])]
    kv = [int(round(c["kv"] * math.exp(c["spread"] * rng.gauss(0.0, 1.0)))) for _ in range(c["n"])]
    return nq, [max(1, m, min(t, c["kv_max"])) for m, t in zip(nq, kv)]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    if c["op"] in ("attend", "append"):
        nq, kv = _lengths(c)
        s["max_q"], s["max_kv"] = max(nq), max(kv)
        nq, kv = torch.tensor(nq, device=DEV), torch.tensor(kv, device=DEV)
        per = -(-s["max_kv"] // c["page"])                        # table entries of a request
        need = (kv + c["page"] - 1) // c["page"]
        pages = int(need.sum()) + 3
        perm = torch.rand(pages, device=DEV, generator=g).argsort()
        col = torch.arange(per, device=DEV)[None, :]
        first = torch.cumsum(need, 0) - need
        s["table"] = torch.where(col < need[:, None], perm[(first[:, None] + col).clamp(max=pages - 1)], 0).to(torch.int32)
        s["q_begin"] = torch.cat([nq.new_zeros(1), torch.cumsum(nq, 0)]).to(torch.int32)
        s["kv_len"] = kv.to(torch.int32)
        rows = int(nq.sum()) + c.get("spare", 0)
        shape = _pool_shape(c, pages)
        if c["q8"]:
            s["k"], s["scale_k"] = _codes(shape, g)
            s["v"], s["scale_v"] = _codes(shape, g)
        else:
            s["k"], s["v"] = _rows(shape, g, _head_axis(c)), _rows(shape, g)
        if c["op"] == "attend":
            s["q"] = _rows((rows, c["hq"], c["d"]), g)
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(rows, c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        else:
            s["k_new"], s["v_new"] = _rows((rows, c["h"], c["d"]), g, 1), _rows((rows, c["h"], c["d"]), g)
        return s
    if c["page"]:
        pages = -(-c["tokens"] // c["page"]) + 2
        shape = _pool_shape(c, pages, c["layers"])
        s["table"] = torch.rand(pages, device=DEV, generator=g).argsort()[: pages - 2].to(torch.int32)
    else:
        t, h, d = c["tokens"], c["h"], c["d"]
        shape = (c["layers"], t, h, d) if c["token_major"] else (c["layers"], h, t, d)
        s["table"] = None
    axis = _head_axis(c) if c["page"] else (2 if c["token_major"] else 1)
    if c["op"] == "quantize":
        s["src_k"], s["src_v"] = _rows(shape, g, axis), _rows(shape, g)
        s["k"], s["v"] = (torch.zeros(shape, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
        s["scale_k"], s["scale_v"] = (torch.zeros(shape[:-1], dtype=torch.uint8, device=DEV) for _ in range(2))
    else:
        s["k"], s["scale_k"] = _codes(shape, g)
        s["v"], s["scale_v"] = _codes(shape, g)
        s["dst_k"], s["dst_v"] = (torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _attend, "append": _append, "quantize": _quantize, "dequantize": _dequantize}[state["case"]["op"]](state)


def _encode(x):
    """e4m3 codes and biased exponents of rows: the smallest power of two under which the row's largest value fits."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))
    e = e - 9 + (m > 0.875).to(e.dtype)                          # 448 = 0.875 * 2^9
    e = torch.where(m == 0, torch.full_like(e, -127), e.clamp(min=-127))
    down = ((127 - e) << 23).view(torch.float32)                 # 2^-e, exactly
    return (x * down[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _decode(code, e):
    scale = ((e.long() + (1023 - 127)) << 52).view(torch.float64)  # down to 2^-127: below float32's normal range
    return (code.double() * scale[..., None]).float()


def _quantize(s):
    ck, ek = _encode(s["src_k"])
    cv, ev = _encode(s["src_v"])
    outs = {"k": s["k"], "v": s["v"], "scale_k": s["scale_k"], "scale_v": s["scale_v"]}
    return _put(s, outs, {"k": ck, "v": cv, "scale_k": ek, "scale_v": ev})


def _dequantize(s):
    outs = {"k": s["dst_k"], "v": s["dst_v"]}
    return _put(s, outs, {"k": _decode(s["k"], s["scale_k"]).to(torch.bfloat16), "v": _decode(s["v"], s["scale_v"]).to(torch.bfloat16)})


def _put(s, outs, new):
    """Rows of the named pages (and of them the first `tokens`) replaced, everything else as it was."""
    c = s["case"]
    if not c["page"]:
        return {k: o.copy_(new[k]) for k, o in outs.items()}
    pages = s["k"].shape[1]
    at = torch.full((pages,), 1 << 30, dtype=torch.long, device=DEV)
    at[s["table"].long()] = torch.arange(s["table"].numel(), device=DEV) * c["page"]
    live = at[:, None] + torch.arange(c["page"], device=DEV) < c["tokens"]                    # [pages, page]
    live = live[None, :, :, None] if c["token_major"] else live[None, :, None, :]
    byte = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t
    return {k: byte(o).copy_(torch.where(live[..., None] if o.dim() == 5 else live, byte(new[k]), byte(o))).view(o.dtype)
            for k, o in outs.items()}


def _row_plan(s, rows):
    """Request of every packed row, its place among the request's new tokens, and whether it belongs to one."""
    n = s["kv_len"].numel()
    r = torch.arange(rows, device=DEV)
    req = torch.searchsorted(s["q_begin"][1:].long(), r, right=True)
    live = req < n
    req = req.clamp(max=n - 1)
    return req, torch.where(live, r - s["q_begin"][req].long(), 0), live


def _append(s):
    c = s["case"]
    req, i, _ = _row_plan(s, s["k_new"].shape[0])
    nq = (s["q_begin"][1:] - s["q_begin"][:-1]).long()
    pos = s["kv_len"].long()[req] - nq[req] + i
    page, slot = s["table"][req, pos // c["page"]].long(), pos % c["page"]
    if c["q8"]:
        (ck, ek), (cv, ev) = _encode(s["k_new"]), _encode(s["v_new"])
        new = {"k": ck, "v": cv, "scale_k": ek, "scale_v": ev}
    else:
        new = {"k": s["k_new"], "v": s["v_new"]}
    for name, x in new.items():
        pool = s[name][0]
        pool, x = (pool.view(torch.uint8), x.view(torch.uint8)) if x.element_size() == 1 else (pool, x)
        if c["token_major"]:
            pool[page, slot] = x
        else:
            pool[page, :, slot] = x
    return {k: s[k] for k in new}


def _dense(s, name):
    """Keys or values of all requests in float32, [n, h, max_kv, d]."""
    c = s["case"]
    t = s["table"].long()
    pool = s[name][0]
    x = _decode(pool.view(torch.uint8)[t].view(torch.float8_e4m3fn), s["scale_" + name][0][t]) if c["q8"] else pool[t].float()
    if not c["token_major"]:
        x = x.transpose(2, 3)                                                                # [n, per, page, h, d]
    return x.reshape(c["n"], -1, c["h"], c["d"])[:, : s["max_kv"]].transpose(1, 2)


def _attend(s):
    c = s["case"]
    n, h, d, g = c["n"], c["h"], c["d"], c["hq"] // c["h"]
    rows = s["q"].shape[0]
    begin, kv = s["q_begin"].long(), s["kv_len"].long()
    nq = begin[1:] - begin[:-1]
    i = torch.arange(s["max_q"], device=DEV)
    q = s["q"][(begin[:-1, None] + i).clamp(max=rows - 1)].float()                           # [n, max_q, hq, d]
    q = q.view(n, -1, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, -1, d)                   # [n, h, g max_q, d]
    score = torch.matmul(q, _dense(s, "k").transpose(2, 3)).view(n, h, g, s["max_q"], -1)
    score *= 1.0 / math.sqrt(d)
    t = torch.arange(s["max_kv"], device=DEV)
    seen = t[None, None, :] < kv[:, None, None]
    if c["causal"]:
        seen = seen & (t[None, None, :] <= (kv - nq)[:, None, None] + i[None, :, None])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (score - top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, -1, p.shape[-1]), _dense(s, "v")).view(n, h, g, -1, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, -1, c["hq"], d)
    req, at, live = _row_plan(s, rows)
    out = {"out": s["out"].copy_(torch.where(live[:, None, None], o[req, at].to(torch.bfloat16), s["out"]))}
    if c["lse"]:
        lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n, -1, c["hq"])
        out["lse"] = s["lse"].copy_(torch.where(live[:, None], lse[req, at], s["lse"]))
    return out


def _handles(s):
    """The descriptors and the scratch that a program keeps beside its buffers."""
    if "handles" in s:
        return s["handles"]
    import paper_2609_34060_b200 as kvc
    c, tm = s["case"], s["case"]["token_major"]
    hd = {"kvc": kvc}
    if c["op"] in ("attend", "append"):
        hd["req"] = kvc.Requests(s["q_begin"], s["kv_len"], s["max_q"], s["max_kv"], page_table=s["table"])
        hd["cache"] = (kvc.QCache.pool(s["k"], s["v"], s["scale_k"], s["scale_v"], token_major=tm) if c["q8"]
                       else kvc.Cache.pool(s["k"], s["v"], token_major=tm))
        if c["op"] == "attend":
            hd["workspace"] = torch.empty(kvc.kvc_attend_workspace_bytes(hd["req"], hd["cache"], c["hq"]), dtype=torch.uint8, device=DEV)
    else:
        t = None if s["table"] is None else c["tokens"]
        hd["q8"] = kvc.QCache(s["k"], s["v"], s["scale_k"], s["scale_v"], T=t, page_table=s["table"], token_major=tm)
        k, v = (s["src_k"], s["src_v"]) if c["op"] == "quantize" else (s["dst_k"], s["dst_v"])
        hd["bf16"] = kvc.Cache(k, v, T=t, page_table=s["table"], token_major=tm)
    s["handles"] = hd
    return hd


def _run_own(s):
    c, hd = s["case"], _handles(s)
    kvc = hd["kvc"]
    if c["op"] == "attend":
        kvc.kvc_attend(hd["req"], s["q"], hd["cache"], 0, s["out"], hd["workspace"], causal=c["causal"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    if c["op"] == "append":
        kvc.kvc_append(hd["req"], s["k_new"], s["v_new"], hd["cache"], 0)
        return {k: s[k] for k in (("k", "v", "scale_k", "scale_v") if c["q8"] else ("k", "v"))}
    if c["op"] == "quantize":
        kvc.kvc_quantize(hd["bf16"], hd["q8"])
        return {k: s[k] for k in ("k", "v", "scale_k", "scale_v")}
    kvc.kvc_dequantize(hd["q8"], hd["bf16"])
    return {"k": s["dst_k"], "v": s["dst_v"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    if c["op"] in ("quantize", "dequantize"):
        rows = 2.0 * c["layers"] * c["h"] * c["tokens"]
        return {"bytes": rows * (3 * c["d"] + 1), "flops": rows * 2 * c["d"]}
    nq, kv = _lengths(c)
    row = c["d"] + 1.0 if c["q8"] else 2.0 * c["d"]
    if c["op"] == "append":
        rows = 2.0 * sum(nq) * c["h"]
        return {"bytes": rows * (2 * c["d"] + row), "flops": rows * 2 * c["d"]}
    seen = sum(m * t - (m * (m - 1) // 2 if c["causal"] else 0) for m, t in zip(nq, kv))     # (row, key) pairs
    return {"bytes": 2.0 * c["h"] * sum(kv) * row + sum(nq) * c["hq"] * (4.0 * c["d"] + (4 if c["lse"] else 0)),
            "flops": 4.0 * c["hq"] * seen * c["d"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append}.get(case["op"], _exact_convert)(s)


def _exact_code(x):
    """Nearest e4m3 value (ties to even) of x / 2^e, as float64, and 2^e: e from the row's largest magnitude."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448.0))
    e = torch.where(448.0 * _two(e - 1) >= top, e - 1, e)
    e = torch.where(448.0 * _two(e) < top, e + 1, e)
    e = torch.where(top > 0, e.clamp(min=-127), -127.0)
    y = x / _two(e)
    step = _two(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _two(e):
    """2^e for whole e, exactly (a power function may be off by its last bit)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_value(code, e):
    return code.float().double() * _two(e.double() - 127.0).unsqueeze(-1)


def _exact_convert(s):
    c = s["case"]
    if c["op"] == "quantize":
        full = {"k": _exact_code(s["src_k"]), "v": _exact_code(s["src_v"])}
    else:
        full = {"k": _exact_value(s["k"], s["scale_k"]), "v": _exact_value(s["v"], s["scale_v"])}
    if c["page"]:
        for name, x in full.items():
            keep = torch.zeros_like(x)
            for j, p in enumerate(s["table"].tolist()):
                m = min(c["page"], c["tokens"] - j * c["page"])
                if c["token_major"]:
                    keep[:, p, :m] = x[:, p, :m]
                else:
                    keep[:, p, :, :m] = x[:, p, :, :m]
            full[name] = keep
    return dict(full, scale_k=None, scale_v=None) if c["op"] == "quantize" else full


def _exact_append(s):
    c = s["case"]
    out = {}
    for name in ("k", "v"):
        pool = s[name][0].float().double()
        new = _exact_code(s[name + "_new"]) if c["q8"] else s[name + "_new"].double()
        begin, kv, table = s["q_begin"].tolist(), s["kv_len"].tolist(), s["table"].long()
        for b in range(c["n"]):
            m = begin[b + 1] - begin[b]
            pos = torch.arange(kv[b] - m, kv[b], device=DEV)
            page, slot = table[b][pos // c["page"]], pos % c["page"]
            if c["token_major"]:
                pool[page, slot] = new[begin[b]: begin[b + 1]]
            else:
                pool[page, :, slot] = new[begin[b]: begin[b + 1]]
        out[name] = pool[None]
    return dict(out, scale_k=None, scale_v=None) if c["q8"] else out


def _exact_attend(s):
    c = s["case"]
    g = c["hq"] // c["h"]
    begin, kv = s["q_begin"].tolist(), s["kv_len"].tolist()
    out = s["out"].double()
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEV)
    for b in range(c["n"]):
        m, length = begin[b + 1] - begin[b], kv[b]
        pages = s["table"][b, : -(-length // c["page"])].long()
        side = {}
        for name in ("k", "v"):
            x = s[name][0].view(torch.uint8)[pages].view(torch.float8_e4m3fn) if c["q8"] else s[name][0][pages]
            x = _exact_value(x, s["scale_" + name][0][pages]) if c["q8"] else x.double()
            x = x if c["token_major"] else x.permute(0, 2, 1, 3)
            side[name] = x.reshape(-1, c["h"], c["d"])[:length]
        last = (length - m + torch.arange(m, device=DEV))[:, None] if c["causal"] else length
        hidden = torch.arange(length, device=DEV)[None, :] > last if c["causal"] else None
        for head in range(c["hq"]):
            z = s["q"][begin[b]: begin[b + 1], head].double() @ side["k"][:, head // g].T / math.sqrt(c["d"])
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(z, -1)
            w = torch.exp(z - torch.where(norm == -math.inf, 0.0, norm)[:, None])
            out[begin[b]: begin[b + 1], head] = w @ side["v"][:, head // g]
            lse[begin[b]: begin[b + 1], head] = norm
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
