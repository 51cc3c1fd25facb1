"""Operators of a step of drafted tokens over a cache: measured cases and plain forms.

``kvc_tree_build`` (masks and depths of the drafted tokens from their parents), ``kvc_append_rotated`` (queries and keys
turned to their positions, keys and values written into the cache), ``kvc_attend_tree`` (attention of a tree of drafted
tokens over a cache), ``kvc_verify`` (which of them stay, and the next token) and ``kvc_keep`` (their rows put together in
the cache).  ``run`` computes a case with elementary torch operations, or, where ``own`` is true, with the calls a user
makes of the library.
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
        # one request's tree of drafts, once a step: latency
        dict(name="build_one", op="build", n=1, q_lo=24, q_hi=24, shape="tree"),
        # a large serving batch, trees of up to 200 drafts
        dict(name="build_batch", op="build", n=192, q_lo=40, q_hi=200, shape="tree"),
        # a decode step: 64 requests' single tokens into 8-bit pages, 8K-context model: latency
        dict(name="rotate_tokens_q8", op="rotate", n=64, q_lo=1, q_hi=1, shape="chain", hq=32, h=8, d=128, page=16, kv=1024,
             kv_max=2048, q8=True, token_major=False, rot=128, pairing="half", theta=500000.0, factor=1.0, far=0),
        # trees of drafts behind medium contexts, half of each head rotated in interleaved pairs
        dict(name="rotate_trees_part", op="rotate", n=32, q_lo=9, q_hi=63, shape="tree", hq=32, h=4, d=128, page=16, kv=700,
             kv_max=1400, q8=False, token_major=True, rot=64, pairing="interleaved", theta=10000.0, factor=1.0, far=0),
        # prompts of an image model written into bf16 pages, frequencies scaled for four times the trained length, positions
        # far beyond it
        dict(name="rotate_prompts_scaled", op="rotate", n=5, q_lo=1500, q_hi=2500, shape="chain", hq=28, h=4, d=128, page=16, kv=2900,
             kv_max=4096, q8=False, token_major=False, rot=128, pairing="half", theta=1000000.0, factor=4.0, far=120000),
        # one request's drafts over a short context: latency
        dict(name="attend_one", op="attend", n=1, q_lo=13, q_hi=13, shape="tree", hq=32, h=8, d=128, page=16, kv=777, kv_max=777,
             q8=False, token_major=False, lse=False, spare=0),
        # a serving batch over 4K contexts, 32 drafts each
        dict(name="attend_batch", op="attend", n=24, q_lo=32, q_hi=32, shape="tree", hq=32, h=8, d=128, page=16, kv=4096, kv_max=8192,
             q8=False, token_major=False, lse=False, spare=0),
        # agents of the long-context shape, 7 drafts each over 32K in 8 bits, log-sum-exps kept
        dict(name="attend_long_q8", op="attend", n=4, q_lo=5, q_hi=9, shape="tree", hq=64, h=8, d=128, page=16, kv=32000, kv_max=32768,
             q8=True, token_major=False, lse=True, spare=3),
        # one request, a chain of five drafts, a small vocabulary: latency
        dict(name="verify_one", op="verify", n=1, q_lo=6, q_hi=6, shape="chain", vocab=32000, drafts=True),
        # a serving batch, trees of drafts, a large vocabulary
        dict(name="verify_batch", op="verify", n=64, q_lo=8, q_hi=16, shape="tree", vocab=128000, drafts=True),
        # one request's accepted drafts put together in every layer of a bf16 pool: latency
        dict(name="keep_one", op="keep", n=1, q_lo=24, q_hi=24, kept=5, layers=32, h=8, d=128, page=16, kv=500, q8=False, token_major=False),
        # a serving batch in 8-bit pages
        dict(name="keep_batch_q8", op="keep", n=64, q_lo=20, q_hi=40, kept=6, layers=32, h=8, d=128, page=16, kv=160, q8=True,
             token_major=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["build", "rotate", "rotate", "attend", "attend", "attend", "verify", "verify", "keep"])
    shape = rng.choice(["tree", "tree", "chain"])
    d, page = rng.choice([64, 128, 128]), rng.choice([8, 16, 16, 32, 64, 128])
    q_hi = _log_int(rng, 1, 200)
    q_lo = rng.randint(1, q_hi)
    if op == "build":
        q_hi = max(q_hi, 12)
        return dict(op=op, n=_log_int(rng, 1, 192), q_lo=rng.randint(12, q_hi), q_hi=q_hi, shape="tree")
    h = rng.choice([1, 2, 4, 8])
    if op == "rotate":
        g, n = rng.choice([1, 2, 3, 4, 7, 8]), _log_int(rng, 1, 64)
        if rng.random() < 0.4:                                    # prompts
            shape, q_hi = "chain", _log_int(rng, 16, 9000 // n + 17)
            q_lo = max(1, q_hi // 2)
        kv = q_hi + _log_int(rng, 1, 1000)
        return dict(op=op, n=n, q_lo=q_lo, q_hi=q_hi, shape=shape, hq=h * g, h=h, d=d, page=page, kv=kv, kv_max=2 * kv, q8=rng.random() < 0.5,
                    token_major=rng.random() < 0.3, rot=rng.choice([d, d, d // 2, d // 4, 16]), pairing=rng.choice(["half", "half", "interleaved"]),
                    theta=rng.choice([10000.0, 500000.0, 1000000.0]), factor=rng.choice([1.0, 1.0, 4.0, 16.0]), far=rng.choice([0, 0, 50000, 1000000]))
    if op == "attend":
        g, n = rng.choice([1, 2, 3, 4, 7, 8]), _log_int(rng, 1, 48)
        kv = _log_int(rng, q_hi, 24000)
        kv_max = max(kv, q_hi) if n == 1 else max(q_hi, min(2 * kv, 32768))
        while n * kv_max * h > 1500000:
            n = max(1, n // 2)
        while g > 1 and n * q_hi * h * g * kv_max > 250000000:
            g -= 1
        while n > 1 and n * q_hi * h * g * kv_max > 250000000:
            n -= 1
        return dict(op=op, n=n, q_lo=q_lo, q_hi=q_hi, shape=shape, hq=h * g, h=h, d=d, page=page, kv=kv, kv_max=kv_max, q8=rng.random() < 0.5,
                    token_major=rng.random() < 0.3, lse=rng.random() < 0.5, spare=rng.choice([0, 0, 5]))
    if op == "verify":
        vocab, drafts = _log_int(rng, 1000, 128000), rng.random() < 0.75
        q_hi = _log_int(rng, 1, 24)
        return dict(op=op, n=max(1, min(_log_int(rng, 1, 96), 130000000 // (q_hi * vocab))), q_lo=rng.randint(1, q_hi), q_hi=q_hi, shape=shape, vocab=vocab,
                    drafts=drafts)
    return dict(op=op, n=_log_int(rng, 1, 64), q_lo=q_lo, q_hi=q_hi, kept=_log_int(rng, 1, 12), layers=rng.randint(1, 28), h=h, d=d, page=page,
                kv=q_hi + _log_int(rng, 1, 60), q8=rng.random() < 0.5, token_major=rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


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


def _codes(shape, g):
    """Codes as a quantised cache holds them (normal rows under their power-of-two scale) and exponents near 1."""
    x = torch.empty(shape, dtype=torch.float32, device=DEV).normal_(generator=g) * 110.0
    x = x.clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    e = torch.randint(118, 121, shape[:-1], device=DEV, generator=g, dtype=torch.int32).to(torch.uint8)
    return x, e


def _rng(c):
    return random.Random(" ".join("%s=%s" % kv for kv in sorted(c.items()) if kv[0] != "name"))


def _lengths(c):
    """New tokens and cache lengths of the requests: the case's own, whatever the seed (buffers keep their shapes)."""
    rng = _rng(c)
    nq = [rng.randint(c["q_lo"], c["q_hi"]) for _ in range(c["n"])]
    top = c.get("kv_max", 4 * c.get("kv", 1))
    kv = [int(round(c.get("kv", 0) * math.exp((0.0 if c["n"] == 1 else 0.3) * rng.gauss(0.0, 1.0)))) for _ in range(c["n"])]
    return nq, [max(1, m, min(t, top)) for m, t in zip(nq, kv)]


def _kept_lists(c):
    """Accepted rows of every request, the case's own: row 0, then ascending ones.  Rows that a move would overwrite are not
    among those it reads (a second pass over one state finds the same rows)."""
    rng, (nq, _) = _rng(c), _lengths(c)
    lists = []
    for m in nq:
        want = min(rng.randint(1, 2 * c["kept"] - 1), m)
        stay = rng.randint(1, max(1, want // 2))
        far = range(want, m)
        lists.append(list(range(stay)) + sorted(rng.sample(far, min(want - stay, len(far)))))
    return lists


def _parents(c, nq, g):
    """Parents [n, max_q] of the drafts: row 0 follows the cache; a tree's row one of the earlier rows (near ones more
    often), a chain's the one before it; -2 behind the request's rows."""
    q = max(nq)
    j = torch.arange(q, device=DEV)[None, :].expand(len(nq), q)
    if c["shape"] == "chain":
        par = j - 1
    else:
        back = torch.rand(len(nq), q, device=DEV, generator=g) ** 1.5
        par = torch.minimum(j - 1, (j - 1 - (back * j).floor()).long()).clamp(min=0)
    par = torch.where(j == 0, -1, par)
    return torch.where(j < torch.tensor(nq, device=DEV)[:, None], par, -2)


def _packed(dense, nq):
    """[n, max_q, ...] -> the requests' rows one after the other."""
    live = torch.arange(dense.shape[1], device=DEV)[None, :] < torch.tensor(nq, device=DEV)[:, None]
    return dense[live]


def _reach(par):
    """reach[b, j, a]: whether row a is row j or an ancestor of it."""
    n, q = par.shape
    link = torch.zeros(n, q, q + 1, device=DEV).scatter_(2, torch.where(par >= 0, par, q).long()[..., None], 1.0)[:, :, :q]
    reach = link + torch.eye(q, device=DEV)
    for _ in range(max(1, (q - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()
    return reach


def _words(reach):
    """Rows of bits as 32-bit words."""
    n, q, _ = reach.shape
    w = -(-q // 32)
    bits = torch.nn.functional.pad(reach, (0, 32 * w - q)).view(n, q, w, 32).long()
    v = (bits << torch.arange(32, device=DEV)).sum(-1)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).to(torch.int32)


def frequencies(c):
    """Frequencies of the rotated pairs, scaled "by parts": pairs that turn often over the trained length keep theirs, slow
    ones are divided by the factor, in between a linear mix in the number of turns; and the amplitude that goes with it."""
    f = [c["theta"] ** (-2.0 * k / c["rot"]) for k in range(c["rot"] // 2)]
    if c["factor"] == 1.0:
        return f, 1.0
    keep = [min(1.0, max(0.0, (8192.0 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
    return [x * (w + (1.0 - w) / c["factor"]) for x, w in zip(f, keep)], 0.1 * math.log(c["factor"]) + 1.0


def _pool(c, s, nq, kv, layers, g):
    """Pages of all requests, shuffled, and their tables."""
    s["max_q"], s["max_kv"] = max(nq), max(kv)
    nq, kv = torch.tensor(nq, device=DEV), torch.tensor(kv, device=DEV)
    per = -(-s["max_kv"] // c["page"])                            # table entries of a request
    need = (kv + c["page"] - 1) // c["page"]
    pages = int(need.sum()) + 3
    perm = torch.rand(pages, device=DEV, generator=g).argsort()
    col = torch.arange(per, device=DEV)[None, :]
    first = torch.cumsum(need, 0) - need
    s["table"] = torch.where(col < need[:, None], perm[(first[:, None] + col).clamp(max=pages - 1)], 0).to(torch.int32)
    s["q_begin"] = torch.cat([nq.new_zeros(1), torch.cumsum(nq, 0)]).to(torch.int32)
    s["kv_len"] = kv.to(torch.int32)
    shape = (layers, pages, c["page"], c["h"], c["d"]) if c["token_major"] else (layers, pages, c["h"], c["page"], c["d"])
    if c["q8"]:
        s["k"], s["scale_k"] = _codes(shape, g)
        s["v"], s["scale_v"] = _codes(shape, g)
    else:
        s["k"], s["v"] = _rows(shape, g, 3 if c["token_major"] else 2), _rows(shape, g)
    return int(nq.sum())


def _distributions(rows, vocab, g):
    """Two related distributions a row: softmax of normal logits, small probabilities cut off."""
    z = torch.empty(rows, vocab, device=DEV).normal_(generator=g).mul_(3.0)

    def soft(z):
        p = torch.softmax(z, -1)
        p = torch.where(p >= p.amax(-1, keepdim=True) * 1e-5, p, 0.0)
        return p / p.sum(-1, keepdim=True)

    p = soft(z)
    z += torch.empty_like(z).normal_(generator=g)
    return p, soft(z)


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    nq, kv = _lengths(c)
    rows = sum(nq)
    s["max_q"], s["max_kv"] = max(nq), max(kv)
    s["q_begin"] = torch.tensor([sum(nq[:i]) for i in range(len(nq) + 1)], dtype=torch.int32, device=DEV)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=DEV)
    if c["op"] == "keep":
        lists = _kept_lists(c)
        _pool(c, s, nq, kv, c["layers"], g)
        s["kept"] = torch.tensor([x + [-1] * (s["max_q"] - len(x)) for x in lists], dtype=torch.int32, device=DEV)
        s["n_kept"] = torch.tensor([len(x) for x in lists], dtype=torch.int32, device=DEV)
        s["kv_out"] = torch.zeros_like(s["kv_len"])
        return s
    par = _parents(c, nq, g)
    s["parent"] = _packed(par, nq).to(torch.int32)
    words = -(-s["max_q"] // 32)
    if c["op"] == "build":
        s["mask"] = torch.zeros(rows, words, dtype=torch.int32, device=DEV)
        s["depth"] = torch.zeros(rows, dtype=torch.int32, device=DEV)
        return s
    if c["op"] == "verify":
        s["target"], s["draft"] = _distributions(rows, c["vocab"], g)
        at = torch.arange(rows, device=DEV)
        first = torch.repeat_interleave(s["q_begin"][:-1].long(), torch.tensor(nq, device=DEV))
        above = torch.where(s["parent"] >= 0, first + s["parent"].long(), at)
        cdf = torch.cumsum(s["draft"], -1)
        pick = torch.rand(rows, device=DEV, generator=g) * cdf[above, -1] * 0.9999
        s["token"] = torch.searchsorted(cdf[above], pick[:, None], right=True)[:, 0].clamp(max=c["vocab"] - 1).to(torch.int32)
        if not c["drafts"]:
            s["draft"] = None
        s["u"] = torch.rand(rows, device=DEV, generator=g)
        s["u_next"] = torch.rand(c["n"], device=DEV, generator=g)
        s["kept"] = torch.zeros(c["n"], s["max_q"], dtype=torch.int32, device=DEV)
        s["n_kept"], s["next"] = (torch.zeros(c["n"], dtype=torch.int32, device=DEV) for _ in range(2))
        return s
    _pool(c, s, nq, kv, 1, g)
    if c["op"] == "attend" or c["shape"] == "tree":
        reach = _reach(par)
        s["depth"], s["mask"] = _packed((reach.sum(-1) - 1).to(torch.int32), nq), _packed(_words(reach), nq)
    else:
        s["depth"] = s["parent"] + 1
    rows += c.get("spare", 0)
    if c["op"] == "attend" and c["spare"]:
        pad = torch.nn.functional.pad
        s["mask"], s["depth"], s["parent"] = pad(s["mask"], (0, 0, 0, c["spare"])), pad(s["depth"], (0, c["spare"])), pad(s["parent"], (0, c["spare"]))
    s["q"] = _rows((rows, c["hq"], c["d"]), g)
    s["out"] = torch.zeros_like(s["q"])
    if c["op"] == "attend":
        s["lse"] = torch.zeros(rows, c["hq"], dtype=torch.float32, device=DEV) if c["lse"] else None
        return s
    s["k_new"], s["v_new"] = _rows((rows, c["h"], c["d"]), g, 1), _rows((rows, c["h"], c["d"]), g)
    s["pos_begin"] = torch.randint(0, c["far"] + 1, (c["n"],), device=DEV, generator=g, dtype=torch.int32) if c["far"] else None
    s["freq"], s["amplitude"] = frequencies(c)
    s["freq_dev"] = torch.tensor(s["freq"], dtype=torch.float64, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(state):
    if own:
        return _run_own(state)
    return {"build": _build, "rotate": _rotate, "attend": _attend, "verify": _verify, "keep": _keep}[state["case"]["op"]](state)


def _row_plan(s, rows):
    """Request of every packed row, its place among the request's new tokens, and whether it belongs to one."""
    n = s["kv_len"].numel()
    r = torch.arange(rows, device=DEV)
    req = torch.searchsorted(s["q_begin"][1:].long(), r, right=True)
    live = req < n
    req = req.clamp(max=n - 1)
    return req, torch.where(live, r - s["q_begin"][req].long(), 0), live


def _by_request(s, x, fill):
    """Packed rows -> [n, max_q, ...]."""
    begin = s["q_begin"].long()
    i = torch.arange(s["max_q"], device=DEV)
    at = begin[:-1, None] + i
    dense = x[at.clamp(max=x.shape[0] - 1)]
    live = at < begin[1:, None]
    return torch.where(live.view(live.shape + (1,) * (dense.dim() - 2)), dense, fill)


def _build(s):
    reach = _reach(_by_request(s, s["parent"], -2))
    req, at, _ = _row_plan(s, s["parent"].shape[0])
    return {"mask": s["mask"].copy_(_words(reach)[req, at]), "depth": s["depth"].copy_((reach.sum(-1) - 1)[req, at])}


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


def _turned(c, x, cos, sin):
    """The first `rot` channels of rows [rows, heads, d] rotated, in float32."""
    x, r = x.float(), c["rot"]
    a, b = (x[..., : r // 2], x[..., r // 2: r]) if c["pairing"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([y, z], -1) if c["pairing"] == "half" else torch.stack([y, z], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _write(c, s, req, pos, new):
    page, slot = s["table"][req, pos // c["page"]].long(), pos % c["page"]
    for name, x in new.items():
        pool = s[name][0]
        pool, x = (pool.view(torch.uint8), x.view(torch.uint8)) if x.element_size() == 1 else (pool, x)
        if c["token_major"]:
            pool[page, slot] = x
        else:
            pool[page, :, slot] = x
    return {k: s[k] for k in new}


def _rotate(s):
    c = s["case"]
    req, place, _ = _row_plan(s, s["q"].shape[0])
    nq = (s["q_begin"][1:] - s["q_begin"][:-1]).long()
    first = (s["kv_len"].long() - nq)[req]
    pos = first + s["depth"] + (s["pos_begin"].long()[req] if c["far"] else 0)
    angle = pos.double()[:, None] * s["freq_dev"]
    cos, sin = ((f(angle) * s["amplitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    k = _turned(c, s["k_new"], cos, sin)
    if c["q8"]:
        (ck, ek), (cv, ev) = _encode(k), _encode(s["v_new"])
        new = {"k": ck, "v": cv, "scale_k": ek, "scale_v": ev}
    else:
        new = {"k": k.to(torch.bfloat16), "v": s["v_new"]}
    return dict(_write(c, s, req, first + place, new), q=s["out"].copy_(_turned(c, s["q"], cos, sin)))


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
    begin, kv = s["q_begin"].long(), s["kv_len"].long()
    first = kv - (begin[1:] - begin[:-1])
    q = _by_request(s, s["q"], 0).float()                                                    # [n, max_q, hq, d]
    q = q.view(n, -1, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, -1, d)                   # [n, h, g max_q, d]
    score = torch.matmul(q, _dense(s, "k").transpose(2, 3)).view(n, h, g, s["max_q"], -1)
    score *= 1.0 / math.sqrt(d)
    t = torch.arange(s["max_kv"], device=DEV)
    words = _by_request(s, s["mask"], 0).long()                                              # [n, max_q, words]
    a = (t[None, :] - first[:, None])[:, None, :].expand(n, s["max_q"], -1)                  # key's place among the new tokens
    bit = torch.gather(words, 2, (a >> 5).clamp(0, words.shape[2] - 1)) >> (a & 31) & 1
    seen = torch.where(a < 0, True, (bit == 1) & (t < kv[:, None])[:, None, :])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (score - top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, h, -1, p.shape[-1]), _dense(s, "v")).view(n, h, g, -1, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, -1, c["hq"], d)
    req, at, live = _row_plan(s, s["q"].shape[0])
    out = {"out": s["out"].copy_(torch.where(live[:, None, None], o[req, at].to(torch.bfloat16), s["out"]))}
    if c["lse"]:
        lse = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n, -1, c["hq"])
        out["lse"] = s["lse"].copy_(torch.where(live[:, None], lse[req, at], s["lse"]))
    return out


def _verify(s):
    """All requests at once: the rows in their order (a row's children lie behind it), each tried where its parent is the
    request's current node.  Sums and comparisons in 64 bits."""
    c = s["case"]
    n, v = c["n"], c["vocab"]
    begin = s["q_begin"].long()
    nq, last = begin[1:] - begin[:-1], s["parent"].shape[0] - 1
    par, tok, u = _by_request(s, s["parent"], -2), _by_request(s, s["token"], 0).long(), _by_request(s, s["u"], 1.0).double()
    node = torch.zeros(n, dtype=torch.long, device=DEV)
    one, zero = torch.ones(n, dtype=torch.float64, device=DEV), torch.zeros(n, dtype=torch.float64, device=DEV)
    a, b, spent = one, zero, torch.zeros(n, dtype=torch.bool, device=DEV)                    # P = max(a p - b q, 0)
    gone = torch.zeros(n, v, dtype=torch.bool, device=DEV)
    stays = torch.zeros(n, s["max_q"], dtype=torch.bool, device=DEV)
    stays[:, 0] = True
    for i in range(1, s["max_q"]):
        row, x = (begin[:-1] + node).clamp(max=last), tok[:, i]
        asked = (par[:, i] == node) & ~spent
        px = s["target"][row, x].double()
        if s["draft"] is not None:
            qx = s["draft"][row, x].double()
            ok = u[:, i] * qx < (px * a - qx * b).clamp(min=0)
            z = (s["target"][row].double() * a[:, None] - s["draft"][row].double() * (b + 1)[:, None]).clamp_(min=0).sum(-1)
            no, more = asked & ~ok, z > 0
            a, b = torch.where(no, torch.where(more, a / z, one), a), torch.where(no, torch.where(more, (b + 1) / z, zero), b)
            spent = spent | (no & ~more)
        else:
            fresh = ~gone.gather(1, x[:, None])[:, 0]
            ok = (u[:, i] * a < px) & fresh                                                  # a: what is left of one
            no = asked & ~ok
            a = torch.where(no & fresh, a - px, a)
            gone.scatter_(1, x[:, None], (gone.gather(1, x[:, None])[:, 0] | no)[:, None])
        yes = asked & ok
        node, a, b = torch.where(yes, i, node), torch.where(yes, one, a), torch.where(yes, zero, b)
        gone &= ~yes[:, None]
        stays[:, i] = yes
    row = begin[:-1] + node
    p = s["target"][row].double()
    w = (p * a[:, None] - s["draft"][row].double() * b[:, None]).clamp_(min=0) if s["draft"] is not None else torch.where(gone, 0.0, p)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, p)
    cdf = torch.cumsum(w, -1)
    nxt = (cdf <= s["u_next"].double()[:, None] * cdf[:, -1:]).sum(-1).clamp(max=v - 1)
    i = torch.arange(s["max_q"], device=DEV)
    path = torch.where(stays, i, 1 << 30).sort(-1).values
    count = stays.sum(-1)
    return {"kept": s["kept"].copy_(torch.where(path < 1 << 30, path, -1)), "n_kept": s["n_kept"].copy_(count), "next": s["next"].copy_(nxt)}


def _keep(s):
    c = s["case"]
    first = (s["kv_len"] - (s["q_begin"][1:] - s["q_begin"][:-1])).long()[:, None]
    j = torch.arange(s["max_q"], device=DEV)[None, :]
    live = j < s["n_kept"][:, None]
    src, dst = (torch.where(live, first + x, first).flatten() for x in (s["kept"], j))       # others: row 0 onto itself
    req = torch.arange(c["n"], device=DEV)[:, None].expand(-1, s["max_q"]).flatten()
    (sp, sr), (dp, dr) = ((s["table"][req, x // c["page"]].long(), x % c["page"]) for x in (src, dst))
    names = ("k", "v", "scale_k", "scale_v") if c["q8"] else ("k", "v")
    for name in names:
        pool = s[name].view(torch.uint8) if c["q8"] else s[name]
        if c["token_major"]:
            pool[:, dp, dr] = pool[:, sp, sr]
        else:
            pool[:, dp, :, dr] = pool[:, sp, :, sr]
    return dict({k: s[k] for k in names}, kv_out=s["kv_out"].copy_(first[:, 0] + s["n_kept"]))


def _handles(s):
    """The descriptors and the scratch that a program keeps beside its buffers."""
    if "handles" in s:
        return s["handles"]
    import paper_2609_34060_b200 as kvc
    c = s["case"]
    hd = {"kvc": kvc}
    hd["req"] = kvc.Requests(s["q_begin"], s["kv_len"], s["max_q"], s["max_kv"], page_table=s.get("table"))
    if c["op"] in ("rotate", "attend", "keep"):
        hd["cache"] = (kvc.QCache.pool(s["k"], s["v"], s["scale_k"], s["scale_v"], token_major=c["token_major"]) if c["q8"]
                       else kvc.Cache.pool(s["k"], s["v"], token_major=c["token_major"]))
    if c["op"] in ("build", "attend"):
        hd["tree"] = kvc.Tree(s["parent"], s["max_q"], mask=s["mask"], depth=s["depth"])
    if c["op"] == "attend":
        hd["workspace"] = torch.empty(kvc.kvc_attend_workspace_bytes(hd["req"], hd["cache"], c["hq"]), dtype=torch.uint8, device=DEV)
    if c["op"] == "rotate":
        pairing = kvc.KVC_ROPE_HALF if c["pairing"] == "half" else kvc.KVC_ROPE_INTERLEAVED
        hd["rotary"] = kvc.Rotary(kvc.Rope(c["theta"], pairing, inv_freq=s["freq"]), rot_dim=c["rot"], amplitude=s["amplitude"],
                                  depth=s["depth"], pos_begin=s["pos_begin"])
    s["handles"] = hd
    return hd


def _run_own(s):
    c, hd = s["case"], _handles(s)
    kvc = hd["kvc"]
    if c["op"] == "build":
        kvc.kvc_tree_build(hd["req"], hd["tree"])
        return {"mask": s["mask"], "depth": s["depth"]}
    if c["op"] == "rotate":
        kvc.kvc_append_rotated(hd["req"], hd["rotary"], s["k_new"], s["v_new"], hd["cache"], 0, q=s["q"], q_out=s["out"])
        return dict({k: s[k] for k in (("k", "v", "scale_k", "scale_v") if c["q8"] else ("k", "v"))}, q=s["out"])
    if c["op"] == "attend":
        kvc.kvc_attend_tree(hd["req"], hd["tree"], s["q"], hd["cache"], 0, s["out"], hd["workspace"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    if c["op"] == "verify":
        kvc.kvc_verify(hd["req"], s["parent"], s["token"], s["target"], s["u"], s["u_next"], s["kept"], s["n_kept"], s["next"], draft=s["draft"])
        return {k: s[k] for k in ("kept", "n_kept", "next")}
    kvc.kvc_keep(hd["req"], s["kept"], s["n_kept"], hd["cache"], s["kv_out"])
    return {k: s[k] for k in (("k", "v", "scale_k", "scale_v") if c["q8"] else ("k", "v")) + ("kv_out",)}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    nq, kv = _lengths(c)
    rows = float(sum(nq))
    if c["op"] == "build":
        words = -(-max(nq) // 32)
        return {"bytes": rows * (8 + 4 * words), "flops": rows * words}
    if c["op"] == "verify":                                       # the rows that the next token is drawn from
        return {"bytes": c["n"] * c["vocab"] * (8.0 if c["drafts"] else 4.0) + rows * 12, "flops": c["n"] * c["vocab"] * 3.0}
    row = c["d"] + 1.0 if c["q8"] else 2.0 * c["d"]
    if c["op"] == "keep":
        moved = sum(i != j for x in _kept_lists(c) for i, j in enumerate(x))
        return {"bytes": 4.0 * moved * c["layers"] * c["h"] * row + 12.0 * c["n"], "flops": 0.0}
    if c["op"] == "rotate":
        return {"bytes": rows * (4.0 * c["d"] * c["hq"] + 2 * c["h"] * (2 * c["d"] + row)), "flops": rows * (c["hq"] + c["h"]) * 3.0 * c["rot"]}
    # every row sees its context and its ancestors: a tree's depth is about the logarithm of its size
    seen = sum(m * (t - m) + m * ((m + 1) / 2 if c["shape"] == "chain" else 1 + math.log(m)) for m, t in zip(nq, kv))
    return {"bytes": 2.0 * c["h"] * sum(kv) * row + rows * c["hq"] * (4.0 * c["d"] + (4 if c["lse"] else 0)), "flops": 4.0 * c["hq"] * seen * c["d"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    if case["op"] not in ("rotate", "attend"):                    # whole numbers and copies
        return None
    return {"rotate": _exact_rotate, "attend": _exact_attend}[case["op"]](prepare(case, seed))


def _two(e):
    """2^e for whole e, exactly (a power function may be off by its last bit)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_code(x):
    """Nearest e4m3 value (ties to even) of x / 2^e, as float64: e from the row's largest magnitude."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448.0))
    e = torch.where(448.0 * _two(e - 1) >= top, e - 1, e)
    e = torch.where(448.0 * _two(e) < top, e + 1, e)
    e = torch.where(top > 0, e.clamp(min=-127), -127.0)
    y = x / _two(e)
    step = _two(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_rotate(s):
    c, r = s["case"], s["case"]["rot"]
    begin, kv, table = s["q_begin"].tolist(), s["kv_len"].tolist(), s["table"].long()
    out = {"q": torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)}
    for name in ("k", "v"):
        out[name] = s[name][0].float().double()
    k = torch.arange(r // 2, device=DEV)
    for b in range(c["n"]):
        lo, hi = begin[b], begin[b + 1]
        first = kv[b] - (hi - lo)
        pos = first + s["depth"][lo:hi].double() + (float(s["pos_begin"][b]) if c["far"] else 0.0)
        turn = torch.polar(torch.full((hi - lo, r // 2), s["amplitude"], dtype=torch.float64, device=DEV), pos[:, None] * s["freq_dev"])[:, None, :]
        ia, ib = (k, k + r // 2) if c["pairing"] == "half" else (2 * k, 2 * k + 1)
        new = {"v": s["v_new"][lo:hi].double()}
        for name, x in (("q", s["q"]), ("k", s["k_new"])):
            y = x[lo:hi].double()
            w = torch.complex(y[..., ia], y[..., ib]) * turn
            y[..., ia], y[..., ib] = w.real, w.imag
            new[name] = y
        out["q"][lo:hi] = new["q"]
        at = torch.arange(first, kv[b], device=DEV)
        page, slot = table[b][at // c["page"]], at % c["page"]
        for name in ("k", "v"):
            x = _exact_code(new[name]) if c["q8"] else new[name]
            if c["token_major"]:
                out[name][page, slot] = x
            else:
                out[name][page, :, slot] = x
    out["k"], out["v"] = out["k"][None], out["v"][None]
    return dict(out, scale_k=None, scale_v=None) if c["q8"] else out


def _exact_attend(s):
    c = s["case"]
    g = c["hq"] // c["h"]
    begin, kv, parent = s["q_begin"].tolist(), s["kv_len"].tolist(), s["parent"].tolist()
    out = s["out"].double()
    lse = torch.zeros(out.shape[:2], dtype=torch.float64, device=DEV)
    for b in range(c["n"]):
        m, length = begin[b + 1] - begin[b], kv[b]
        pages = s["table"][b, : -(-length // c["page"])].long()
        side = {}
        for name in ("k", "v"):
            if c["q8"]:
                x = s[name][0].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * _two(s["scale_" + name][0][pages].long() - 127).unsqueeze(-1)
            else:
                x = s[name][0][pages].double()
            x = x if c["token_major"] else x.permute(0, 2, 1, 3)
            side[name] = x.reshape(-1, c["h"], c["d"])[:length]
        hidden = torch.zeros(m, length, dtype=torch.bool)
        hidden[:, length - m:] = True
        for i in range(m):                                        # a row sees itself and its parents
            j = i
            while j >= 0:
                hidden[i, length - m + j] = False
                j = parent[begin[b] + j]
        hidden = hidden.to(DEV)
        for head in range(c["hq"]):
            z = s["q"][begin[b]: begin[b + 1], head].double() @ side["k"][:, head // g].T / math.sqrt(c["d"])
            z = z.masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(z, -1)
            out[begin[b]: begin[b + 1], head] = torch.exp(z - norm[:, None]) @ side["v"][:, head // g]
            lse[begin[b]: begin[b + 1], head] = norm
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
