"""float64 oracle of a step of drafted tokens (numpy, one row at a time): trees, rotary positions, verification."""
import numpy as np


def tree_rows(parent):
    """parent: list of one request -> (list of sets: the new tokens a row sees, list of depths).  A parent that does not come
    before its row counts as -1."""
    seen, depth = [], []
    for j, a in enumerate(parent):
        ok = 0 <= a < j
        seen.append((seen[a] if ok else set()) | {j})
        depth.append(depth[a] + 1 if ok else 0)
    return seen, depth


def mask_words(seen, words):
    out = np.zeros((len(seen), words), np.uint32)
    for j, s in enumerate(seen):
        for a in s:
            out[j, a // 32] |= np.uint32(1 << (a % 32))
    return out


def rotate(x, pos, freq, rot, interleaved, amplitude=1.0):
    """x [..., d] at position pos -> (rotated, |x| + |y| of every channel's pair times the amplitude, 0 where nothing turns)."""
    x = np.asarray(x, np.float64)
    a = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    b = a + 1 if interleaved else a + rot // 2
    ang = float(pos) * np.asarray(freq, np.float64)
    c, s = np.cos(ang) * amplitude, np.sin(ang) * amplitude
    out, size = x.copy(), np.zeros_like(x)
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out, size


def _clean(p):
    with np.errstate(invalid="ignore"):
        return np.where(p > 0, p, 0.0)            # NaN and negative entries count as 0


def verify(parent, token, target, draft, u, u_next):
    """One request (lists and float64 [rows, n]) -> (kept places, next token)."""
    n = target.shape[1]
    if draft is not None:
        draft = _clean(draft)
    node, kept, P, spent, left, gone = 0, [0], _clean(target[0]), False, 1.0, []
    for c in range(1, len(parent)):
        if parent[c] != node or spent or not 0 <= token[c] < n:
            continue
        x = token[c]
        if draft is not None:
            yes = u[c] * draft[node][x] < P[x]
        else:
            yes = x not in gone and u[c] * left < target[node][x]
        if yes:
            node, P, left, gone = c, _clean(target[c]), 1.0, []
            kept.append(c)
            continue
        if draft is not None:
            with np.errstate(invalid="ignore"):
                rest = _clean(P - draft[node])
            z = rest.sum()
            if z > 0:
                P = rest / z
            else:
                spent, P = True, _clean(target[node])
        elif x not in gone:
            left -= max(float(np.nan_to_num(target[node][x])), 0.0)
            gone.append(x)
    if gone:
        P = P.copy()
        P[gone] = 0.0
        if not P.sum() > 0:
            P = _clean(target[node])
    cdf = np.cumsum(P)
    if not (cdf[-1] > 0 and np.isfinite(cdf[-1])):
        return kept, -1
    above = np.nonzero((cdf > u_next * cdf[-1]) & (P > 0))[0]
    return kept, int(above[0]) if len(above) else int(np.nonzero(P > 0)[0][-1])
