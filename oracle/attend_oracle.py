"""float64 oracle of the serving step: 8-bit rows, appended tokens, attention over a cache (numpy, one row at a time)."""
import numpy as np

E4M3_MAX = 448.0


def e4m3_values() -> np.ndarray:
    """Value of every code byte: sign, four exponent bits of bias 7, three mantissa bits; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = np.nan if (b & 127) == 127 else (-v if s else v)
    return out


_VAL = e4m3_values()


def quantize_rows(x: np.ndarray):
    """x [..., d] float64 -> (codes uint8 [..., d], exponents uint8 [...]): the rule of kvc_quantize."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    amax = np.max(np.where(fin, np.abs(x), 0.0), axis=-1, initial=0.0)
    e = np.full(amax.shape, -127, np.int64)
    while True:                                    # the smallest power of two under which the row fits
        up = amax > E4M3_MAX * np.ldexp(1.0, e)
        if not up.any():
            break
        e = np.where(up, e + 1, e)
    y = np.where(fin, x, 0.0) / np.ldexp(1.0, e)[..., None]
    y = np.where((e == 120)[..., None], np.clip(y, -240.0, 240.0), y)   # 256 * 2^120 would be no finite bf16
    mag = np.abs(y)
    step = np.ldexp(1.0, np.where(mag < 2.0 ** -6, -9, np.frexp(np.maximum(mag, 2.0 ** -6))[1] - 1 - 3))
    r = np.rint(mag / step) * step                 # to nearest, ties to even
    pos = _VAL[:127]                               # ascending
    code = np.searchsorted(pos, r).astype(np.uint8)
    assert np.array_equal(pos[code], r)
    code = np.where(np.signbit(y), code | 0x80, code).astype(np.uint8)
    code = np.where(fin, code, np.where(code < 128, 0x7F, 0xFF)).astype(np.uint8)
    return code, (e + 127).astype(np.uint8)


def dequantize_rows(code: np.ndarray, e: np.ndarray) -> np.ndarray:
    v = _VAL[code] * np.ldexp(1.0, e.astype(np.int64) - 127)[..., None]
    return np.where((e == 255)[..., None], np.nan, v)


def attend_row(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """q [d], k, v [n, d] (the keys the row sees) -> (out [d], lse, sum_t p_t |v_t| [d], largest sum_c |q_c k_c|)."""
    if k.shape[0] == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    s = scale * (k @ q)
    m = s.max()
    p = np.exp(s - m)
    l = p.sum()
    return (p @ v) / l, m + np.log(l), (p @ np.abs(v)) / l, float((np.abs(k) @ np.abs(q)).max())
