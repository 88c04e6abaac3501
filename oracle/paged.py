"""Paged serving in 64 bits: attention of rows at the end of a sequence's keys, and
8-bit rows with a power of two (the definitions the kernels are tested against)."""

import numpy as np

E_MIN, E_MAX = -80, 120


def attend(q, k, v, labels, sink, window):
    """q [n, Hq, d] are the last n of the m positions of k, v [m, Hkv, d]. Row i sees
    key j iff j <= p_i = m - n + i and, on a streaming head, j < sink or p_i - j <
    window. A row that sees nothing gives zeros."""
    n, hq, d = q.shape
    m, hkv, _ = k.shape
    out = np.zeros((n, hq, d))
    pos = np.arange(m - n, m)[:, None]
    j = np.arange(m)[None, :]
    for h in range(hq):
        kv = h // (hq // hkv)
        see = j <= pos
        if labels[kv]:
            see = see & ((j < sink) | (pos - j < window))
        used = see.any(0)
        s = q[:, h] @ k[used, kv].T / np.sqrt(d)
        s = np.where(see[:, used], s, -np.inf)
        rows = see.any(1)
        if not rows.any():
            continue
        s = s[rows]
        p = np.exp(s - s.max(1, keepdims=True))
        out[rows, h] = p @ v[used, kv] / p.sum(1, keepdims=True)
    return out


def e4m3_values():
    """The value of each 8-bit code: sign, 4 bits of exponent (bias 7), 3 of mantissa;
    0x7f and 0xff are NaN, there is no infinity."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c & 128, -x, x)


def encode(x):
    """Codes and powers of rows x [..., d]: for each row the least power e in [E_MIN,
    E_MAX] with max |x| <= 448 * 2^e over its finite numbers, and for each number the
    code nearest to x * 2^-e (ties to the even code; with the power E_MAX at most 240, as
    256 * 2^120 is no bf16 number; NaN for what is not finite)."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    most = np.where(finite, np.abs(x), 0).max(-1)
    powers = np.arange(E_MIN, E_MAX + 1)
    fits = most[..., None] <= 448.0 * 2.0 ** powers
    e = np.where(fits.any(-1), E_MIN + fits.argmax(-1), E_MAX)
    y = np.where(finite, x, 0) / 2.0 ** e[..., None].astype(np.float64)
    val = e4m3_values()[:127]  # codes 0 .. 126 in increasing order
    a = np.abs(y)
    hi = np.clip(np.searchsorted(val, a), 1, 126)
    lo = hi - 1
    up = (a - val[lo] > val[hi] - a) | ((a - val[lo] == val[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, lo)
    code = np.where(e[..., None] == E_MAX, np.minimum(code, np.searchsorted(val, 240.0)), code)
    code = np.where(np.signbit(y), code | 128, code)
    return np.where(finite, code, 127).astype(np.uint8), e.astype(np.int8)


def decode(codes, powers):
    return e4m3_values()[codes] * 2.0 ** powers[..., None].astype(np.float64)
