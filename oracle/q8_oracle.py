"""fp64 oracle of the 8-bit cache and of the step that fills it, from their definitions: e4m3 values on their grid, the
block exponent by search, norms and rotations with plain loops over pairs. A plane of a cache is (values, exponents): the
values that the codes stand for divided by 2^e, [tokens, d], and one exponent a block."""
from __future__ import annotations

import numpy as np

__all__ = ["E4M3_MAX", "E_MIN", "E_MAX", "e4m3_grid", "e4m3_round", "block_exponent", "append_codes", "cache_values",
           "norm_rope", "codes_of_bytes"]

E4M3_MAX, E_MIN, E_MAX = 448.0, -100, 112


def codes_of_bytes(b):
    """Value of every e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    b = np.asarray(b, dtype=np.int64)
    s, e, m = b >> 7, (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(s == 1, -v, v)


def e4m3_grid():
    """The finite non-negative values, ascending; the index is the code."""
    return codes_of_bytes(np.arange(127))


def e4m3_round(y):
    """Nearest e4m3 value of y, ties to the even code, saturated; NaN stays."""
    y = np.asarray(y, dtype=np.float64)
    g = e4m3_grid()
    a = np.minimum(np.abs(np.where(np.isnan(y), 0.0, y)), E4M3_MAX)
    hi = np.clip(np.searchsorted(g, a), 1, len(g) - 1)
    lo = hi - 1
    dlo, dhi = a - g[lo], g[hi] - a
    pick = np.where(dlo < dhi, lo, np.where(dhi < dlo, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(y), np.nan, np.copysign(g[pick], y))


def block_exponent(top):
    """Smallest e in [E_MIN, E_MAX] with top <= 448 * 2^e (E_MAX where none is)."""
    for e in range(E_MIN, E_MAX + 1):
        if top <= E4M3_MAX * 2.0 ** e:
            return e
    return E_MAX


def append_codes(values, exps, rows, t0, G):
    """Writes rows [n, d] to tokens [t0, t0 + n) of a plane in place: every block they touch is encoded over its tokens
    before t0 + n, those before t0 with the values they hold."""
    n = len(rows)
    for j in range(t0 // G, -(-(t0 + n) // G)):
        a, b = j * G, min(j * G + G, t0 + n)
        old = values[a:min(max(t0, a), b)] * 2.0 ** float(exps[j]) if a < t0 else values[a:a]
        x = np.concatenate([old, np.asarray(rows, dtype=np.float64)[max(a - t0, 0):b - t0]])
        mag = np.abs(x)
        top = np.max(np.where(np.isnan(mag), 0.0, mag)) if x.size else 0.0
        e = block_exponent(top)
        values[a:b] = e4m3_round(x * 2.0 ** -e)
        exps[j] = e


def cache_values(values, exps, G):
    """The values a plane stands for."""
    return values * 2.0 ** np.asarray(exps, dtype=np.float64)[np.arange(len(values)) // G][:, None]


def norm_rope(x, norm, eps, w, cs, layout):
    """x [n, d] of one head: norm (None, "rms", "l2"), weight w [d] or None, rotation by cs [n, d/2, 2] or None."""
    y = np.array(x, dtype=np.float64)
    n, d = y.shape
    for i in range(n):
        if norm == "rms":
            y[i] /= np.sqrt(np.mean(y[i] ** 2) + eps)
        elif norm == "l2":
            y[i] /= max(np.sqrt(np.sum(y[i] ** 2)), eps)
    if w is not None:
        y = y * np.asarray(w, dtype=np.float64)
    if cs is not None:
        cs = np.asarray(cs, dtype=np.float64)
        z = y.copy()
        for p in range(d // 2):
            a, b = (2 * p, 2 * p + 1) if layout == "pairs" else (p, p + d // 2)
            z[:, a] = y[:, a] * cs[:, p, 0] - y[:, b] * cs[:, p, 1]
            z[:, b] = y[:, a] * cs[:, p, 1] + y[:, b] * cs[:, p, 0]
        y = z
    return y
