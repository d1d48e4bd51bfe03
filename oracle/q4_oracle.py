"""fp64 oracle of the 4-bit cache, of the weights of its keys and of eviction, from their definitions: e2m1 values on their
grid, a group's exponent by search, weights by plain sums, the kept tokens by sorting."""
from __future__ import annotations

import numpy as np

__all__ = ["E2M1", "GROUP", "Q4_E_MIN", "Q4_E_MAX", "e2m1_round", "group_exponent", "encode_rows", "decode_rows", "key_weights",
           "kept_tokens"]

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])  # the index is the code
GROUP = 32
Q4_E_MIN, Q4_E_MAX = -100, 112


def e2m1_round(y):
    """Code 0..7 of |y|: the nearest value's, ties to the even code, saturated."""
    a = np.minimum(np.abs(np.asarray(y, dtype=np.float64)), 6.0)
    hi = np.clip(np.searchsorted(E2M1, a), 1, 7)
    lo = hi - 1
    dlo, dhi = a - E2M1[lo], E2M1[hi] - a
    return np.where(dlo < dhi, lo, np.where(dhi < dlo, hi, np.where(lo % 2 == 0, lo, hi)))


def group_exponent(top):
    """Smallest e in [Q4_E_MIN, Q4_E_MAX] with top <= 7 * 2^e (Q4_E_MAX where none is)."""
    for e in range(Q4_E_MIN, Q4_E_MAX + 1):
        if top <= 7.0 * 2.0 ** e:
            return e
    return Q4_E_MAX


def encode_rows(x):
    """Rows [n, d]: (packed code bytes [n, d / 2], scale bytes [n, d / 32]); a group with a NaN has byte 255 (its codes
    are not defined: 0 here)."""
    x = np.asarray(x, dtype=np.float64)
    n, d = x.shape
    code, scale = np.zeros((n, d), np.uint8), np.zeros((n, d // GROUP), np.uint8)
    for i in range(n):
        for g in range(d // GROUP):
            part = x[i, g * GROUP:(g + 1) * GROUP]
            if np.isnan(part).any():
                scale[i, g] = 255
                continue
            e = group_exponent(np.abs(part).max())
            scale[i, g] = e + 127
            y = np.where(np.isinf(part), np.copysign(8.0, part), np.where(np.isinf(part), 0.0, part) * 2.0 ** -e)
            code[i, g * GROUP:(g + 1) * GROUP] = e2m1_round(y) + 8 * np.signbit(part)
    return code[:, 0::2] | code[:, 1::2] << 4, scale


def decode_rows(code, scale):
    """The values that packed codes [.., d / 2] and scale bytes [.., d / 32] stand for."""
    code = np.asarray(code)
    nib = np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], -1)
    v = np.where(nib >= 8, -1.0, 1.0) * E2M1[nib & 7]
    s = np.where(np.asarray(scale) == 255, np.nan, 2.0 ** (np.asarray(scale, dtype=np.float64) - 127.0))
    return v * np.repeat(s, GROUP, axis=-1)


def key_weights(q, k, lse, scale):
    """Attention weight that keys k [n, d] got from queries q [rows, d] with softmax denominators lse [rows]."""
    w = np.zeros(len(k))
    for qi, li in zip(q, lse):
        if li == -np.inf:
            continue
        w += np.exp(k @ qi * scale - li)
    return w


def kept_tokens(w, n_keep, n_first, n_last):
    """The tokens of a plane of len(w) that stay, ascending."""
    n = len(w)
    if n <= n_keep:
        return list(range(n))
    rest = list(range(n_first, n - n_last))
    rest.sort(key=lambda t: (0 if np.isnan(w[t]) else 1, 0.0 if np.isnan(w[t]) else -w[t], t))
    return sorted(list(range(n_first)) + rest[:n_keep - n_first - n_last] + list(range(n - n_last, n)))
