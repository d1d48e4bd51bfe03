"""Shared by the tests of the 4-bit cache: caches whose groups differ in scale, and one head's attention against fp64.

Bound of an output: K and V are exact, so what is rounded to 16 bits are the probabilities and the output, each by at most
u = 2^-8 of its value: |o - ref| <= u (sum_j p_j |v_j| + |ref|), times 1.02 for what 32-bit sums, the exponential and queries'
elements below 2^-13 of their row's largest (held to 2^-21 of it) add. The log of the softmax denominator is held to 2e-4, as
everywhere."""
import numpy as np
import torch

import oracle as O
from paper_2602_04361_amd import sparvar as sv

U16, U24 = 2.0 ** -8, 2.0 ** -24


def values_of(q4):
    """fp64 values of a Q4Cache's K and V, by the oracle."""
    return [O.decode_rows(c.view(torch.uint8).cpu().numpy(), s.view(torch.uint8).cpu().numpy())
            for c, s in ((q4.k, q4.k_scale), (q4.v, q4.v_scale))]


def make_cache(B, Hkv, n, d, seed, cap=None):
    """A cache of n written tokens (capacity cap: the rest are NaN) whose groups differ in scale, and its values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q4 = sv.Q4Cache.empty(B, Hkv, n if cap is None else cap, d)
    for t in (q4.k, q4.v):
        t.fill_(0x77)
    for t in (q4.k_scale, q4.v_scale):
        t.fill_(255)
    x = torch.randn(2, B, Hkv, n, d, generator=g, device="cuda")
    tok, grp = torch.arange(n, device="cuda")[:, None], torch.arange(d, device="cuda")[None] // 32
    x[0] *= 2.0 ** (-((tok + grp) % 3).float())
    x[1] *= 2.0 ** (((tok + 2 * grp) % 5).float() - 2)
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, q4)
    torch.cuda.synchronize()
    k, v = values_of(q4)
    return q4, k[:, :, :n], v[:, :, :n]


def check_rows(got, lse, q, k, v, scale, mask=None, what=""):
    """One head: got [n_q, d], lse [n_q] or None; mask [n_q, n_kv] or None."""
    s = q @ k.T * scale
    if mask is not None:
        s = np.where(mask, s, -np.inf)
    m = s.max(1, initial=-np.inf, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    p = np.exp(s - m)
    l = p.sum(1, keepdims=True)
    full = l[:, 0] > 0
    p = p / np.where(l > 0, l, 1.0)
    ref = p @ v
    bound = 1.02 * U16 * (p @ np.abs(v) + np.abs(ref)) + 1e-30
    assert np.isfinite(got).all(), what
    worst = (np.abs(got - ref) / bound).max() if len(k) else 0.0
    assert (np.abs(got - ref) <= bound).all(), f"{what}: {worst:.3f} of the bound"
    assert (got[~full] == 0).all(), what
    if lse is not None:
        want = np.where(full, m[:, 0] + np.log(np.where(full, l[:, 0], 1.0)), -np.inf)
        assert np.array_equal(np.isinf(lse), ~full), what
        assert (np.abs(lse[full] - want[full]) <= 2e-4).all(), what
