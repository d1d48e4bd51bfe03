"""Queries of attention over an 8-bit cache whose elements lie far apart: one channel many times the others, as outlier
channels are. The kernels of many rows hold a query as the sum of two 8-bit values; the log of the softmax denominator of
such rows keeps the bar of all others, 2e-4, against the fp64 oracle.

Bound of a row, derived: with u the power of two that brings the row's largest into (224, 448], elements of 2^-6 u and more
are exact and the others off by at most 2^-14 u (the smaller part's last place is 2^-13 u), so a score is off by at most
scale (2^-14 u sum |k_j| over those + d 2^-23 sum |q_j k_j|), the second term for products summed in 32 bits, cut or
rounded. The LSE is off by no more than its worst score, and by 8 2^-24 max |s| + (n + 16) 2^-24 for the exponents, the sum
over n keys and the logarithm in 32 bits. An LSE is held to both, that and 2e-4."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24


def outlier_rows(B, H, n, d, top, rest, seed):
    """Rows of normals times rest whose channel 5 is top, and 8-bit keys of normals times 4 without that channel."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, H, n, d, generator=g, device="cuda") * rest
    q[..., 5] = top
    return q.bfloat16(), g


def keys(B, H, n, d, G, g):
    x = torch.randn(2, B, H, n, d, generator=g, device="cuda")
    x[0] *= 4.0
    x[0, ..., 5] = 0.0
    q8 = sv.Q8Cache.empty(B, H, n, d, G)
    sv.sparvar_kv_quantize(x[0], x[1], 0, q8)
    out = [torch.empty(B, H, n, d, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize(q8, 0, out[0], out[1])
    return q8, out[0].double().cpu().numpy(), out[1].double().cpu().numpy()


def check(q, k, v, o, lse, scale, mask=None):
    """One head in fp64: the LSE and the output within the bound above."""
    n, d = k.shape
    s = q @ k.T * scale
    u = 2.0 ** np.ceil(np.log2(np.abs(q).max(1, keepdims=True) / 448.0))
    lost = np.where(np.abs(q) < 2.0 ** -6 * u, 2.0 ** -14 * u, 0.0)
    off = scale * (lost @ np.abs(k).T + d * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T))
    if mask is not None:
        s, off = np.where(mask, s, -np.inf), np.where(mask, off, 0.0)
    m = s.max(1)
    p = np.exp(s - m[:, None])
    l = p.sum(1)
    bound = off.max(1) + 8 * U32 * np.abs(np.where(np.isfinite(s), s, 0.0)).max(1) + (n + 16) * U32
    err = np.abs(lse - (m + np.log(l)))
    assert (err <= np.minimum(bound, 2e-4)).all(), f"LSE off by {err.max():.2e}, {(err / bound).max():.1f} of the bound"
    p /= l[:, None]
    ref, size = p @ v, p @ np.abs(v)
    assert (np.abs(o - ref) <= 1.02 * U16 * (size + np.abs(ref)) + 2 * bound[:, None] * size + 1e-30).all()


@pytest.mark.parametrize("top,rest", [(100.0, 0.1), (100.0, 0.2), (150.0, 0.15)])
@pytest.mark.parametrize("H,nq,nkv,d", [(1, 3, 64, 128), (16, 1600, 64, 128), (32, 1600, 64, 64)])
def test_dense_outlier_channel(H, nq, nkv, d, top, rest):
    """Few rows (bf16 products) and many (the two parts)."""
    note(f"[q8 dense] outlier {top} beside {rest}, H={H} nq={nq} nkv={nkv} d={d}")
    q, g = outlier_rows(1, H, nq, d, top, rest, nq + d)
    q8, k, v = keys(1, H, nkv, d, 64, g)
    o, lse = torch.empty_like(q), torch.empty(1, H, nq, device="cuda")
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse)
    torch.cuda.synchronize()
    for h in range(H):
        check(q[0, h].double().cpu().numpy(), k[0, h], v[0, h], o[0, h].double().cpu().numpy(),
              lse[0, h].double().cpu().numpy(), scale_of(d))


@pytest.mark.parametrize("top,rest", [(100.0, 0.1), (100.0, 0.2)])
@pytest.mark.parametrize("d", [64, 128])
def test_sparse_outlier_channel(d, top, rest):
    note(f"[q8 sparse] outlier {top} beside {rest}, d={d}")
    h, k, H = [1, 2, 4, 8, 16], 5, 2
    og, g = O.Geometry(h, h, 8, 1), sv.Geometry(h, h, 8, 1)
    q, gen = outlier_rows(1, H, og.N(k), d, top, rest, d)
    q8, kk, vv = keys(1, H, og.C(k), d, 64, gen)
    G_k = og.tiles(k)
    rows = [[0, 2, i % og.nb_le(k), og.nb_le(k) - 1] for i in range(3, 3 + H * G_k)]
    rows = [sorted(set(x)) for x in rows]
    ptr = np.cumsum([0] + [len(x) for x in rows])
    rp, ci = torch.from_numpy(ptr.astype(np.int32)).cuda(), torch.tensor(sum(rows, []), dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(1, H, og.N(k), device="cuda")
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o, rp, ci, lse=lse)
    torch.cuda.synchronize()
    for hh in range(H):
        check(q[0, hh].double().cpu().numpy(), kk[0, hh], vv[0, hh], o[0, hh].double().cpu().numpy(),
              lse[0, hh].double().cpu().numpy(), scale_of(d), mask=O.block_mask(og, k, rows[hh * G_k:(hh + 1) * G_k]))
