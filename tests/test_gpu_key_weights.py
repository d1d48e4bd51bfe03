"""GPU parity of the attention weights of a cache's keys, through the C ABI, against fp64 sums.

Bound, derived. A score's exponent is c s - l' with s summed over d products in 32 bits (cut or rounded, so a unit of 2^-23 a
step: d 2^-23 sum |q k|; a product of fp32 values is rounded too, once more 2^-24 of it), c and l' rounded once each, the
difference once: off by e = scale d 2^-23 sum |q k| + 2^-24 (3 |s scale| + 3 |lse|) (in units of the natural logarithm). Its
exponential is off by e and by 2^-22 of itself. A sum of r terms in 32 bits, in chains of r / 16 and 16 more, adds
(r / 16 + 24) 2^-24 of it, the fused multiply-add with the old weight 2^-24 of the result; decay is taken in 32 bits, 2^-24 of it."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from q4_helpers import U24, make_cache

pytestmark = pytest.mark.gpu


def keys(cache, B, Hkv, n, d, seed, pad=5):
    """(arguments of the call, fp64 keys); keys behind the n are NaN."""
    if cache == "q4":
        q4, k, _ = make_cache(B, Hkv, n, d, seed, cap=n + pad)
        return dict(q4=q4), k
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.randn(B, Hkv, n + pad, d, generator=g, device="cuda")
    k[:, :, n:] = float("nan")
    k = k.bfloat16() if cache == "bf16" else k
    return dict(k_cache=k), k[:, :, :n].double().cpu().numpy()


def expected(q, k, lse, scale, w_old, decay):
    """fp64 weights of one key head, and the bound: q [rows, d], k [n, d], lse [rows], w_old [n] or zeros."""
    d, live = q.shape[1], lse > -np.inf
    q, lse = q[live], lse[live, None]
    s = q @ k.T * scale
    p = np.exp(s - lse)
    e = scale * d * 2.0 ** -23 * (np.abs(q) @ np.abs(k).T) + U24 * (3 * np.abs(s) + 3 * np.abs(lse))
    new = p.sum(0)
    w = decay * w_old + new
    # (the new weights may be of any size beside the old ones: those carry their own error)
    bound = (p * (np.expm1(e) + 2.0 ** -22)).sum(0) + (len(q) / 16 + 24) * U24 * new + U24 * (np.abs(w) + np.abs(decay * w_old))
    return w, bound + 1e-37


def run(cache, B, H, Hkv, nq, nkv, d, lens=None, old=None, decay=1.0, in_place=False, seed=0, qpad=0, empty=()):
    args, k = keys(cache, B, Hkv, nkv, d, seed + 1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, H, nq + qpad, d, generator=g, device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    q = q[:, :, :nq]
    qn = q.double().cpu().numpy()
    scale = scale_of(d)
    lse = np.empty((B, H, nq), np.float32)
    sizes = [nkv if lens is None else min(max(n, 0), nkv) for n in lens or [nkv] * B]
    for b in range(B):
        for h in range(H):
            s = qn[b, h] @ k[b, h // (H // Hkv), :sizes[b]].T * scale
            m = s.max(1, initial=-np.inf, keepdims=True)
            lse[b, h] = (m[:, 0] + np.log(np.exp(s - m).sum(1))) if sizes[b] else -np.inf
    for i in empty:
        lse.reshape(-1)[i % lse.size] = -np.inf
    w0 = torch.rand(B, Hkv, nkv + 3, generator=g, device="cuda") * 5
    w0[:, :, 0 if old is None else old:] = float("nan")  # never read
    w = w0 if in_place else torch.full_like(w0, 7.0)
    before = w.clone()
    old_n = w0.double().cpu().numpy().copy()
    sv.sparvar_key_weights(q, nkv, torch.from_numpy(lse).cuda(), w, w_old=None if old is None else w0, n_old=old, decay=decay,
                           kv_len=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"), **args)
    torch.cuda.synchronize()
    got, before = w.double().cpu().numpy(), before.double().cpu().numpy()
    for b in range(B):
        n = sizes[b]
        for g_ in range(Hkv):
            rep = H // Hkv
            had = np.zeros(nkv)
            if old:
                had[:old] = old_n[b, g_, :old]
            want, bound = expected(qn[b, g_ * rep:(g_ + 1) * rep].reshape(-1, d), k[b, g_, :n],
                                   lse[b, g_ * rep:(g_ + 1) * rep].reshape(-1).astype(np.float64), scale, had[:n], decay)
            err = np.abs(got[b, g_, :n] - want)
            assert (err <= bound).all(), f"entry {b} key head {g_}: {(err / bound).max():.2f} of the bound"
            assert np.array_equal(got[b, g_, n:], before[b, g_, n:], equal_nan=True)


CACHES = ["bf16", "f32", "q4"]


@pytest.mark.parametrize("B,H,Hkv,nq,nkv,d", [
    (1, 1, 1, 1, 1, 64), (2, 2, 2, 1, 33, 128), (1, 8, 2, 1, 3001, 128), (2, 4, 4, 3, 100, 64), (1, 8, 1, 4, 700, 64),
    (1, 8, 1, 5, 257, 128), (1, 2, 1, 48, 95, 64), (1, 2, 1, 49, 64, 128), (1, 1, 1, 128, 130, 128),
    # more rows than fit LDS at once: few keys (rows shared out), more and more of them
    (1, 1, 1, 129, 31, 128), (1, 2, 1, 300, 65, 64), (2, 6, 3, 150, 500, 128), (1, 8, 8, 190, 2100, 64),
    (2, 16, 16, 130, 2150, 128), (2, 20, 20, 135, 3300, 64), (2, 20, 20, 140, 3300, 128), (1, 8, 1, 401, 1000, 128)])
@pytest.mark.parametrize("cache", CACHES)
def test_weights(cache, B, H, Hkv, nq, nkv, d):
    note(f"[key weights] {cache} B={B} H={H}/{Hkv} nq={nq} nkv={nkv} d={d}")
    run(cache, B, H, Hkv, nq, nkv, d, seed=nq + nkv, qpad=(nq % 3))
    run(cache, B, H, Hkv, nq, nkv, d, seed=nq + nkv, old=nkv // 2, decay=0.75, qpad=2 * (nq % 2), empty=(0, 5, nq))


@pytest.mark.parametrize("B,H,nkv,d", [(2, 16, 1800, 128), (2, 16, 1800, 64), (1, 8, 3000, 128), (1, 8, 1800, 64)])
@pytest.mark.parametrize("cache", CACHES)
def test_keys_of_a_workgroup(cache, B, H, nkv, d):
    """As many keys as make the workgroups 256 keys each (bf16, 4 bits), 128 and 64; an odd tile of rows at the end."""
    note(f"[key weights] forms {cache} B={B} H={H} nkv={nkv} d={d}")
    run(cache, B, H, H, 161, nkv, d, seed=nkv + d, old=nkv - 100, decay=0.5, empty=(3, 160))


@pytest.mark.parametrize("nq,nkv,d", [(1, 3000, 128), (200, 300, 64), (300, 900, 128)])
@pytest.mark.parametrize("cache", CACHES)
def test_lengths(cache, nq, nkv, d):
    """Lengths of their own, keys past them NaN in the cache's tail; weights past a length stay as they were."""
    note(f"[key weights] lengths {cache} nq={nq} nkv={nkv} d={d}")
    lens = [0, -3, 1, 31, 32, 33, nkv - 1, nkv, nkv + 99]
    run(cache, len(lens), 2, 1, nq, nkv, d, lens=lens, old=nkv, decay=0.5, seed=3)
    run(cache, len(lens), 2, 1, nq, nkv, d, lens=lens, old=40, in_place=True, seed=4)


@pytest.mark.parametrize("cache", CACHES)
def test_in_place_twice(cache):
    """Two steps into the same weights: the second adds to what the first gave, and a decay of zero forgets it."""
    note(f"[key weights] in place {cache}")
    B, H, Hkv, nq, nkv, d = 1, 4, 2, 7, 200, 128
    args, k = keys(cache, B, Hkv, nkv, d, 9)
    q = torch.randn(B, H, nq, d, device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    lse = torch.full((B, H, nq), 5.0, device="cuda")
    w = [torch.full((B, Hkv, nkv), 3.0, device="cuda") for _ in range(3)]
    sv.sparvar_key_weights(q, nkv, lse, w[0], **args)
    sv.sparvar_key_weights(q, nkv, lse, w[1], **args)
    sv.sparvar_key_weights(q, nkv, lse, w[1], w_old=w[1], **args)
    sv.sparvar_key_weights(q, nkv, lse, w[2], w_old=w[2], decay=0.0, **args)
    torch.cuda.synchronize()
    assert torch.equal(w[1], w[0] + w[0]) and torch.equal(w[2], w[0])


@pytest.mark.parametrize("nq,nkv", [(1, 100), (200, 100)])
@pytest.mark.parametrize("cache", CACHES)
def test_nan(cache, nq, nkv):
    """A NaN key has a NaN weight, and no other; a query whose LSE is NaN makes those of its head group NaN, not others'."""
    note(f"[key weights] NaN {cache} nq={nq}")
    B, H, Hkv, d = 1, 4, 2, 64
    args, _ = keys(cache, B, Hkv, nkv, d, 2)
    if cache == "q4":
        args["q4"].k_scale[0, 0, 37, 1] = 255
    else:
        args["k_cache"][0, 0, 37, 3] = float("nan")
    q = torch.randn(B, H, nq, d, device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    lse, w = torch.full((B, H, nq), 5.0, device="cuda"), torch.empty(B, Hkv, nkv, device="cuda")
    sv.sparvar_key_weights(q, nkv, lse, w, **args)
    torch.cuda.synchronize()
    bad = torch.isnan(w)
    assert bad.sum() == 1 and bad[0, 0, 37]
    lse[0, 2, nq - 1] = float("nan")
    sv.sparvar_key_weights(q, nkv, lse, w, **args)
    torch.cuda.synchronize()
    assert torch.isnan(w[0, 1]).all() and torch.isnan(w[0, 0]).sum() == 1


def test_weights_of_a_whole_attention():
    """After attention over the same keys every query gives one in all, shared out among the keys of its group."""
    note("[key weights] after attention")
    B, H, Hkv, nq, nkv, d = 2, 8, 4, 65, 500, 128
    q4, _, _ = make_cache(B, Hkv, nkv, d, 8)
    q = torch.randn(B, H, nq, d, device="cuda").bfloat16()
    o, lse, w = torch.empty_like(q), torch.empty(B, H, nq, device="cuda"), torch.empty(B, Hkv, nkv, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse)
    sv.sparvar_key_weights(q, nkv, lse, w, q4=q4)
    torch.cuda.synchronize()
    # (the two calls' scores may differ by the bound of attention's LSE, 2e-4)
    assert (w.double().sum(2) - nq * (H // Hkv)).abs().max() <= 2.1e-4 * nq * (H // Hkv)


def test_streams():
    """Two calls side by side on streams of their own, of few rows and of many, give what each gives alone."""
    note("[key weights] two streams")
    jobs = []
    for nq in (1, 200):
        q4, _, _ = make_cache(2, 2, 3000, 128, 60 + nq)
        q = torch.randn(2, 8, nq, 128, device="cuda").bfloat16()
        lse = torch.randn(2, 8, nq, device="cuda") + 9
        jobs.append((q, lse, q4, torch.cuda.Stream(), torch.empty(2, 2, 3000, device="cuda"), torch.empty(2, 2, 3000, device="cuda")))
    for q, lse, q4, _, alone, _ in jobs:
        sv.sparvar_key_weights(q, 3000, lse, alone, q4=q4)
    torch.cuda.synchronize()
    for _ in range(10):
        for q, lse, q4, stream, _, w in jobs:
            sv.sparvar_key_weights(q, 3000, lse, w, q4=q4, stream=stream)
    torch.cuda.synchronize()
    for _, _, _, _, alone, w in jobs:
        assert torch.equal(alone, w)
