"""Queries that had no keys (LSE -inf) add nothing to a key's weight, whatever they hold and whatever the key is: rows that were
never written (padding) may hold NaN and infinities. The weights are those of the same call without such rows' values, to the
bit, and within the fp64 bound."""
import numpy as np
import pytest
import torch

from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from test_gpu_key_weights import CACHES, expected, keys

pytestmark = pytest.mark.gpu

ODD = [float("nan"), float("inf"), float("-inf"), 3e38, -3e38]


@pytest.mark.parametrize("B,H,Hkv,nq,nkv,d", [
    (1, 1, 1, 1, 100, 64), (1, 8, 2, 1, 300, 128), (2, 4, 2, 17, 100, 128), (1, 2, 1, 48, 95, 64),  # few rows
    # many: workgroups of 32, 64, 128 and 256 keys, a last tile of one row and of 9
    (1, 8, 1, 401, 1000, 128), (1, 1, 1, 129, 70, 64), (1, 8, 8, 161, 1800, 64), (1, 8, 8, 161, 3000, 128),
    (2, 16, 16, 161, 1800, 64), (2, 16, 16, 161, 1800, 128)])
@pytest.mark.parametrize("cache", CACHES)
def test_unseen_queries(cache, B, H, Hkv, nq, nkv, d):
    note(f"[key weights] unseen {cache} B={B} H={H}/{Hkv} nq={nq} nkv={nkv} d={d}")
    args, k = keys(cache, B, Hkv, nkv, d, 7)
    g = torch.Generator(device="cuda").manual_seed(nq + nkv)
    q = torch.randn(B, H, nq, d, generator=g, device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    lse = torch.rand(B, H, nq, generator=g, device="cuda") + 5
    unseen = torch.rand(B, H, nq, generator=g, device="cuda") < 0.3
    unseen[:, :, -1] = True
    if nq > 64:
        unseen[:, :, 32:64] = True  # a whole tile
    lse[unseen] = float("-inf")
    w0 = torch.rand(B, Hkv, nkv, generator=g, device="cuda")
    clean, odd = torch.empty_like(w0), torch.empty_like(w0)
    sv.sparvar_key_weights(q, nkv, lse, clean, w_old=w0, decay=0.5, **args)
    bad = torch.tensor(ODD, device="cuda")[torch.randint(0, len(ODD), (B, H, nq, d), generator=g, device="cuda")].to(q.dtype)
    sv.sparvar_key_weights(torch.where(unseen[..., None], bad, q), nkv, lse, odd, w_old=w0, decay=0.5, **args)
    torch.cuda.synchronize()
    qn, ln, wn, old = (t.double().cpu().numpy() for t in (q, lse, clean, w0))
    rep = H // Hkv
    for b in range(B):
        for h in range(Hkv):
            want, bound = expected(qn[b, h * rep:(h + 1) * rep].reshape(-1, d), k[b, h], ln[b, h * rep:(h + 1) * rep].reshape(-1),
                                   scale_of(d), old[b, h], 0.5)
            assert (np.abs(wn[b, h] - want) <= bound).all()
    assert torch.equal(odd, clean)


@pytest.mark.parametrize("nq", [1, 40, 200])
@pytest.mark.parametrize("cache", CACHES)
def test_no_query_at_all(cache, nq):
    """Without any query that had keys even a NaN key keeps what it had."""
    note(f"[key weights] no query {cache} nq={nq}")
    B, H, Hkv, nkv, d = 1, 2, 2, 130, 64
    args, _ = keys(cache, B, Hkv, nkv, d, 3)
    if cache == "q4":
        args["q4"].k_scale[0, 0, 37, 1] = 255
    else:
        args["k_cache"][0, 0, 37, 3] = float("nan")
    q = torch.full((B, H, nq, d), float("nan"), device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    w = torch.rand(B, Hkv, nkv, device="cuda")
    before = w.clone()
    sv.sparvar_key_weights(q, nkv, torch.full((B, H, nq), float("-inf"), device="cuda"), w, w_old=w, decay=0.5, **args)
    torch.cuda.synchronize()
    assert torch.equal(w, before * 0.5)


@pytest.mark.parametrize("nq", [1, 200])
def test_an_lse_of_plus_infinity(nq):
    """By the formula: nothing for a finite score, NaN for a NaN one."""
    note(f"[key weights] LSE of +inf nq={nq}")
    q, k = torch.zeros(1, 1, nq, 64, device="cuda"), torch.zeros(1, 1, 50, 64, device="cuda")
    k[0, 0, 7] = float("nan")
    w = torch.empty(1, 1, 50, device="cuda")
    sv.sparvar_key_weights(q, 50, torch.full((1, 1, nq), float("inf"), device="cuda"), w, k_cache=k)
    torch.cuda.synchronize()
    assert torch.isnan(w[0, 0, 7]) and (w[0, 0, torch.arange(50, device="cuda") != 7] == 0).all()
