"""Refusals of the 4-bit cache's calls, of the key weights and of eviction, before anything reaches a GPU (host only)."""
import ctypes

import pytest
import torch

from paper_2602_04361_amd import sparvar as sv
from paper_2602_04361_amd.pipeline import BudgetPath, Q4SparsePath

FAKE, FAKE2 = 1 << 20, 1 << 21  # never dereferenced: validation fails first
SIDES = [1, 2, 4, 8]
INV, UNS, CAP = sv.ERR_INVALID, sv.ERR_UNSUPPORTED, sv.ERR_CAPACITY


def cache(d=64, **kw):
    cap = kw.get("capacity", 1000)
    a = dict(capacity=cap, k=FAKE, v=FAKE, bh_stride=cap * (d // 2), k_scale=FAKE, v_scale=FAKE, scale_bh_stride=cap * (d // 32))
    a.update(kw)
    return sv._CQ4Cache(*[a[n] for n, _ in sv._CQ4Cache._fields_])


BAD_CACHES = [dict(capacity=0), dict(capacity=1 << 26, bh_stride=1 << 40), dict(k=None), dict(v=None), dict(k_scale=None),
              dict(v_scale=None), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(bh_stride=999 * 32), dict(bh_stride=1000 * 32 + 8),
              dict(scale_bh_stride=1999), dict(scale_bh_stride=2001), dict(k_scale=FAKE + 1), dict(v_scale=FAKE + 1)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_cache_struct(bad):
    lib, c, good = sv.load_library(), ctypes.byref(cache(**bad)), ctypes.byref(cache(k=FAKE2, v=FAKE2, k_scale=FAKE2, v_scale=FAKE2))
    assert lib.sparvar_kv_quantize_q4(2, 2, 64, sv.BF16, 10, 5, FAKE, FAKE, 640, c, None) == INV
    assert lib.sparvar_kv_dequantize_q4(2, 2, 64, sv.F32, 10, 5, c, FAKE, FAKE, 640, None) == INV
    assert lib.sparvar_dense_attn_q4_fwd(2, 4, 2, 10, 100, 64, sv.BF16, FAKE, 640, c, None, FAKE, None, 0.1, None, 0, None) == INV
    g = sv.Geometry(SIDES, SIDES, 4, 1)
    assert lib.sparvar_block_sparse_attn_q4_fwd(g.ref, 4, 2, 4, 2, 64, sv.BF16, FAKE, 64 * 64, c, FAKE, None, 0.1, FAKE, FAKE, None,
                                                None) == INV
    assert lib.sparvar_key_weights(2, 4, 2, 10, 100, 64, sv.BF16, FAKE, 640, None, 0, c, FAKE, None, None, 0, 1.0, FAKE, 100, 0.1,
                                   None) == INV
    for src, dst in ((c, good), (good, c)):
        assert lib.sparvar_kv_evict(2, 2, 64, sv.BF16, 100, 50, 0, 0, None, FAKE, 100, None, None, 0, None, None, 0, src, dst, FAKE,
                                    FAKE2, 50, None) == INV
    assert lib.sparvar_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(d=96), UNS), (dict(dt=7), UNS), (dict(B=0), INV), (dict(H=0), INV), (dict(n=0), INV), (dict(t0=-1), INV),
    (dict(t0=991), CAP), (dict(t0=(1 << 31) - 5), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(k=FAKE + 2), INV),
    (dict(s=639), INV), (dict(s=641), INV), (dict(n=1 << 25, d=128), INV), (dict(c=None), INV)])
def test_rows_arguments(bad, status):
    a = dict(B=2, H=2, d=64, dt=sv.BF16, n=10, t0=5, k=FAKE, v=FAKE, s=640, c=ctypes.byref(cache()))
    a.update(bad)
    lib = sv.load_library()
    assert lib.sparvar_kv_quantize_q4(a["B"], a["H"], a["d"], a["dt"], a["n"], a["t0"], a["k"], a["v"], a["s"], a["c"], None) == status
    assert lib.sparvar_kv_dequantize_q4(a["B"], a["H"], a["d"], a["dt"], a["n"], a["t0"], a["c"], a["k"], a["v"], a["s"], None) == status


LONG = cache(capacity=30000)


@pytest.mark.parametrize("bad,status", [
    (dict(dt=sv.F32), UNS), (dict(d=80), UNS), (dict(H=5), INV), (dict(nq=0), INV), (dict(nkv=0), INV), (dict(nkv=30001), CAP),
    (dict(q=None), INV), (dict(qs=639), INV), (dict(o=FAKE + 2), INV), (dict(sc=0.0), INV), (dict(sc=float("inf")), INV),
    (dict(ws=FAKE, size=16, nkv=30000), CAP), (dict(ws=FAKE + 4, size=1 << 30, nkv=30000), INV)])
def test_dense_arguments(bad, status):
    a = dict(B=2, H=4, Hkv=2, nq=10, nkv=100, d=64, dt=sv.BF16, q=FAKE, qs=640, o=FAKE, sc=0.1, ws=None, size=0)
    a.update(bad)
    assert sv.load_library().sparvar_dense_attn_q4_fwd(
        a["B"], a["H"], a["Hkv"], a["nq"], a["nkv"], a["d"], a["dt"], a["q"], a["qs"], ctypes.byref(LONG), None, a["o"], None, a["sc"],
        a["ws"], a["size"], None) == status


def test_workspace_and_forms():
    assert sv.sparvar_dense_attn_q4_workspace(1, 4, 2, 1, 30000, 64) >= 2 * 4 * (64 + 2) * 4  # two parts of four rows
    assert sv.sparvar_dense_attn_q4_workspace(2, 16, 16, 4096, 10521, 128) == 0
    assert sv.sparvar_dense_attn_q4_workspace(2, 16, 16, 1, 40, 128) == 0
    lib = sv.load_library()
    assert lib.sparvar_dense_attn_q4_workspace(1, 3, 2, 1, 1000, 64) == INV
    assert lib.sparvar_dense_attn_q4_workspace(1, 4, 2, 1, 1000, 65) == UNS
    assert lib.sparvar_dense_attn_q4_form(1, 4, 2, 1, 1000, 64, 0, None) == INV
    for fn in (sv.sparvar_dense_attn_q4_workspace,):
        with pytest.raises(sv.SparvarError):
            fn(1, 3, 2, 1, 1000, 64)


@pytest.mark.parametrize("bad,status", [
    (dict(k=5), INV), (dict(dt=sv.F32), UNS), (dict(H=3), INV), (dict(rp=None), INV), (dict(ci=None), INV), (dict(cap=84), CAP),
    (dict(sc=-1.0), INV)])
def test_sparse_arguments(bad, status):
    a = dict(k=4, H=4, dt=sv.BF16, rp=FAKE, ci=FAKE, cap=85, sc=0.1)
    a.update(bad)
    g = sv.Geometry(SIDES, SIDES, 4, 1)
    assert sv.load_library().sparvar_block_sparse_attn_q4_fwd(
        g.ref, a["k"], 2, a["H"], 2, 64, a["dt"], FAKE, 64 * 64, ctypes.byref(cache(capacity=a["cap"])), FAKE, None, a["sc"], a["rp"],
        a["ci"], None, None) == status


@pytest.mark.parametrize("bad,status", [
    (dict(d=32), UNS), (dict(dt=5), UNS), (dict(H=3), INV), (dict(B=0), INV), (dict(nq=0), INV), (dict(nkv=0), INV),
    (dict(nkv=0x7fffff00, ks=1 << 40, ws=1 << 32), INV), (dict(B=1 << 15, Hkv=1 << 15, H=1 << 15, nq=2), INV), (dict(sc=0.0), INV),
    (dict(B=1, H=1, Hkv=1, nq=0x7fffff00, qs=1 << 38), INV),
    (dict(sc=float("nan")), INV), (dict(decay=-0.1), INV), (dict(decay=float("inf")), INV), (dict(q=None), INV), (dict(q=FAKE + 8), INV),
    (dict(qs=63), INV), (dict(k=None), INV), (dict(c=True), INV), (dict(k=FAKE + 4), INV), (dict(ks=6399), INV), (dict(lse=None), INV),
    (dict(w=None), INV), (dict(old=-1), INV), (dict(old=101), INV), (dict(old=5, w0=None), INV), (dict(ws=99), INV),
    (dict(k=None, c=True, dt=sv.F32), UNS), (dict(k=None, c=True, nkv=1001, ws=2000), CAP)])
def test_weights_arguments(bad, status):
    a = dict(B=2, H=4, Hkv=2, nq=10, nkv=100, d=64, dt=sv.BF16, q=FAKE, qs=640, k=FAKE, ks=6400, c=False, lse=FAKE, w0=FAKE, old=100,
             decay=1.0, w=FAKE, ws=100, sc=0.1)
    a.update(bad)
    assert sv.load_library().sparvar_key_weights(
        a["B"], a["H"], a["Hkv"], a["nq"], a["nkv"], a["d"], a["dt"], a["q"], a["qs"], a["k"], a["ks"],
        ctypes.byref(cache()) if a["c"] else None, a["lse"], None, a["w0"], a["old"], a["decay"], a["w"], a["ws"], a["sc"], None) == status
    assert sv.load_library().sparvar_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(d=32), UNS), (dict(dt=5), UNS), (dict(B=0), INV), (dict(H=0), INV), (dict(n=0), INV), (dict(keep=0), INV), (dict(first=-1), INV),
    (dict(last=-1), INV), (dict(first=30, last=21), INV), (dict(first=0x7fffffff, last=0x7fffffff), INV),
    (dict(n=0x7ffe0000, ss=1 << 40, ws=1 << 32), INV), (dict(keep=0x7ffe0000, ds=1 << 40, wos=1 << 32), INV),
    (dict(B=1 << 15, H=1 << 15, keep=200, ds=12800, wos=200), INV), (dict(w=None), INV), (dict(kept=None), INV), (dict(wo=None), INV),
    (dict(wo=FAKE), INV), (dict(ws=99), INV), (dict(wos=49), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(kd=None), INV),
    (dict(vd=None), INV), (dict(kd=FAKE), INV), (dict(vd=FAKE), INV), (dict(ss=6399), INV), (dict(ds=3199), INV), (dict(k=FAKE + 2), INV),
    (dict(src=True, dst=True), INV), (dict(src=True), INV), (dict(four=True, dst=False), INV), (dict(four=True, src=False), INV),
    (dict(four=True, alias=True), INV), (dict(four=True, n=1001, ws=1001), CAP), (dict(four=True, keep=1001, wos=1001), CAP)])
def test_evict_arguments(bad, status):
    a = dict(B=2, H=2, d=64, dt=sv.BF16, n=100, keep=50, first=5, last=5, w=FAKE, ws=100, k=FAKE, v=FAKE, ss=6400, kd=FAKE2, vd=FAKE2,
             ds=3200, src=False, dst=False, kept=FAKE, wo=FAKE2, wos=50, four=False, alias=False)
    if bad.get("four"):
        a.update(k=None, v=None, kd=None, vd=None, src=True, dst=True)
    a.update(bad)
    other = FAKE if a["alias"] else FAKE2
    src, dst = cache(), cache(k=other, v=other, k_scale=other, v_scale=other)
    assert sv.load_library().sparvar_kv_evict(
        a["B"], a["H"], a["d"], a["dt"], a["n"], a["keep"], a["first"], a["last"], None, a["w"], a["ws"], a["k"], a["v"], a["ss"], a["kd"],
        a["vd"], a["ds"], ctypes.byref(src) if a["src"] else None, ctypes.byref(dst) if a["dst"] else None, a["kept"], a["wo"], a["wos"],
        None) == status
    assert sv.load_library().sparvar_last_error()


# ---- the binding's own checks (tensors on the CPU: each fails before the library is called)
def planes(B=1, H=2, n=64, d=64, dtype=torch.bfloat16):
    return torch.zeros(B, H, n, d, dtype=dtype)


def q4(B=1, H=2, n=64, d=64):
    return sv.Q4Cache.empty(B, H, n, d, device="cpu")


def refused(what, fn, *args, **kw):
    with pytest.raises(sv.SparvarError, match=what):
        fn(*args, **kw)


def test_q4_cache_class():
    code, scale = torch.zeros(1, 2, 64, 32, dtype=torch.uint8), torch.zeros(1, 2, 64, 2, dtype=torch.uint8)
    c = sv.Q4Cache(code, code.clone(), scale, scale.clone())
    assert (c.B, c.H_kv, c.capacity, c.d) == (1, 2, 64, 64)
    sv.Q4Cache(code.view(torch.float4_e2m1fn_x2), code, scale.view(torch.float8_e8m0fnu), scale)
    refused("is torch", sv.Q4Cache, code.bfloat16(), code, scale, scale)
    refused("is torch", sv.Q4Cache, code, code, scale.int(), scale)
    refused("share", sv.Q4Cache, code, code[:, :, :32], scale, scale)
    refused("v_scale must be", sv.Q4Cache, code, code, scale, scale[:, :, :63])
    refused("k_scale must be", sv.Q4Cache, code, code, scale[..., :1], scale)
    narrow = code[..., :16].contiguous()
    refused("head dim", sv.Q4Cache, narrow, narrow, scale, scale)
    refused("contiguous", sv.Q4Cache, code.transpose(2, 3).contiguous().transpose(2, 3), code, scale, scale)
    refused("head dim", sv.Q4Cache.empty, 1, 1, 8, 96, device="cpu")
    for bad in (dict(B=0), dict(H_kv=-1), dict(capacity=0)):
        refused("is empty", sv.Q4Cache.empty, **{**dict(B=1, H_kv=2, capacity=64, d=64, device="cpu"), **bad})


def weights(n=64):
    return torch.zeros(1, 2, n)


def test_tensors_off_the_gpu():
    k, c, w = planes(), q4(), weights()
    kept = torch.zeros(1, 2, 32, dtype=torch.int32)
    refused("not on a GPU", sv.sparvar_kv_quantize_q4, k, k, 0, c)
    refused("not on a GPU", sv.sparvar_kv_dequantize_q4, c, 0, k, k)
    refused("not on a GPU", sv.sparvar_dense_attn_q4_fwd, k, c, 64, torch.empty_like(k))
    refused("not on a GPU", sv.sparvar_key_weights, k, 64, w, w, q4=c)
    refused("not on a GPU", sv.sparvar_kv_evict, w, 64, 32, 0, 0, kept, weights(32), q4_src=c, q4_dst=q4(n=32))
    i = torch.zeros(9, dtype=torch.int32)
    refused("not on a GPU", sv.sparvar_block_sparse_attn_q4_fwd, sv.Geometry([8], [8], 4, 0), 1, k, c, torch.empty_like(k), i, i)


@pytest.mark.parametrize("extra", [1 << 32, -(1 << 32), 1 << 31, 3 << 40])
def test_numbers_past_32_bits(extra):
    k, c, w = planes(), q4(), weights()
    g, i, kept = sv.Geometry([8], [8], 4, 0), torch.zeros(9, dtype=torch.int32), torch.zeros(1, 2, 32, dtype=torch.int32)
    refused("32 bits", sv.sparvar_kv_quantize_q4, k, k, extra, c)
    refused("32 bits", sv.sparvar_kv_dequantize_q4, c, extra, k, k)
    refused("32 bits", sv.sparvar_dense_attn_q4_fwd, k, c, 64 + extra, torch.empty_like(k))
    refused("32 bits", sv.sparvar_block_sparse_attn_q4_fwd, g, 1 + extra, k, c, torch.empty_like(k), i, i)
    refused("32 bits", sv.sparvar_dense_attn_q4_workspace, 1, 2, 2, 1, 64 + extra, 64)
    refused("32 bits", sv.sparvar_dense_attn_q4_form, 1, 2, 2, 64 + extra, 64, 64, True)
    refused("32 bits", sv.sparvar_block_sparse_attn_q4_form, g, 1, 1 + extra, 2, 2, 64)
    refused("32 bits", sv.sparvar_key_weights, k, 64 + extra, w, w, q4=c)
    refused("32 bits", sv.sparvar_key_weights, k, 64, w, w, w_old=w, n_old=5 + extra, q4=c)
    for bad in ((64 + extra, 32, 0, 0), (64, 32 + extra, 0, 0), (64, 32, extra, 0), (64, 32, 0, extra)):
        refused("32 bits", sv.sparvar_kv_evict, w, *bad, kept, weights(32), q4_src=c, q4_dst=q4(n=32))


def test_mismatched_tensors():
    k = planes()
    refused("share", sv.sparvar_kv_quantize_q4, k, planes(n=32), 0, q4())
    refused("share", sv.sparvar_kv_quantize_q4, k, k.float(), 0, q4())
    refused("contiguous", sv.sparvar_dense_attn_q4_fwd, k, q4(), 64, planes(n=32))
    refused("float32", sv.sparvar_dense_attn_q4_fwd, k, q4(), 64, k, lse=torch.zeros(1, 2, 64, dtype=torch.float64))
    refused("64 tokens", sv.sparvar_block_sparse_attn_q4_fwd, sv.Geometry([8], [8], 4, 0), 1, planes(n=63), q4(), k, k, k)
    refused("row_ptr", sv.sparvar_block_sparse_attn_q4_fwd, sv.Geometry([8], [8], 4, 0), 1, k, q4(), torch.empty_like(k),
            torch.zeros(8, dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    refused("lse", sv.sparvar_key_weights, k, 64, weights(63), weights(), q4=q4())
    refused("lse", sv.sparvar_key_weights, k, 64, weights().double(), weights(), q4=q4())


def test_paths():
    args = (sv.Geometry(SIDES, SIDES, 4, 1), 3, [4], 1, 2, 64, 2, 1)
    p = Q4SparsePath(*args, device="cpu", prev_dilation=1, softmax_scale=0.5, projection="cover")
    assert (p.dil, p.scale, p.projection, set(p.out)) == (1, 0.5, sv.PROJECT_COVER, {1, 2, 3, 4})
    for option in (dict(use_schedule=True), dict(fused_decision=False), dict(dtype=torch.float32)):
        with pytest.raises(TypeError):
            Q4SparsePath(*args, device="cpu", **option)
    for bad in (dict(budget=0), dict(n_max=0), dict(n_first=-1), dict(n_last=-1), dict(n_first=6, n_last=5)):
        with pytest.raises(ValueError):
            BudgetPath(**{**dict(B=1, H=2, H_kv=2, d=64, n_max=4, budget=10, device="cpu"), **bad})
    b = BudgetPath(1, 2, 2, 64, 4, 10, device="cpu")
    x = torch.zeros(1, 5, 2, 64).bfloat16()
    with pytest.raises(ValueError):
        b.append(x, x, x)
    heads = sv.NormRope(cos_sin=torch.zeros(6, 32, 2))
    assert heads.rows(2, 4).cos_sin.data_ptr() == heads.cos_sin[2:].data_ptr()
    refused("rows", heads.rows, 3, 4)
