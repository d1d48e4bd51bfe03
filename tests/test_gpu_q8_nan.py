"""NaN in attention over an 8-bit cache: a NaN key or query makes its rows' outputs and their log of the softmax denominator
NaN, in every form of a call; -inf stands for rows without keys alone. Other rows are as without it."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from test_gpu_q8_attn import check_rows, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ws", [False, True])
@pytest.mark.parametrize("B,H,Hkv,nq,nkv,d", [
    (2, 2, 2, 5, 70, 128), (2, 4, 2, 1, 9000, 64),                              # few rows, with parts too
    (1, 4, 2, 701, 3000, 128), (1, 8, 8, 646, 2755, 64),                        # sets of waves
    (2, 8, 8, 900, 1000, 128), (2, 16, 16, 1600, 200, 64), (2, 16, 16, 1600, 1000, 128)])
def test_dense(B, H, Hkv, nq, nkv, d, ws):
    note(f"[q8 NaN] dense B={B} H={H}/{Hkv} nq={nq} nkv={nkv} d={d} ws={ws}")
    q8, k, v = make_cache(B, Hkv, nkv, d, 64, nq + d)
    at, dead = nkv - 3, nq // 2
    q8.k.view(torch.uint8)[0, 0, at, 7] = 0xff
    q = torch.randn(B, H, nq, d, device="cuda").bfloat16()
    q[:, H - 1, dead, 3] = float("nan")
    o, lse = torch.full_like(q, 5.0), torch.full((B, H, nq), 5.0, device="cuda")
    lens = [nkv] + [at - 1, 0][:B - 1]
    work = None
    if ws:
        size = sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, nq, nkv, d)
        work = torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                 workspace=work)
    torch.cuda.synchronize()
    rows = torch.arange(nq, device="cuda")
    for b in range(B):
        for h in range(H):
            kv = h // (H // Hkv)
            nan = torch.zeros(nq, dtype=torch.bool, device="cuda")
            if b == 0 and kv == 0:
                nan[:] = True
            if h == H - 1:
                nan |= rows == dead
            assert torch.equal(torch.isnan(lse[b, h]), nan), (b, h)
            assert torch.equal(torch.isnan(o[b, h].float()), nan[:, None].expand(nq, d)), (b, h)
    for b, h in ((0, H - 1), (B - 1, 0)):
        ok = torch.ones(nq, dtype=torch.bool)
        if h == H - 1:
            ok[dead] = False
        if (b == 0 and h // (H // Hkv) == 0) or not ok.any():
            continue
        kv, n = h // (H // Hkv), lens[b]
        pick = np.flatnonzero(ok.numpy())[::max(1, nq // 64)]
        check_rows(o[b, h].double().cpu().numpy()[pick], lse[b, h].double().cpu().numpy()[pick],
                   q[b, h].double().cpu().numpy()[pick], k[b, kv, :n], v[b, kv, :n], scale_of(d), what=f"entry {b} head {h}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H", [2, 8, 30])  # rows in four, two and one part
def test_sparse(d, H):
    """The NaN lies in a block that some rows list; rows without blocks stay -inf."""
    note(f"[q8 NaN] sparse H={H} d={d}")
    h, k = [1, 2, 4, 8, 16, 32], 6
    og, g = O.Geometry(h, h, 8, 1), sv.Geometry(h, h, 8, 1)
    q8, kk, vv = make_cache(2, H, og.C(k), d, 64, d + H)
    G_k, nb = og.tiles(k), og.nb_le(k)
    q8.k.view(torch.uint8)[:, :, og.C(k) - 1, 7] = 0x7f  # the last token, of the last block
    q = torch.randn(2, H, og.N(k), d, device="cuda").bfloat16()
    one = [[] if t == 0 else [0, 3, nb - 1] if t % 2 else [0, 3, nb - 2] for t in range(G_k)]
    rows = one * (2 * H)
    ptr = np.cumsum([0] + [len(x) for x in rows])
    rp, ci = torch.from_numpy(ptr.astype(np.int32)).cuda(), torch.tensor(sum(rows, []), dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 5.0), torch.full((2, H, og.N(k)), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o, rp, ci, lse=lse)
    torch.cuda.synchronize()
    mask = O.block_mask(og, k, one)
    nan, none = torch.from_numpy(mask[:, -1]).cuda(), torch.from_numpy(~mask.any(1)).cuda()
    for b in range(2):
        for hh in range(H):
            assert torch.equal(torch.isnan(lse[b, hh]), nan) and torch.equal(torch.isnan(o[b, hh].float()), nan[:, None].expand(-1, d))
            assert torch.equal(torch.isinf(lse[b, hh]), none) and (o[b, hh][none] == 0).all()
    ok = np.flatnonzero(~mask[:, -1])
    check_rows(o[1, 0].double().cpu().numpy()[ok], lse[1, 0].double().cpu().numpy()[ok], q[1, 0].double().cpu().numpy()[ok],
               kk[1, 0], vv[1, 0], scale_of(d), mask=mask[ok])
