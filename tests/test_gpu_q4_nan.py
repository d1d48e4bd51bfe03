"""NaN in attention over a 4-bit cache: a NaN key or query makes its rows' outputs and their log of the softmax denominator NaN, in
every form of a call; -inf stands for rows without keys alone. Other rows are as without it."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from q4_helpers import check_rows, make_cache
from test_q4_forms import DENSE, SPARSE
from test_q8_forms import sampled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,d,sizes", DENSE)
def test_dense(form, d, sizes):
    """The key lies in the first key head's plane of every entry; all entries but the first end before it, the last at once."""
    B, H, Hkv, nq, nkv, _ = sizes
    note(f"[q4 NaN] dense {form} d={d} {sizes}")
    q4, k, v = make_cache(B, Hkv, nkv, d, nq + d, cap=nkv + 5)
    at, dead = nkv - 3, nq // 2
    q4.k_scale[:, 0, at, 1] = 255
    q = torch.randn(B, H, nq, d, generator=torch.Generator(device="cuda").manual_seed(nkv), device="cuda").bfloat16()
    q[:, H - 1, dead, 3] = float("nan")
    o, lse = torch.full_like(q, 5.0), torch.full((B, H, nq), 5.0, device="cuda")
    lens = ([nkv] + [at] * (B - 2) + [0])[:B] if B > 1 else [nkv]
    work = torch.full((max(sv.sparvar_dense_attn_q4_workspace(B, H, Hkv, nq, nkv, d), 16),), 0xff, dtype=torch.uint8, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), workspace=work)
    torch.cuda.synchronize()
    rows = torch.arange(nq, device="cuda")
    for b in range(B):
        for h in range(H):
            kv, n = h // (H // Hkv), lens[b]
            nan = torch.zeros(nq, dtype=torch.bool, device="cuda")
            if n > at and kv == 0:
                nan[:] = True
            if h == H - 1 and n > 0:
                nan |= rows == dead
            assert torch.equal(torch.isnan(lse[b, h]), nan), (b, h)
            assert torch.equal(torch.isnan(o[b, h].float()), nan[:, None].expand(nq, d)), (b, h)
            if n == 0:
                assert torch.isinf(lse[b, h]).all() and (o[b, h] == 0).all()
                continue
            pick = sampled(nq, nq, 64)
            pick = pick[~nan.cpu().numpy()[pick]]
            if len(pick):
                check_rows(o[b, h].double().cpu().numpy()[pick], lse[b, h].double().cpu().numpy()[pick], q[b, h].double().cpu().numpy()[pick],
                           k[b, kv, :n], v[b, kv, :n], scale_of(d), what=f"entry {b} head {h}")


@pytest.mark.parametrize("form,d,sizes", SPARSE)
def test_sparse(form, d, sizes):
    """The key is the last token, of a block that every second row lists; the first row is empty, a query of it NaN and one
    of the second row too."""
    h, w, b, k, B, H, Hkv = sizes
    note(f"[q4 NaN] sparse {form} d={d} {sizes}")
    og, g = O.Geometry(h, w, b, 1), sv.Geometry(h, w, b, 1)
    q4, kk, vv = make_cache(B, Hkv, og.C(k), d, d + H)
    G_k, nb, N = og.tiles(k), og.nb_le(k), og.N(k)
    q4.k_scale[:, :, og.C(k) - 1, 0] = 255
    q = torch.randn(B, H, N, d, generator=torch.Generator(device="cuda").manual_seed(N), device="cuda").bfloat16()
    one = [[] if t == 0 else [0, nb - 1] if t % 2 else [0, 1, nb - 2] for t in range(G_k)]
    mask = O.block_mask(og, k, one)
    sees, none = mask[:, -1], ~mask.any(1)
    empty, live = np.flatnonzero(none)[0], np.flatnonzero(~none & ~sees)
    q[:, :, empty, 1] = float("nan")
    nan = sees.copy()
    if len(live):
        q[:, :, live[0], 2] = float("nan")
        nan[live[0]] = True
    ptr = np.cumsum([0] + [len(x) for x in one * (B * H)])
    rp, ci = torch.from_numpy(ptr.astype(np.int32)).cuda(), torch.tensor(sum(one, []) * (B * H), dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 5.0), torch.full((B, H, N), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q4_fwd(g, k, q, q4, o, rp, ci, lse=lse)
    torch.cuda.synchronize()
    nan_t, none_t = torch.from_numpy(nan).cuda(), torch.from_numpy(none).cuda()
    assert torch.equal(torch.isnan(lse), nan_t.expand(B, H, N)) and torch.equal(torch.isnan(o.float()), nan_t[:, None].expand(B, H, N, d))
    assert torch.equal(torch.isinf(lse), none_t.expand(B, H, N)) and (o[:, :, none_t] == 0).all()
    ok = np.flatnonzero(~nan & ~none)[:200]
    for bb, hh in {(0, 0), (B - 1, H - 1)}:
        if len(ok):
            check_rows(o[bb, hh].double().cpu().numpy()[ok], lse[bb, hh].double().cpu().numpy()[ok], q[bb, hh].double().cpu().numpy()[ok],
                       kk[bb, hh // (H // Hkv)], vv[bb, hh // (H // Hkv)], scale_of(d), mask=mask[ok], what=f"entry {bb} head {hh}")
