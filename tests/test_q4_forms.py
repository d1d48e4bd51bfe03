"""Every form that a call over a 4-bit cache can take is run by a case that is known to take it: the library says which one
(host only), so a case that a change of the rules moves to another form fails here."""
import numpy as np
import pytest
import torch

from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from test_q8_forms import sampled

# (waves, sets, more than one part), d: B, H, H_kv, n_q, n_kv, lengths (None: n_kv; 0 and 70 leave parts empty). No waves:
# few rows a workgroup, 16 (no sets) or 32 (one)
DENSE = [
    ((0, 0, False), 64, (2, 2, 1, 5, 65, [65, 0])), ((0, 0, False), 128, (1, 4, 2, 7, 33, None)),
    ((0, 0, True), 64, (3, 8, 1, 1, 1970, [1970, 0, 70])), ((0, 0, True), 128, (3, 2, 1, 9, 1479, [1479, 65, 0])),
    ((0, 1, False), 64, (3, 8, 2, 1359, 68, [68, 0, 33])), ((0, 1, False), 128, (3, 8, 4, 173, 193, [193, 1, 0])),
    ((0, 1, True), 64, (3, 3, 3, 147, 3528, [3528, 0, 70])), ((0, 1, True), 128, (3, 1, 1, 464, 1800, [1800, 65, 0])),
    ((2, 4, False), 64, (3, 3, 3, 1387, 1473, [1473, 0, 70])), ((2, 4, False), 128, (3, 2, 2, 1372, 1480, [1480, 70, 0])),
    ((4, 2, False), 64, (3, 6, 6, 1374, 1872, [1872, 70, 0])), ((4, 2, False), 128, (2, 4, 1, 3089, 968, [968, 449])),
    ((4, 1, False), 64, (3, 12, 3, 580, 30, [30, 0, 29])), ((4, 1, False), 128, (2, 24, 6, 440, 30, [30, 1])),
    ((4, 1, True), 64, (1, 16, 4, 258, 4731, None)), ((4, 1, True), 128, (3, 4, 4, 338, 5235, [5235, 0, 70])),
    ((8, 1, False), 64, (2, 6, 6, 3588, 1448, [1448, 0])), ((8, 1, False), 128, (3, 6, 3, 2071, 257, [257, 0, 63])),
    ((8, 1, True), 64, (3, 8, 2, 692, 3875, [3875, 70, 0])), ((8, 1, True), 128, (1, 16, 4, 516, 4471, [4400])),
]


def test_dense_cases_take_their_forms():
    seen = set()
    for (waves, sets, cut), d, (B, H, Hkv, nq, nkv, _) in DENSE:
        w, s, parts = sv.sparvar_dense_attn_q4_form(B, H, Hkv, nq, nkv, d, True)
        assert (w, s, parts > 1) == (waves, sets, cut), (d, B, H, Hkv, nq, nkv)
        size = sv.sparvar_dense_attn_q4_workspace(B, H, Hkv, nq, nkv, d)
        assert size == (4 * parts * B * H * nq * (d + 2) if cut else 0)
        assert sv.sparvar_dense_attn_q4_form(B, H, Hkv, nq, nkv, d, False)[2] == 1
        seen.add((w, s, parts > 1, d))
    # sets of waves take no parts
    assert seen == {(w, s, cut, d) for d in (64, 128) for w, s, cuts in
                    [(0, 0, (False, True)), (0, 1, (False, True)), (4, 1, (False, True)), (8, 1, (False, True)),
                     (4, 2, (False,)), (2, 4, (False,))] for cut in cuts}


# (waves, parts of a row), d: sides h, w, block edge, scale, B, H, H_kv. Tiles of 33 to 64 queries take parts by the number of
# workgroups; of up to 32, 65 to 128 and more they take none
S5 = [1, 2, 4, 8]
SPARSE = [
    ((1, 1), 64, (S5 + [13], S5 + [11], 4, 5, 1, 3, 3)), ((1, 1), 128, (S5 + [13], S5 + [16], 5, 5, 2, 2, 1)),
    ((2, 1), 64, ([1, 4, 30], [1, 4, 30], 8, 3, 2, 26, 26)), ((2, 1), 128, ([1, 4, 30], [1, 4, 27], 8, 3, 2, 18, 9)),
    ((2, 2), 64, ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20)), ((2, 2), 128, ([1, 4, 30], [1, 4, 30], 8, 3, 1, 20, 10)),
    ((2, 4), 64, (S5 + [16, 25], S5 + [16, 29], 8, 6, 1, 4, 2)), ((2, 4), 128, (S5 + [16, 29], S5 + [16, 25], 8, 6, 1, 3, 3)),
    ((4, 1), 64, (S5 + [23], S5 + [20], 9, 5, 2, 3, 1)), ((4, 1), 128, ([1, 20, 33], [1, 4, 8], 16, 3, 1, 2, 1)),
    ((8, 1), 64, ([1, 45], [1, 50], 20, 2, 1, 2, 2)), ((8, 1), 128, (S5 + [20], S5 + [20], 16, 5, 2, 2, 1)),
]


def test_sparse_cases_take_their_forms():
    seen = set()
    for form, d, (h, w, b, k, B, H, Hkv) in SPARSE:
        assert sv.sparvar_block_sparse_attn_q4_form(sv.Geometry(h, w, b, 1), k, B, H, Hkv, d) == form, (d, h, w, b)
        seen.add((*form, d))
    assert seen == {(*f, d) for d in (64, 128) for f in [(1, 1), (2, 1), (2, 2), (2, 4), (4, 1), (8, 1)]}


@pytest.mark.gpu
@pytest.mark.parametrize("form,d,sizes", DENSE)
def test_dense_form(form, d, sizes):
    """With a workspace of NaN, lengths of their own, a capacity past the cache of NaN codes."""
    from q4_helpers import check_rows, make_cache

    B, H, Hkv, nq, nkv, lens = sizes
    note(f"[q4 forms] dense {form} d={d} {sizes}")
    w, s, parts = sv.sparvar_dense_attn_q4_form(B, H, Hkv, nq, nkv, d, True)
    assert (w, s, parts > 1) == form
    q4, k, v = make_cache(B, Hkv, nkv, d, nq + nkv, cap=nkv + 70)
    g = torch.Generator(device="cuda").manual_seed(nq)
    q = torch.randn(B, H, nq + 3, d, generator=g, device="cuda").bfloat16()[:, :, :nq]
    o, lse = torch.full((B, H, nq, d), 5.0, device="cuda").bfloat16(), torch.full((B, H, nq), 5.0, device="cuda")
    size = sv.sparvar_dense_attn_q4_workspace(B, H, Hkv, nq, nkv, d)
    work = torch.full((max(size, 16) + 64,), 0xff, dtype=torch.uint8, device="cuda")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse, kv_len=kv_len, workspace=work[:max(size, 16)])
    torch.cuda.synchronize()
    assert (work[max(size, 16):] == 0xff).all()
    at = sampled(nq, nq)
    for b in range(B):
        n = nkv if lens is None else lens[b]
        for h in range(H):
            check_rows(o[b, h].double().cpu().numpy()[at], lse[b, h].double().cpu().numpy()[at],
                       q[b, h].double().cpu().numpy()[at], k[b, h // (H // Hkv), :n], v[b, h // (H // Hkv), :n], scale_of(d),
                       what=f"entry {b} head {h}")
    # every row, by the form without parts: both calls are within their bounds of the same values
    alone, alone_l = torch.empty_like(o), torch.empty_like(lse)
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, alone, lse=alone_l, kv_len=kv_len)
    torch.cuda.synchronize()
    assert torch.equal(torch.isinf(lse), torch.isinf(alone_l)) and torch.isfinite(o.float()).all()
    full = ~torch.isinf(lse)
    assert (lse[full] - alone_l[full]).abs().max() <= 4e-4
    vmax = np.abs(v).max()  # sum p |v| and |o| are at most this
    assert (o.float() - alone.float()).abs().max() <= 2 * 1.02 * 2.0 ** -8 * 2 * vmax


@pytest.mark.gpu
@pytest.mark.parametrize("order", [False, True])
@pytest.mark.parametrize("form,d,sizes", SPARSE)
def test_sparse_form(form, d, sizes, order):
    """Random rows, three of them empty, ids out of range among the others, codes past the cache NaN."""
    from test_gpu_q4_attn import run_sparse

    h, w, b, k, B, H, Hkv = sizes
    note(f"[q4 forms] sparse {form} d={d} {sizes} order={order}")
    assert sv.sparvar_block_sparse_attn_q4_form(sv.Geometry(h, w, b, 1), k, B, H, Hkv, d) == form
    run_sparse(h, w, b, k, B, H, Hkv, d, seed=d + b + sum(w), empty=(0, 3, 8), order=order)
