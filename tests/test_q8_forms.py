"""Every form that a call over an 8-bit cache can take is run by a case that is known to take it: the library says which one
(host only), so a case that a change of the rules moves to another form fails here."""
import numpy as np
import pytest
import torch

from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv


def sampled(n, seed, most=192):
    """All of n rows, or the first, the last and a sample of them."""
    if n <= most:
        return np.arange(n)
    r = np.random.default_rng(seed)
    return np.unique(np.concatenate([[0, 1, n - 2, n - 1], r.choice(n, most - 4, replace=False)]))


# (waves, sets, more than one part), d: B, H, H_kv, n_q, n_kv, scale block, lengths (None: n_kv; 0 and 70 leave parts empty)
DENSE = [
    ((0, 1, False), 64, (2, 2, 1, 5, 65, 16, [65, 0])), ((0, 1, False), 128, (1, 4, 2, 7, 33, 64, None)),
    ((0, 1, True), 64, (3, 1, 1, 32, 647, 32, [647, 0, 70])), ((0, 1, True), 128, (3, 1, 1, 33, 513, 64, [513, 65, 0])),
    ((2, 4, False), 64, (1, 4, 2, 2122, 965, 64, None)), ((2, 4, False), 128, (3, 2, 2, 1381, 649, 32, [649, 70, 0])),
    ((4, 2, False), 64, (1, 8, 2, 3130, 2174, 128, [2101])), ((4, 2, False), 128, (3, 3, 3, 1821, 970, 64, [970, 70, 0])),
    ((4, 1, False), 64, (1, 4, 4, 4123, 34, 16, [33])), ((4, 1, False), 128, (3, 4, 2, 1370, 520, 64, [520, 0, 449])),
    ((4, 1, True), 64, (3, 8, 4, 161, 2983, 64, [2983, 0, 70])), ((4, 1, True), 128, (3, 8, 4, 165, 2126, 32, [2126, 65, 1])),
    ((4, 1, True), 64, (1, 2, 1, 1428, 4889, 128, None)), ((4, 1, True), 128, (1, 8, 2, 513, 2422, 16, [2400])),
    ((8, 1, False), 64, (3, 4, 4, 3433, 1284, 64, [1284, 0, 63])), ((8, 1, False), 128, (3, 6, 3, 1856, 513, 64, [513, 0, 300])),
    ((8, 1, True), 64, (3, 6, 3, 917, 3877, 64, [3877, 70, 0])), ((8, 1, True), 128, (3, 6, 3, 450, 4267, 32, [4267, 64, 0])),
]


def test_dense_cases_take_their_forms():
    seen = set()
    for (waves, sets, cut), d, (B, H, Hkv, nq, nkv, _, _) in DENSE:
        w, s, parts = sv.sparvar_dense_attn_q8_form(B, H, Hkv, nq, nkv, d, True)
        assert (w, s, parts > 1) == (waves, sets, cut), (d, B, H, Hkv, nq, nkv)
        size = sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, nq, nkv, d)
        assert size == (4 * parts * B * H * nq * (d + 2) if cut else 0)
        assert sv.sparvar_dense_attn_q8_form(B, H, Hkv, nq, nkv, d, False)[2] == 1
        seen.add((w, s, parts > 1, d))
    # sets of waves take no parts
    assert seen == {(w, s, cut, d) for d in (64, 128) for w, s, cuts in
                    [(0, 1, (False, True)), (4, 1, (False, True)), (8, 1, (False, True)), (4, 2, (False,)), (2, 4, (False,))]
                    for cut in cuts}


# (waves, parts of a row), d: sides h, w, block edge, scale, B, H, H_kv, scale block. Tiles of 33 to 64 queries take parts by
# the number of workgroups; of up to 32, 65 to 128 and more they take none
S5 = [1, 2, 4, 8]
SPARSE = [
    ((1, 1), 64, (S5 + [13], S5 + [11], 4, 5, 1, 3, 3, 16)), ((1, 1), 128, (S5 + [13], S5 + [16], 5, 5, 2, 2, 1, 64)),
    ((2, 1), 64, ([1, 4, 30], [1, 4, 30], 8, 3, 2, 26, 26, 64)), ((2, 1), 128, ([1, 4, 30], [1, 4, 27], 8, 3, 2, 18, 9, 32)),
    ((2, 2), 64, ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20, 64)), ((2, 2), 128, ([1, 4, 30], [1, 4, 30], 8, 3, 1, 20, 10, 128)),
    ((2, 4), 64, (S5 + [16, 25], S5 + [16, 29], 8, 6, 1, 4, 2, 64)), ((2, 4), 128, (S5 + [16, 29], S5 + [16, 25], 8, 6, 1, 3, 3, 16)),
    # 65 to 128 queries: edges of 9 to 11, and blocks of 16 on a scale 5 to 8 wide
    ((4, 1), 64, (S5 + [23], S5 + [20], 9, 5, 2, 3, 1, 32)), ((4, 1), 128, (S5 + [24], S5 + [25], 11, 5, 1, 4, 4, 64)),
    ((4, 1), 64, ([1, 8, 37], [1, 5, 5], 16, 3, 2, 2, 2, 16)), ((4, 1), 128, ([1, 20, 33], [1, 4, 8], 16, 3, 1, 2, 1, 128)),
    ((8, 1), 64, (S5 + [20], S5 + [35], 16, 5, 1, 2, 2, 64)), ((8, 1), 128, (S5 + [20], S5 + [20], 16, 5, 2, 2, 1, 32)),
    ((8, 1), 64, ([1, 45], [1, 50], 20, 2, 1, 2, 2, 64)), ((8, 1), 128, ([1, 45], [1, 41], 20, 2, 1, 2, 1, 16)),  # two slabs a tile
]


def test_sparse_cases_take_their_forms():
    seen = set()
    for form, d, (h, w, b, k, B, H, Hkv, _) in SPARSE:
        assert sv.sparvar_block_sparse_attn_q8_form(sv.Geometry(h, w, b, 1), k, B, H, Hkv, d) == form, (d, h, w, b)
        seen.add((*form, d))
    assert seen == {(*f, d) for d in (64, 128) for f in [(1, 1), (2, 1), (2, 2), (2, 4), (4, 1), (8, 1)]}


def test_form_arguments():
    g = sv.Geometry([1, 8], [1, 8], 8, 1)
    for bad in ((3, 1, 2, 2, 64), (2, 1, 3, 2, 64), (2, 1, 2, 2, 96)):
        with pytest.raises(sv.SparvarError):
            sv.sparvar_block_sparse_attn_q8_form(g, *bad)
    assert sv.load_library().sparvar_block_sparse_attn_q8_form(g.ref, 2, 1, 2, 2, 64, None) == sv.ERR_INVALID
    with pytest.raises(sv.SparvarError):
        sv.sparvar_dense_attn_q8_form(1, 3, 2, 1, 1000, 64, True)
    assert sv.load_library().sparvar_dense_attn_q8_form(1, 4, 2, 1, 1000, 64, 1, None) == sv.ERR_INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("form,d,sizes", DENSE)
def test_dense_form(form, d, sizes):
    """With a workspace of NaN, lengths of their own, a capacity past the cache of NaN codes."""
    from test_gpu_q8_attn import check_rows, make_cache

    B, H, Hkv, nq, nkv, G, lens = sizes
    note(f"[q8 forms] dense {form} d={d} {sizes}")
    w, s, parts = sv.sparvar_dense_attn_q8_form(B, H, Hkv, nq, nkv, d, True)
    assert (w, s, parts > 1) == form
    q8, k, v = make_cache(B, Hkv, nkv, d, G, nq + nkv, cap=nkv + 70)
    g = torch.Generator(device="cuda").manual_seed(nq)
    q = torch.randn(B, H, nq + 3, d, generator=g, device="cuda").bfloat16()[:, :, :nq]
    o, lse = torch.full((B, H, nq, d), 5.0, device="cuda").bfloat16(), torch.full((B, H, nq), 5.0, device="cuda")
    size = sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, nq, nkv, d)
    work = torch.full((max(size, 16) + 64,), 0xff, dtype=torch.uint8, device="cuda")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse, kv_len=kv_len, workspace=work[:max(size, 16)])
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
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, alone, lse=alone_l, kv_len=kv_len)
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
    from test_gpu_q8_attn import run_sparse

    h, w, b, k, B, H, Hkv, G = sizes
    note(f"[q8 forms] sparse {form} d={d} {sizes} order={order}")
    assert sv.sparvar_block_sparse_attn_q8_form(sv.Geometry(h, w, b, 1), k, B, H, Hkv, d) == form
    run_sparse(h, w, b, k, B, H, Hkv, d, G, seed=d + b + sum(w), empty=(0, 3, 8), order=order)


def test_sets_are_for_launches_of_up_to_a_workgroup_a_cu():
    """In larger ones the other forms are faster; the estimate alone took sets for 1152 workgroups (36 slabs of 64 rows of 32
    planes: 329 us, 281 by slabs of 128 in parts)."""
    taken = set()
    for B, H in ((1, 4), (1, 8), (1, 16), (2, 6), (2, 8), (2, 12), (2, 16)):
        for d in (64, 128):
            for nq, nkv in ((400, 921), (1024, 2521), (1093, 4545), (1382, 4020), (1600, 4121), (2304, 6425), (2563, 9290),
                            (3024, 8955), (3493, 8877), (4096, 10521)):
                for ws in (False, True):
                    waves, sets, _ = sv.sparvar_dense_attn_q8_form(B, H, H, nq, nkv, d, ws)
                    if sets > 1:
                        assert B * H * -(-nq // (32 * waves)) <= 256, (B, H, d, nq, nkv, ws)
                        taken.add((waves, sets))
    assert taken == {(4, 2), (2, 4)}
