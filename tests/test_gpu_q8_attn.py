"""GPU parity of attention over an 8-bit cache, dense and block-sparse, through the C ABI, against the fp64 oracle on the
values that the codes stand for.

Tolerance: K and V are exact and Q is given, so what is rounded to 16 bits are the probabilities and the output, each by
at most u = 2^-8 of its value: |o - ref| <= u (sum_j p_j |v_j| + |ref|), times 1.02 for what 32-bit sums, the exponential
and queries' elements below 2^-9 of their row's largest (held to 2^-17 of it) add: a score is off by less than 2^-14 for
the rows of unit normals here. The log of the softmax denominator is held to 2e-4, as everywhere."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import INF_SIDES, note, scale_of
from paper_2602_04361_amd import sparvar as sv
from paper_2602_04361_amd.pipeline import Q8SparsePath

pytestmark = pytest.mark.gpu

U16 = 2.0 ** -8


def make_cache(B, Hkv, n, d, G, seed, cap=None, scales=True):
    """A cache of n written tokens (capacity cap: the rest are NaN codes) whose blocks differ in scale, and its values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    cap = n if cap is None else cap
    q8 = sv.Q8Cache.empty(B, Hkv, cap, d, G)
    for t in (q8.k, q8.v):
        t.view(torch.uint8).fill_(0x7f)
    for t in (q8.k_scale, q8.v_scale):
        t.fill_(255)
    x = torch.randn(2, B, Hkv, n, d, generator=g, device="cuda")
    if scales:  # neighbouring blocks apart by powers of two
        blocks = torch.arange(n, device="cuda") // G
        x[0] *= 2.0 ** (-(blocks % 3).float())[:, None]
        x[1] *= 2.0 ** ((blocks % 5).float() - 2)[:, None]
    sv.sparvar_kv_quantize(x[0], x[1], 0, q8)
    out = [torch.empty(B, Hkv, n, d, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize(q8, 0, out[0], out[1])
    return q8, out[0].double().cpu().numpy(), out[1].double().cpu().numpy()


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


def run_dense(B, H, Hkv, nq, nkv, d, G, lens=None, ws=False, seed=0, cap=None, pad=0, lse=True):
    q8, k, v = make_cache(B, Hkv, nkv, d, G, seed + 1, cap)
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, H, nq + pad, d, generator=g, device="cuda").bfloat16()[:, :, :nq]
    o = torch.full((B, H, nq, d), 5.0, device="cuda").bfloat16()
    out_l = torch.full((B, H, nq), 5.0, device="cuda") if lse else None
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    work = None
    if ws:
        size = sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, nq, nkv, d)
        work = torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")  # NaN in every float of it
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=out_l, kv_len=kv_len, workspace=work)
    torch.cuda.synchronize()
    qn, on = q.double().cpu().numpy(), o.double().cpu().numpy()
    ln = None if out_l is None else out_l.double().cpu().numpy()
    for b in range(B):
        n = nkv if lens is None else min(max(lens[b], 0), nkv)
        for h in range(H):
            kv = h // (H // Hkv)
            check_rows(on[b, h], None if ln is None else ln[b, h], qn[b, h], k[b, kv, :n], v[b, kv, :n], scale_of(d),
                       what=f"entry {b} head {h}")
    return o, out_l


@pytest.mark.parametrize("B,H,Hkv,nq,nkv,d,G", [
    (1, 1, 1, 1, 1, 128, 64), (2, 3, 3, 4, 5, 64, 32), (1, 2, 2, 16, 21, 128, 16), (2, 2, 2, 64, 121, 128, 64),
    (1, 2, 2, 33, 63, 64, 16), (1, 2, 2, 65, 64, 128, 128), (1, 1, 1, 129, 65, 64, 64), (1, 2, 1, 257, 300, 128, 32),
    (1, 4, 2, 36, 57, 64, 64), (2, 8, 2, 1, 777, 128, 64), (1, 8, 1, 7, 1500, 64, 128), (1, 16, 1, 5, 333, 128, 16),
    # long enough for parts: few rows, odd lengths and more parts than chunks divide into
    (1, 8, 2, 1, 9001, 128, 64), (1, 2, 2, 1, 20011, 64, 16), (1, 8, 1, 6, 7777, 64, 32), (1, 2, 2, 70, 8000, 128, 64),
    # more rows than a join takes a workgroup each; two sets of waves that share the keys
    (1, 4, 4, 700, 3000, 64, 32), (1, 4, 2, 701, 3000, 128, 64), (1, 20, 20, 1000, 1100, 128, 64), (1, 32, 32, 1000, 2600, 64, 16),
    # four sets of two waves
    (2, 8, 8, 646, 2755, 64, 64), (1, 12, 12, 1030, 2500, 128, 32),
    # slabs of 128 and 256 rows
    (2, 8, 8, 900, 1000, 128, 32), (2, 8, 8, 900, 1000, 64, 64), (2, 16, 16, 1600, 1000, 128, 64), (2, 16, 16, 1600, 200, 64, 16)])
@pytest.mark.parametrize("ws", [False, True])
def test_dense(B, H, Hkv, nq, nkv, d, G, ws):
    note(f"[q8 dense] B={B} H={H}/{Hkv} nq={nq} nkv={nkv} d={d} G={G} ws={ws}")
    run_dense(B, H, Hkv, nq, nkv, d, G, ws=ws, seed=nq + nkv, cap=nkv + 70, pad=3)


@pytest.mark.parametrize("ws", [False, True])
@pytest.mark.parametrize("nq,nkv,d", [(1, 4000, 128), (20, 900, 64), (100, 500, 128), (1000, 300, 128),
                                      (1000, 1500, 128), (700, 5000, 64), (540, 1500, 64)])
def test_dense_lengths(nq, nkv, d, ws):
    """Lengths of their own: none, negative, one, a chunk's edge, past the end; codes past a length are NaN."""
    lens = [0, -3, 1, 63, 64, 65, 200, nkv - 1, nkv, nkv + 99]
    note(f"[q8 dense] lengths nq={nq} nkv={nkv} d={d} ws={ws}")
    B = len(lens)
    q8, k, v = make_cache(B, 1, nkv, d, 32, 7)
    for b, n in enumerate(lens):
        n = min(max(n, 0), nkv)
        for t in (q8.k, q8.v):
            t.view(torch.uint8)[b, 0, n:] = 0x7f
        for t in (q8.k_scale, q8.v_scale):  # whole blocks past the length
            t[b, 0, -(-n // 32):] = 255
    q = torch.randn(B, 2, nq, d, device="cuda").bfloat16()
    o, lse = torch.full_like(q, 5.0), torch.full((B, 2, nq), 5.0, device="cuda")
    size = sv.sparvar_dense_attn_q8_workspace(B, 2, 1, nq, nkv, d)
    work = torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda") if ws else None
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                 workspace=work)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        n = min(max(n, 0), nkv)
        for h in range(2):
            check_rows(o[b, h].double().cpu().numpy(), lse[b, h].double().cpu().numpy(), q[b, h].double().cpu().numpy(),
                       k[b, 0, :n], v[b, 0, :n], scale_of(d), what=f"length {lens[b]}")


@pytest.mark.parametrize("ws", [False, True])
@pytest.mark.parametrize("nq,nkv,d", [(1, 20000, 128), (3, 9000, 64), (300, 500, 128), (2000, 300, 64)])
def test_dense_nan(nq, nkv, d, ws):
    """A NaN among the keys makes its plane's rows NaN, one among the values its channel, in every form and in parts; other
    planes and lengths that end before it are as they were."""
    note(f"[q8 dense] NaN nq={nq} nkv={nkv} d={d} ws={ws}")
    q8, k, v = make_cache(3, 2, nkv, d, 64, 5)
    at = nkv - 70
    q8.k.view(torch.uint8)[0, 0, at, 9] = 0x7f
    q8.v.view(torch.uint8)[0, 1, at, 9] = 0xff
    q8.k.view(torch.uint8)[1, 0, at, 9] = 0x7f
    q = torch.randn(3, 2, nq, d, device="cuda").bfloat16()
    o = torch.full_like(q, 5.0)
    size = sv.sparvar_dense_attn_q8_workspace(3, 2, 2, nq, nkv, d)
    work = torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda") if ws else None
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, kv_len=torch.tensor([nkv, at, nkv], dtype=torch.int32, device="cuda"),
                                 workspace=work)
    torch.cuda.synchronize()
    assert torch.isnan(o[0, 0]).all()
    assert torch.isnan(o[0, 1, :, 9]).all()
    others = [c for c in range(d) if c != 9]
    qn, on = q.double().cpu().numpy(), o.double().cpu().numpy()
    check_rows(on[0, 1][:, others], None, qn[0, 1], k[0, 1], v[0, 1][:, others], scale_of(d), what="channels without")
    for b, h, n in ((1, 0, at), (1, 1, at), (2, 0, nkv), (2, 1, nkv)):
        check_rows(on[b, h], None, qn[b, h], k[b, h, :n], v[b, h, :n], scale_of(d), what=f"entry {b} head {h}")


def test_dense_full_size():
    """The last scale of a 1024x1024 image, heads sampled."""
    note("[q8 dense] 4096 x 10521")
    B, H, d, nq, nkv = 1, 8, 128, 4096, 10521
    q8, k, v = make_cache(B, H, nkv, d, 64, 11)
    q = torch.randn(B, H, nq, d, device="cuda").bfloat16()
    o, lse = torch.empty_like(q), torch.empty(B, H, nq, device="cuda")
    sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse)
    torch.cuda.synchronize()
    r = np.random.default_rng(5)
    for h in (0, 7):
        rows = np.sort(r.choice(nq, 200, replace=False))
        check_rows(o[0, h].double().cpu().numpy()[rows], lse[0, h].double().cpu().numpy()[rows],
                   q[0, h].double().cpu().numpy()[rows], k[0, h], v[0, h], scale_of(d), what=f"head {h}")


def test_queries_of_any_size():
    """Queries times 2^60 under a scale divided by it give the same; rows whose elements spread over 2^24 keep the bound with
    a score's own error added: scale 2^-17 max|q| sum|k|, twice it on a probability.
    (A row is scaled by a power of two to a largest in (224, 448] and split in two e4m3 values, whose last place is 2^-9: what
    is lost is at most half of that, 2^-10, so 2^-10 / 224 = 2^-17.8 of the largest.)"""
    note("[q8 dense] sizes of queries")
    B, H, nq, nkv, d = 1, 1, 300, 400, 128
    for rows in (20, nq):  # few rows, slabs
        q8, k, v = make_cache(B, H, nkv, d, 64, 77)
        g = torch.Generator(device="cuda").manual_seed(rows)
        q = torch.randn(B, H, rows, d, generator=g, device="cuda").bfloat16()
        o = [torch.empty_like(q) for _ in range(2)]
        sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o[0], softmax_scale=0.0625)
        sv.sparvar_dense_attn_q8_fwd(q * 2.0 ** 60, q8, nkv, o[1], softmax_scale=0.0625 * 2.0 ** -60)
        torch.cuda.synchronize()
        assert torch.equal(o[0], o[1])
        spread = torch.randint(-24, 1, q.shape, generator=g, device="cuda").float().exp2()
        q = (q * spread * 4).bfloat16()
        sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o[0], softmax_scale=0.0625)
        torch.cuda.synchronize()
        qn, kn, vn, on = q[0, 0].double().cpu().numpy(), k[0, 0], v[0, 0], o[0][0, 0].double().cpu().numpy()
        s = qn @ kn.T * 0.0625
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        ref, size = p @ vn, p @ np.abs(vn)
        off = 2 * 0.0625 * 2.0 ** -17 * np.abs(qn).max(1) * np.abs(kn).sum(1).max()
        assert (np.abs(on - ref) <= 1.02 * U16 * (size + np.abs(ref)) + 2 * off[:, None] * size + 1e-30).all()


def test_scores_that_spread():
    """Scores far apart (one key takes all, the maximum grows along the walk) and equal ones."""
    note("[q8 dense] spread scores")
    B, H, d, nkv = 1, 1, 64, 500
    q8 = sv.Q8Cache.empty(B, H, nkv, d, 16)
    x = torch.zeros(2, B, H, nkv, d, device="cuda")
    x[0, ..., 0] = torch.arange(nkv, device="cuda") * 0.5   # ascending scores
    x[1] = torch.randn(B, H, nkv, d, device="cuda")
    sv.sparvar_kv_quantize(x[0], x[1], 0, q8)
    kv = [torch.empty(B, H, nkv, d, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize(q8, 0, kv[0], kv[1])
    q = torch.zeros(B, H, 4, d, device="cuda").bfloat16()
    q[0, 0, :, 0] = torch.tensor([100.0, -100.0, 0.0, 0.25])
    for ws in (False, True):
        o, lse = torch.empty_like(q), torch.empty(B, H, 4, device="cuda")
        size = sv.sparvar_dense_attn_q8_workspace(B, H, H, 4, nkv, d)
        sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, lse=lse, softmax_scale=1.0,
                                     workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if ws else None)
        torch.cuda.synchronize()
        # scores reach 25000: 32-bit products and sums of one term, so the exponent's argument is off by 2^-24 of them
        k, v, qn = kv[0][0, 0].double().cpu().numpy(), kv[1][0, 0].double().cpu().numpy(), q[0, 0].double().cpu().numpy()
        got = o[0, 0].double().cpu().numpy()
        check_rows(got[2:], lse[0, 0].double().cpu().numpy()[2:], qn[2:], k, v, 1.0, what="small scores")
        for i in (0, 1):
            s = qn[i] @ k.T
            top = np.flatnonzero(s >= s.max())
            ref = v[top].mean(0)
            assert (np.abs(got[i] - ref) <= 1.02 * U16 * (np.abs(v[top]).mean(0) + np.abs(ref)) + 1e-30).all()


# ------------------------------------------------------------------------------------------------ block-sparse
def run_sparse(h, w, b, k, B, H, Hkv, d, G, seed, empty=(), order=False):
    og, g = O.Geometry(h, w, b, 1), sv.Geometry(h, w, b, 1)
    n = og.C(k)
    q8, kk, vv = make_cache(B, Hkv, n, d, G, seed, cap=n + 9)
    r = np.random.default_rng(seed)
    G_k, nb = og.tiles(k), og.nb_le(k)
    rows = [sorted(r.choice(nb, size=int(r.integers(1, nb + 1)), replace=False).tolist()) for _ in range(B * H * G_k)]
    for i in empty:
        rows[i % len(rows)] = []
    M = max(map(len, rows)) + 2
    ids = np.full((len(rows), M), -1, dtype=np.int32)
    for i, x in enumerate(rows):
        ids[i, :len(x)] = x
        if x and i % 3 == 0:  # ids out of range are skipped wherever they stand
            ids[i, :len(x) + 1] = x[:1] + [nb + 5] + x[1:]
    ci = torch.from_numpy(ids.reshape(-1)).cuda()
    rp = (torch.arange(len(rows) + 1, device="cuda") * M).to(torch.int32)
    sched = torch.from_numpy(r.permutation(len(rows)).astype(np.int32)).cuda() if order else None
    N = og.N(k)
    q = torch.from_numpy(r.standard_normal((B, H, N + 2, d)).astype(np.float32)).cuda().bfloat16()[:, :, :N]
    # codes of blocks that a head's rows never list are NaN for that head only when heads are not shared: checked there
    o, lse = torch.full((B, H, N, d), 5.0, device="cuda").bfloat16(), torch.full((B, H, N), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o, rp, ci, lse=lse, schedule=sched)
    torch.cuda.synchronize()
    qn, on, ln = (t.double().cpu().numpy() for t in (q, o, lse))
    for p in range(B * H):
        bb, hh = divmod(p, H)
        mask = O.block_mask(og, k, rows[p * G_k:(p + 1) * G_k])
        kv = hh // (H // Hkv)
        check_rows(on[bb, hh], ln[bb, hh], qn[bb, hh], kk[bb, kv], vv[bb, kv], scale_of(d), mask=mask, what=f"plane {p}")
    return g, q, q8, o, rp, ci


@pytest.mark.parametrize("h,w,b,k,B,H,Hkv,d,G", [
    ([1, 2, 4, 8, 16], [1, 2, 4, 8, 16], 8, 5, 2, 2, 2, 128, 64),   # one chunk a tile
    ([1, 2, 4, 8, 12], [1, 2, 3, 6, 9], 8, 5, 1, 3, 3, 64, 32),     # tiles cut at the edges
    ([1, 3, 5, 7, 11], [1, 4, 6, 9, 13], 4, 5, 1, 4, 2, 128, 16),   # small tiles, shared heads
    ([1, 2, 4, 8, 20], [1, 2, 4, 8, 20], 16, 5, 1, 2, 1, 128, 128), # tiles of four chunks
    ([2, 9, 13], [2, 9, 13], 3, 3, 1, 2, 2, 64, 16), ([40], [70], 33, 1, 1, 1, 1, 64, 64),
    ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20, 64, 64), ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20, 128, 64),  # one part a row
    ([1, 4, 30], [1, 4, 30], 8, 3, 1, 20, 20, 64, 64), ([1, 4, 30], [1, 4, 30], 5, 3, 1, 2, 2, 128, 16),
    ([1, 70], [1, 70], 64, 2, 1, 1, 1, 128, 64),                    # tile rows of a whole chunk
    ([1, 2, 4, 8, 16, 29], [1, 2, 4, 8, 16, 25], 8, 6, 1, 4, 2, 128, 64),  # rows in four parts, edges of 5 and 1
    ([1, 2, 4, 8, 16, 25], [1, 2, 4, 8, 16, 29], 8, 6, 1, 3, 3, 64, 16),
    ([3, 12], [3, 12], 1, 2, 1, 1, 1, 64, 16), ([5, 9, 7], [1, 3, 2], 2, 3, 2, 2, 1, 128, 32)])  # blocks of one to four tokens
@pytest.mark.parametrize("order", [False, True])
def test_sparse(h, w, b, k, B, H, Hkv, d, G, order):
    note(f"[q8 sparse] h={h} w={w} b={b} k={k} B={B} H={H}/{Hkv} d={d} G={G} order={order}")
    run_sparse(h, w, b, k, B, H, Hkv, d, G, seed=sum(h) + b, empty=(0, 3), order=order)


def test_sparse_reads_only_listed_blocks():
    """Codes of every block that no row lists are NaN."""
    note("[q8 sparse] NaN in unlisted blocks")
    h, b, k, d, G = [1, 2, 4, 8, 16], 4, 5, 128, 16
    og, g = O.Geometry(h, h, b, 1), sv.Geometry(h, h, b, 1)
    q8, kk, vv = make_cache(1, 1, og.C(k), d, G, 3, scales=False)
    keep = [0, 1, 4, 6, og.nb_le(k) - 2]
    mask = O.block_mask(og, k, [keep] * og.tiles(k))
    dead = torch.from_numpy(~mask[0]).cuda()
    for t in (q8.k, q8.v):
        t.view(torch.uint8)[0, 0, dead] = 0x7f
    q = torch.randn(1, 1, og.N(k), d, device="cuda").bfloat16()
    o = torch.empty_like(q)
    rp = (torch.arange(og.tiles(k) + 1, device="cuda") * len(keep)).to(torch.int32)
    ci = torch.tensor(keep * og.tiles(k), dtype=torch.int32, device="cuda")
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o, rp, ci)
    torch.cuda.synchronize()
    check_rows(o[0, 0].double().cpu().numpy(), None, q[0, 0].double().cpu().numpy(), np.nan_to_num(kk[0, 0]),
               np.nan_to_num(vv[0, 0]), scale_of(d), mask=mask)


def test_sparse_long_rows():
    """More chunks than a table holds: 300 blocks a row, walked in several fills."""
    note("[q8 sparse] long rows")
    run_sparse([1, 36], [1, 36], 2, 2, 1, 1, 1, 64, 16, seed=9)


@pytest.mark.parametrize("d", [64, 128])
def test_sparse_long_rows_in_parts(d):
    """A small scale after a large one: few tiles, so rows in four parts, and more blocks than a fill decodes."""
    note(f"[q8 sparse] 534 blocks a row in parts, d={d}")
    h, k = [1, 184, 16], 3
    og, g = O.Geometry(h, h, 8, 1), sv.Geometry(h, h, 8, 1)
    q8, kk, vv = make_cache(1, 1, og.C(k), d, 64, 17)
    q = torch.randn(1, 1, og.N(k), d, device="cuda").bfloat16()
    nb, G_k = og.nb_le(k), og.tiles(k)
    assert nb == 534 and G_k == 4
    ids = [list(range(nb)), list(range(20, nb)), [0, 533], list(range(0, nb, 2))]
    ptr = np.cumsum([0] + [len(x) for x in ids])
    rp, ci = torch.from_numpy(ptr.astype(np.int32)).cuda(), torch.tensor(sum(ids, []), dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 5.0), torch.full((1, 1, og.N(k)), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o, rp, ci, lse=lse)
    torch.cuda.synchronize()
    check_rows(o[0, 0].double().cpu().numpy(), lse[0, 0].double().cpu().numpy(), q[0, 0].double().cpu().numpy(), kk[0, 0],
               vv[0, 0], scale_of(d), mask=O.block_mask(og, k, ids))


def test_every_block_is_dense():
    """All blocks listed: the dense call's result on the same cache, within both calls' bounds."""
    note("[q8 sparse] all blocks")
    h, k, d = [1, 2, 4, 8, 16], 5, 128
    og, g = O.Geometry(h, h, 8, 1), sv.Geometry(h, h, 8, 1)
    q8, kk, vv = make_cache(1, 2, og.C(k), d, 64, 21)
    q = torch.randn(1, 2, og.N(k), d, device="cuda").bfloat16()
    nb, G_k = og.nb_le(k), og.tiles(k)
    rp = (torch.arange(2 * G_k + 1, device="cuda") * nb).to(torch.int32)
    ci = torch.arange(nb, device="cuda").to(torch.int32).repeat(2 * G_k)
    o = [torch.empty_like(q) for _ in range(2)]
    sv.sparvar_block_sparse_attn_q8_fwd(g, k, q, q8, o[0], rp, ci)
    sv.sparvar_dense_attn_q8_fwd(q, q8, og.C(k), o[1])
    torch.cuda.synchronize()
    for x in o:
        for hh in range(2):
            check_rows(x[0, hh].double().cpu().numpy(), None, q[0, hh].double().cpu().numpy(), kk[0, hh], vv[0, hh], scale_of(d))


# ------------------------------------------------------------------------------------------------ together
def test_layer_over_the_8_bit_cache():
    """A whole layer from its projections: scale after scale appended and attended, the decision on the cache read back,
    sparse steps after it. Each step against the oracle on what the library's cache holds at that time."""
    note("[q8 layer]")
    h, S, steps, B, H, d, topk = [1, 2, 4, 6, 8, 12, 16], 5, [6, 7], 1, 2, 64, 2
    og, g = O.Geometry(h, h, 4, 2), sv.Geometry(h, h, 4, 2)
    r = np.random.default_rng(31)
    total = og.C(len(h))
    ang = r.uniform(-3, 3, (total, d // 2))
    cs = torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32)).cuda()
    heads = sv.NormRope("rms", 1e-6, torch.ones(H, d, device="cuda") * 1.5, torch.ones(H, d, device="cuda"), cs)
    path = Q8SparsePath(g, S, steps, B, H, d, topk, 1, heads=heads, block=32)
    for l in range(1, len(h) + 1):
        x = torch.from_numpy(r.standard_normal((B, og.N(l), 3 * H, d)).astype(np.float32)).cuda().bfloat16()
        q, k, v = x.split([H, H, H], 2)
        o = path.step(l, q, k, v)
        kv = [torch.empty(B, H, og.C(l), d, device="cuda") for _ in range(2)]
        sv.sparvar_kv_dequantize(path.q8, 0, kv[0], kv[1])
        torch.cuda.synchronize()
        for hh in range(H):
            kn, vn = (t[0, hh].double().cpu().numpy() for t in kv)
            # the newest values as they were encoded: half a step of the projection's value
            newest, given = vn[og.C(l - 1):], v[0, :, hh].double().cpu().numpy()
            assert (np.abs(newest - given) <= np.maximum(2.0 ** -4 * np.abs(given), 2.0 ** -10 * 2.0 ** -5)).all()
            mask = None
            if l in steps:
                rp, ci, _ = path.csr[l]
                rows = [[y for y in ci[rp[i]:rp[i + 1]].tolist() if y >= 0] for i in range(len(rp) - 1)]
                mask = O.block_mask(og, l, rows[hh * og.tiles(l):(hh + 1) * og.tiles(l)])
            check_rows(o[0, hh].double().cpu().numpy(), None, path.q[l][0, hh].double().cpu().numpy(), kn, vn, path.scale,
                       mask=mask, what=f"scale {l} head {hh}")


def test_streams_and_workspaces():
    """Two calls side by side on streams of their own, each with its own workspace and cache."""
    note("[q8 dense] two streams")
    B, H, Hkv, nkv, d = 2, 8, 2, 5000, 128
    jobs = []
    for s in range(2):
        q8, _, _ = make_cache(B, Hkv, nkv, d, 64, 40 + s)
        q = torch.randn(B, H, 1, d, device="cuda").bfloat16()
        ws = torch.empty(sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, 1, nkv, d), dtype=torch.uint8, device="cuda")
        jobs.append((q8, q, ws, torch.cuda.Stream(), torch.empty_like(q), torch.empty_like(q)))
    for q8, q, ws, _, alone, _ in jobs:
        sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, alone, workspace=ws)
    torch.cuda.synchronize()
    for _ in range(20):
        for q8, q, ws, stream, _, o in jobs:
            sv.sparvar_dense_attn_q8_fwd(q, q8, nkv, o, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for _, _, _, _, alone, o in jobs:
        assert torch.equal(alone, o)


def test_captured_step_replays():
    """Append, dense attention in parts and read-back captured into a graph: replays with new inputs in place, eager work
    between them, equal the eager results."""
    note("[q8 graph]")
    B, H, Hkv, d, n, t0, G = 1, 4, 2, 128, 3, 2000, 64
    r = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(B, n, H + 2 * Hkv, d, generator=r, device="cuda").bfloat16()
    q, k, v = x.split([H, Hkv, Hkv], 2)
    q8, _, _ = make_cache(B, Hkv, t0, d, G, 50, cap=t0 + 100)
    qo, o = torch.empty(B, H, n, d, device="cuda").bfloat16(), torch.empty(B, H, n, d, device="cuda").bfloat16()
    back = [torch.empty(B, Hkv, n, d, device="cuda") for _ in range(2)]
    ws = torch.empty(sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, n, t0 + n, d), dtype=torch.uint8, device="cuda")
    heads = sv.NormRope("rms", 1e-6)

    def step():
        sv.sparvar_qkv_append(q, k, v, t0, heads, qo, q8=q8)
        sv.sparvar_dense_attn_q8_fwd(qo, q8, t0 + n, o, workspace=ws)
        sv.sparvar_kv_dequantize(q8, t0, back[0], back[1])

    inputs = [torch.randn(x.shape, generator=r, device="cuda").bfloat16() for _ in range(3)]
    want = []
    for y in inputs:
        x.copy_(y)
        step()
        want.append([t.clone() for t in (qo, o, *back)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(2):
        for y, w in zip(inputs, want):
            x.copy_(torch.zeros_like(y))
            step()  # eager work of other inputs in between
            torch.cuda.synchronize()
            x.copy_(y)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(w, (qo, o, *back)):
                assert torch.equal(a, b), rep
