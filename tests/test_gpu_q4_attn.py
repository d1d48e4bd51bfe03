"""GPU parity of attention over a 4-bit cache, dense and block-sparse, through the C ABI, against the fp64 oracle on the
values that the codes stand for; the bounds are q4_helpers'."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv
from q4_helpers import U16, U24, check_rows, make_cache

pytestmark = pytest.mark.gpu


def workspace(B, H, Hkv, nq, nkv, d):
    size = sv.sparvar_dense_attn_q4_workspace(B, H, Hkv, nq, nkv, d)
    return torch.full((max(size, 16),), 0xff, dtype=torch.uint8, device="cuda")  # NaN in every float of it


def run_dense(B, H, Hkv, nq, nkv, d, lens=None, ws=False, seed=0, cap=None, pad=0):
    q4, k, v = make_cache(B, Hkv, nkv, d, seed + 1, cap)
    if lens is not None:  # what lies past a length is NaN
        for b, n in enumerate(lens):
            for t in (q4.k_scale, q4.v_scale):
                t[b, :, min(max(n, 0), nkv):] = 255
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(B, H, nq + pad, d, generator=g, device="cuda").bfloat16()[:, :, :nq]
    o, lse = torch.full((B, H, nq, d), 5.0, device="cuda").bfloat16(), torch.full((B, H, nq), 5.0, device="cuda")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse, kv_len=kv_len, workspace=workspace(B, H, Hkv, nq, nkv, d) if ws else None)
    torch.cuda.synchronize()
    qn, on, ln = (t.double().cpu().numpy() for t in (q, o, lse))
    r = np.random.default_rng(seed)
    rows = np.arange(nq) if nq <= 300 else np.unique(np.concatenate([[0, 1, nq - 2, nq - 1], r.choice(nq, 200, replace=False)]))
    for b in range(B):
        n = nkv if lens is None else min(max(lens[b], 0), nkv)
        for h in range(H):
            kv = h // (H // Hkv)
            check_rows(on[b, h][rows], ln[b, h][rows], qn[b, h][rows], k[b, kv, :n], v[b, kv, :n], scale_of(d),
                       what=f"entry {b} head {h}")


@pytest.mark.parametrize("B,H,Hkv,nq,nkv,d", [
    (1, 1, 1, 1, 1, 128), (2, 3, 3, 4, 5, 64), (1, 2, 2, 16, 21, 128), (2, 2, 2, 64, 121, 128), (1, 2, 2, 33, 63, 64),
    (1, 2, 2, 65, 64, 128), (1, 1, 1, 129, 65, 64), (1, 2, 1, 257, 300, 128), (1, 4, 2, 36, 57, 64), (2, 8, 2, 1, 777, 128),
    (1, 8, 1, 7, 1500, 64), (1, 16, 1, 5, 333, 128),
    # long enough for parts: few rows, odd lengths and more parts than chunks divide into
    (1, 8, 2, 1, 9001, 128), (1, 2, 2, 1, 20011, 64), (1, 8, 1, 6, 7777, 64), (1, 2, 2, 70, 8000, 128),
    # more rows than a join takes a workgroup each; sets of waves that share the keys; slabs of 128 and 256 rows
    (1, 4, 4, 700, 3000, 64), (1, 4, 2, 701, 3000, 128), (1, 20, 20, 1000, 1100, 128), (2, 8, 8, 646, 2755, 64),
    (1, 12, 12, 1030, 2500, 128), (2, 8, 8, 900, 1000, 128), (2, 8, 8, 900, 1000, 64), (2, 16, 16, 1600, 200, 64)])
@pytest.mark.parametrize("ws", [False, True])
def test_dense(B, H, Hkv, nq, nkv, d, ws):
    note(f"[q4 dense] B={B} H={H}/{Hkv} nq={nq} nkv={nkv} d={d} ws={ws}")
    run_dense(B, H, Hkv, nq, nkv, d, ws=ws, seed=nq + nkv, cap=nkv + 70, pad=3)


@pytest.mark.parametrize("ws", [False, True])
@pytest.mark.parametrize("nq,nkv,d", [(1, 4000, 128), (20, 900, 64), (100, 500, 128), (1000, 300, 128), (1000, 1500, 128),
                                      (700, 5000, 64), (540, 1500, 64)])
def test_dense_lengths(nq, nkv, d, ws):
    """Lengths of their own: none, negative, one, a chunk's edge, past the end; what lies past a length is NaN."""
    note(f"[q4 dense] lengths nq={nq} nkv={nkv} d={d} ws={ws}")
    run_dense(10, 2, 1, nq, nkv, d, lens=[0, -3, 1, 63, 64, 65, 200, nkv - 1, nkv, nkv + 99], ws=ws, seed=7)


@pytest.mark.parametrize("ws", [False, True])
@pytest.mark.parametrize("nq,nkv,d", [(1, 20000, 128), (3, 9000, 64), (300, 500, 128), (2000, 300, 64)])
def test_dense_nan(nq, nkv, d, ws):
    """A NaN among the keys makes its plane's rows NaN, one among the values its 32 channels, in every form and in parts;
    other planes and lengths that end before it are as they were."""
    note(f"[q4 dense] NaN nq={nq} nkv={nkv} d={d} ws={ws}")
    q4, k, v = make_cache(3, 2, nkv, d, 5)
    at = nkv - 70
    q4.k_scale[0, 0, at, 1] = 255
    q4.v_scale[0, 1, at, 0] = 255
    q4.k_scale[1, 0, at, 0] = 255
    q = torch.randn(3, 2, nq, d, device="cuda").bfloat16()
    o, lse = torch.full_like(q, 5.0), torch.full((3, 2, nq), 5.0, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse, kv_len=torch.tensor([nkv, at, nkv], dtype=torch.int32, device="cuda"),
                                 workspace=workspace(3, 2, 2, nq, nkv, d) if ws else None)
    torch.cuda.synchronize()
    assert torch.isnan(o[0, 0]).all() and torch.isnan(lse[0, 0]).all()
    assert torch.isnan(o[0, 1, :, :32]).all() and not torch.isnan(lse[0, 1]).any()
    qn, on = q.double().cpu().numpy(), o.double().cpu().numpy()
    check_rows(on[0, 1][:, 32:], None, qn[0, 1], k[0, 1], v[0, 1][:, 32:], scale_of(d), what="channels without")
    for b, h, n in ((1, 0, at), (1, 1, at), (2, 0, nkv), (2, 1, nkv)):
        check_rows(on[b, h], None, qn[b, h], k[b, h, :n], v[b, h, :n], scale_of(d), what=f"entry {b} head {h}")


def test_dense_full_size():
    """The last scale of a 1024x1024 image, rows sampled."""
    note("[q4 dense] 4096 x 10521")
    run_dense(1, 8, 8, 4096, 10521, 128, seed=11)


@pytest.mark.parametrize("rows", [20, 300])
def test_scores_that_spread(rows):
    """Scores far apart (one key takes all, the maximum grows along the walk) and equal ones."""
    note(f"[q4 dense] spread scores, {rows} rows")
    B, H, d, nkv = 1, 1, 64, 500
    q4 = sv.Q4Cache.empty(B, H, nkv, d)
    x = torch.zeros(2, B, H, nkv, d, device="cuda")
    x[0, ..., 0] = 2.0 ** (torch.arange(nkv, device="cuda") // 50).float()   # ascending scores
    x[1] = torch.randn(B, H, nkv, d, device="cuda")
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, q4)
    kv = [torch.empty(B, H, nkv, d, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize_q4(q4, 0, kv[0], kv[1])
    q = torch.zeros(B, H, rows, d, device="cuda").bfloat16()
    q[0, 0, :4, 0] = torch.tensor([100.0, -100.0, 0.0, 0.0078125])
    for ws in (False, True):
        o, lse = torch.empty_like(q), torch.empty(B, H, rows, device="cuda")
        sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse, softmax_scale=1.0, workspace=workspace(B, H, H, rows, nkv, d) if ws else None)
        torch.cuda.synchronize()
        k, v, qn = kv[0][0, 0].double().cpu().numpy(), kv[1][0, 0].double().cpu().numpy(), q[0, 0].double().cpu().numpy()
        got = o[0, 0].double().cpu().numpy()
        check_rows(got[2:], lse[0, 0].double().cpu().numpy()[2:], qn[2:], k, v, 1.0, what="small scores")
        for i in (0, 1):
            s = qn[i] @ k.T
            top = np.flatnonzero(s >= s.max())
            ref = v[top].mean(0)
            assert (np.abs(got[i] - ref) <= 1.02 * U16 * (np.abs(v[top]).mean(0) + np.abs(ref)) + 1e-30).all()


def outliers(q, k, v, o, lse, scale, mask=None):
    """One head whose queries' elements lie far apart. With u the power of two that brings a row's largest into (224, 448],
    elements of 2^-6 u and more are exact and the others off by at most 2^-14 u, so a score is off by at most
    scale (2^-14 u sum |k_j| over those + d 2^-23 sum |q_j k_j|), the second term for products summed in 32 bits; the LSE by
    its worst score and by 8 2^-24 max |s| + (n + 16) 2^-24. An LSE is held to both, that and 2e-4."""
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
    bound = off.max(1) + 8 * U24 * np.abs(np.where(np.isfinite(s), s, 0.0)).max(1) + (n + 16) * U24
    err = np.abs(lse - (m + np.log(l)))
    assert (err <= np.minimum(bound, 2e-4)).all(), f"LSE off by {err.max():.2e}, {(err / bound).max():.1f} of the bound"
    p /= l[:, None]
    ref, size = p @ v, p @ np.abs(v)
    assert (np.abs(o - ref) <= 1.02 * U16 * (size + np.abs(ref)) + 2 * bound[:, None] * size + 1e-30).all()


@pytest.mark.parametrize("top,rest", [(100.0, 0.1), (150.0, 0.15)])
@pytest.mark.parametrize("H,nq,nkv,d", [(1, 3, 64, 128), (16, 1600, 64, 128), (32, 1600, 64, 64)])
def test_outlier_channel(H, nq, nkv, d, top, rest):
    """Few rows (bf16 products) and many (the two parts): one channel many times the others, keys large where it is not."""
    note(f"[q4 dense] outlier {top} beside {rest}, H={H} nq={nq} nkv={nkv} d={d}")
    g = torch.Generator(device="cuda").manual_seed(nq + d)
    q = torch.randn(1, H, nq, d, generator=g, device="cuda") * rest
    q[..., 5] = top
    q = q.bfloat16()
    x = torch.randn(2, 1, H, nkv, d, generator=g, device="cuda")
    x[0] *= 4.0
    x[0, ..., 5] = 0.0
    q4 = sv.Q4Cache.empty(1, H, nkv, d)
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, q4)
    kv = [torch.empty(1, H, nkv, d, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize_q4(q4, 0, kv[0], kv[1])
    o, lse = torch.empty_like(q), torch.empty(1, H, nq, device="cuda")
    sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, lse=lse)
    torch.cuda.synchronize()
    k, v, qn, on, ln = (t.double().cpu().numpy() for t in (*kv, q, o, lse))
    for h in range(H):
        outliers(qn[0, h], k[0, h], v[0, h], on[0, h], ln[0, h], scale_of(d))


# ------------------------------------------------------------------------------------------------ block-sparse
def run_sparse(h, w, b, k, B, H, Hkv, d, seed, empty=(), order=False):
    og, g = O.Geometry(h, w, b, 1), sv.Geometry(h, w, b, 1)
    q4, kk, vv = make_cache(B, Hkv, og.C(k), d, seed, cap=og.C(k) + 9)
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
    o, lse = torch.full((B, H, N, d), 5.0, device="cuda").bfloat16(), torch.full((B, H, N), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q4_fwd(g, k, q, q4, o, rp, ci, lse=lse, schedule=sched)
    torch.cuda.synchronize()
    qn, on, ln = (t.double().cpu().numpy() for t in (q, o, lse))
    for p in range(B * H):
        bb, hh = divmod(p, H)
        mask = O.block_mask(og, k, rows[p * G_k:(p + 1) * G_k])
        kv = hh // (H // Hkv)
        check_rows(on[bb, hh], ln[bb, hh], qn[bb, hh], kk[bb, kv], vv[bb, kv], scale_of(d), mask=mask, what=f"plane {p}")


@pytest.mark.parametrize("h,w,b,k,B,H,Hkv,d", [
    ([1, 2, 4, 8, 16], [1, 2, 4, 8, 16], 8, 5, 2, 2, 2, 128),   # one chunk a tile
    ([1, 2, 4, 8, 12], [1, 2, 3, 6, 9], 8, 5, 1, 3, 3, 64),     # tiles cut at the edges
    ([1, 3, 5, 7, 11], [1, 4, 6, 9, 13], 4, 5, 1, 4, 2, 128),   # small tiles, shared heads
    ([1, 2, 4, 8, 20], [1, 2, 4, 8, 20], 16, 5, 1, 2, 1, 128),  # tiles of four chunks
    ([2, 9, 13], [2, 9, 13], 3, 3, 1, 2, 2, 64), ([40], [70], 33, 1, 1, 1, 1, 64),
    ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20, 64), ([1, 4, 30], [1, 4, 30], 8, 3, 2, 20, 20, 128),  # one part a row
    ([1, 4, 30], [1, 4, 30], 8, 3, 1, 20, 20, 64), ([1, 4, 30], [1, 4, 30], 5, 3, 1, 2, 2, 128),
    ([1, 2, 4, 8, 23], [1, 2, 4, 8, 20], 9, 5, 2, 3, 1, 64), ([1, 2, 4, 8, 24], [1, 2, 4, 8, 25], 11, 5, 1, 4, 4, 128),
    ([1, 2, 4, 8, 20], [1, 2, 4, 8, 35], 16, 5, 1, 2, 2, 64),
    ([1, 70], [1, 70], 64, 2, 1, 1, 1, 128),                    # tile rows of a whole chunk
    ([1, 2, 4, 8, 16, 29], [1, 2, 4, 8, 16, 25], 8, 6, 1, 4, 2, 128),  # rows in four parts, edges of 5 and 1
    ([1, 2, 4, 8, 16, 25], [1, 2, 4, 8, 16, 29], 8, 6, 1, 3, 3, 64),
    ([3, 12], [3, 12], 1, 2, 1, 1, 1, 64), ([5, 9, 7], [1, 3, 2], 2, 3, 2, 2, 1, 128),  # blocks of one to four tokens
    ([1, 36], [1, 36], 2, 2, 1, 1, 1, 64)])                     # 300 blocks a row, in several fills
@pytest.mark.parametrize("order", [False, True])
def test_sparse(h, w, b, k, B, H, Hkv, d, order):
    note(f"[q4 sparse] h={h} w={w} b={b} k={k} B={B} H={H}/{Hkv} d={d} order={order}")
    run_sparse(h, w, b, k, B, H, Hkv, d, seed=sum(h) + b, empty=(0, 3), order=order)


def test_sparse_reads_only_listed_blocks():
    """Every block that no row lists is NaN."""
    note("[q4 sparse] NaN in unlisted blocks")
    h, b, k, d = [1, 2, 4, 8, 16], 4, 5, 128
    og, g = O.Geometry(h, h, b, 1), sv.Geometry(h, h, b, 1)
    q4, kk, vv = make_cache(1, 1, og.C(k), d, 3)
    keep = [0, 1, 4, 6, og.nb_le(k) - 2]
    mask = O.block_mask(og, k, [keep] * og.tiles(k))
    dead = torch.from_numpy(~mask[0]).cuda()
    for t in (q4.k_scale, q4.v_scale):
        t[0, 0, dead] = 255
    q = torch.randn(1, 1, og.N(k), d, device="cuda").bfloat16()
    o = torch.empty_like(q)
    rp = (torch.arange(og.tiles(k) + 1, device="cuda") * len(keep)).to(torch.int32)
    ci = torch.tensor(keep * og.tiles(k), dtype=torch.int32, device="cuda")
    sv.sparvar_block_sparse_attn_q4_fwd(g, k, q, q4, o, rp, ci)
    torch.cuda.synchronize()
    check_rows(o[0, 0].double().cpu().numpy(), None, q[0, 0].double().cpu().numpy(), kk[0, 0], vv[0, 0], scale_of(d), mask=mask)


@pytest.mark.parametrize("d", [64, 128])
def test_sparse_long_rows_in_parts(d):
    """A small scale after a large one: few tiles, so rows in four parts, and more blocks than a fill decodes."""
    note(f"[q4 sparse] 534 blocks a row in parts, d={d}")
    h, k = [1, 184, 16], 3
    og, g = O.Geometry(h, h, 8, 1), sv.Geometry(h, h, 8, 1)
    q4, kk, vv = make_cache(1, 1, og.C(k), d, 17)
    q = torch.randn(1, 1, og.N(k), d, device="cuda").bfloat16()
    nb = og.nb_le(k)
    ids = [list(range(nb)), list(range(20, nb)), [0, 533], list(range(0, nb, 2))]
    ptr = np.cumsum([0] + [len(x) for x in ids])
    rp, ci = torch.from_numpy(ptr.astype(np.int32)).cuda(), torch.tensor(sum(ids, []), dtype=torch.int32, device="cuda")
    o, lse = torch.full_like(q, 5.0), torch.full((1, 1, og.N(k)), 5.0, device="cuda")
    sv.sparvar_block_sparse_attn_q4_fwd(g, k, q, q4, o, rp, ci, lse=lse)
    torch.cuda.synchronize()
    check_rows(o[0, 0].double().cpu().numpy(), lse[0, 0].double().cpu().numpy(), q[0, 0].double().cpu().numpy(), kk[0, 0],
               vv[0, 0], scale_of(d), mask=O.block_mask(og, k, ids))


# ------------------------------------------------------------------------------------------------ together
def test_streams_and_workspaces():
    """Two calls side by side on streams of their own, each with its own workspace and cache."""
    note("[q4 dense] two streams")
    B, H, Hkv, nkv, d = 2, 8, 2, 5000, 128
    jobs = []
    for s in range(2):
        q4, _, _ = make_cache(B, Hkv, nkv, d, 40 + s)
        q = torch.randn(B, H, 1, d, device="cuda").bfloat16()
        jobs.append((q4, q, workspace(B, H, Hkv, 1, nkv, d), torch.cuda.Stream(), torch.empty_like(q), torch.empty_like(q)))
    for q4, q, ws, _, alone, _ in jobs:
        sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, alone, workspace=ws)
    torch.cuda.synchronize()
    for _ in range(20):
        for q4, q, ws, stream, _, o in jobs:
            sv.sparvar_dense_attn_q4_fwd(q, q4, nkv, o, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for _, _, _, _, alone, o in jobs:
        assert torch.equal(alone, o)
