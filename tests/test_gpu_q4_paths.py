"""The operators of the 4-bit cache together, as layers use them: a sparse layer from its projections, a dense layer held to a
budget of tokens, and such a step captured into a graph."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv
from paper_2602_04361_amd.pipeline import BudgetPath, Q4SparsePath
from q4_helpers import check_rows, make_cache, values_of
from test_gpu_key_weights import expected

pytestmark = pytest.mark.gpu


def table(r, rows, d):
    ang = r.uniform(-3, 3, (rows, d // 2))
    return torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32)).cuda()


def same_codes(cache, t0, k, v):
    """The cache's tokens from t0 on hold what rows k, v [B,H,n,d] are in 4 bits."""
    n = k.shape[2]
    for c, s, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
        c, s = c.cpu().numpy()[:, :, t0:t0 + n], s.cpu().numpy()[:, :, t0:t0 + n]
        for b in range(k.shape[0]):
            for h in range(k.shape[1]):
                assert np.array_equal(O.decode_rows(c[b, h], s[b, h]), O.decode_rows(*O.encode_rows(x[b, h].double().cpu().numpy())))


def test_sparse_layer():
    """Scale after scale appended and attended, the decision on the cache read back, sparse steps after it, each against the
    oracle on what the library's cache holds at that time."""
    note("[q4 layer]")
    h, S, steps, B, H, d, topk = [1, 2, 4, 6, 8, 12, 16], 5, [6, 7], 1, 2, 64, 2
    og, g = O.Geometry(h, h, 4, 2), sv.Geometry(h, h, 4, 2)
    r = np.random.default_rng(31)
    heads = sv.NormRope("rms", 1e-6, torch.ones(H, d, device="cuda") * 1.5, torch.ones(H, d, device="cuda"), table(r, og.C(len(h)), d))
    path = Q4SparsePath(g, S, steps, B, H, d, topk, 1, heads=heads)
    # the 16-bit append of the whole cache at once, for comparison
    total = og.C(len(h))
    kc, vc, qo = (torch.empty(B, H, total, d, device="cuda").bfloat16() for _ in range(3))
    for l in range(1, len(h) + 1):
        x = torch.from_numpy(r.standard_normal((B, og.N(l), 3 * H, d)).astype(np.float32)).cuda().bfloat16()
        q, k, v = x.split([H, H, H], 2)
        o = path.step(l, q, k, v)
        t0, n = og.C(l - 1), og.N(l)
        ql = torch.empty(B, H, n, d, device="cuda").bfloat16()
        sv.sparvar_qkv_append(q, k, v, t0, heads, ql, kc, vc)
        torch.cuda.synchronize()
        assert torch.equal(ql, path.q[l])
        same_codes(path.q4, t0, kc[:, :, t0:t0 + n], vc[:, :, t0:t0 + n])
        kn, vn = values_of(path.q4)
        for hh in range(H):
            mask = None
            if l in steps:
                rp, ci, _ = path.csr[l]
                rows = [[y for y in ci[rp[i]:rp[i + 1]].tolist() if y >= 0] for i in range(len(rp) - 1)]
                mask = O.block_mask(og, l, rows[hh * og.tiles(l):(hh + 1) * og.tiles(l)])
            check_rows(o[0, hh].double().cpu().numpy(), None, path.q[l][0, hh].double().cpu().numpy(), kn[0, hh, :og.C(l)],
                       vn[0, hh, :og.C(l)], path.scale, mask=mask, what=f"scale {l} head {hh}")


@pytest.mark.parametrize("H,H_kv,d,budget,first,last,decay,steps", [
    (4, 2, 64, 50, 5, 10, 1.0, [1, 4, 16, 36, 36, 1, 1, 30]), (2, 2, 128, 200, 0, 0, 0.9, [64, 1, 100, 200, 1, 144]),
    (8, 1, 128, 7, 1, 1, 0.5, [5, 1, 1, 1, 1, 3, 1])])
def test_budget_layer(H, H_kv, d, budget, first, last, decay, steps):
    """Every step: the cache's rows, attention over it, its weights and what stays, each against the oracle on what the
    library held before."""
    note(f"[budget layer] H={H}/{H_kv} d={d} budget={budget}")
    B, r = 2, np.random.default_rng(budget)
    heads = sv.NormRope("l2", 1e-6, torch.full((H, d), 4.0, device="cuda"), torch.full((H_kv, d), 4.0, device="cuda"),
                        table(r, sum(steps), d))
    path = BudgetPath(B, H, H_kv, d, max(steps), budget, first, last, heads=heads, decay=decay)
    seen = 0
    for n in steps:
        x = torch.from_numpy(r.standard_normal((B, n, H + 2 * H_kv, d)).astype(np.float32)).cuda().bfloat16()
        q, k, v = x.split([H, H_kv, H_kv], 2)
        held = path.held
        old = path.w.double().cpu().numpy()[:, :, :held].copy()
        path.append(q, k, v)
        kc, vc, ql = (torch.empty(B, hh, seen + n, d, device="cuda").bfloat16() for hh in (H_kv, H_kv, H))
        qa = torch.empty(B, H, n, d, device="cuda").bfloat16()
        sv.sparvar_qkv_append(q, k, v, seen, heads, qa, kc, vc)
        torch.cuda.synchronize()
        same_codes(path.q4, held, kc[:, :, seen:], vc[:, :, seen:])
        seen += n
        path.attend()
        path.weigh()
        torch.cuda.synchronize()
        kn, vn = values_of(path.q4)
        qn, on, ln, wn = (t.double().cpu().numpy() for t in (qa, path.out, path.lse, path.w))
        m = held + n
        for b in range(B):
            for hh in range(H):
                g = hh * H_kv // H
                check_rows(on[b, hh], ln[b, hh], qn[b, hh], kn[b, g, :m], vn[b, g, :m], path.scale)
            for g in range(H_kv):
                rep = H // H_kv
                had = np.concatenate([old[b, g], np.zeros(n)])
                want, bound = expected(qn[b, g * rep:(g + 1) * rep].reshape(-1, d), kn[b, g, :m],
                                       ln[b, g * rep:(g + 1) * rep].reshape(-1), path.scale, had, decay)
                assert (np.abs(wn[b, g, :m] - want) <= bound).all()
        tokens = path.tokens.cpu().numpy()
        path.evict()
        torch.cuda.synchronize()
        assert path.held == min(m, budget)
        k2, v2 = values_of(path.q4)
        w2 = path.w.double().cpu().numpy()
        for b in range(B):
            for g in range(H_kv):
                stay = O.kept_tokens(wn[b, g, :m], budget, first, last)
                assert path.tokens[b, g].tolist() == tokens[b, g][stay].tolist()
                for a, c in ((k2, kn), (v2, vn), (w2, wn)):
                    assert np.array_equal(a[b, g, :len(stay)], c[b, g][stay])


def test_captured_step_replays():
    """Rows written, dense attention in parts, weights added up and the cache evicted from, captured into one graph: replays
    with new inputs in place, eager work and synchronizations between them, equal the eager results."""
    note("[q4 graph]")
    B, H, Hkv, d, n, t0, keep = 1, 8, 2, 128, 3, 4000, 2500
    total = t0 + n
    g = torch.Generator(device="cuda").manual_seed(5)
    q4, _, _ = make_cache(B, Hkv, t0, d, 50, cap=total)
    dst = sv.Q4Cache.empty(B, Hkv, keep, d)
    x = torch.randn(3, B, H, n, d, generator=g, device="cuda").bfloat16()
    q, k, v = x[0], x[1][:, :Hkv], x[2][:, :Hkv]
    o, lse = torch.empty_like(q), torch.empty(B, H, n, device="cuda")
    w0 = torch.rand(B, Hkv, total, generator=g, device="cuda") * 0.01
    w, wo = torch.empty_like(w0), torch.empty(B, Hkv, keep, device="cuda")
    kept = torch.empty(B, Hkv, keep, dtype=torch.int32, device="cuda")
    ko, vo = (torch.empty(B, Hkv, keep, d, device="cuda").bfloat16() for _ in range(2))
    size = sv.sparvar_dense_attn_q4_workspace(B, H, Hkv, n, total, d)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step():
        sv.sparvar_kv_quantize_q4(k, v, t0, q4)
        sv.sparvar_dense_attn_q4_fwd(q, q4, total, o, lse=lse, workspace=ws)
        sv.sparvar_key_weights(q, total, lse, w, w_old=w0, n_old=t0, decay=0.9, q4=q4)
        sv.sparvar_kv_evict(w, total, keep, 4, n, kept, wo, q4_src=q4, q4_dst=dst)
        sv.sparvar_kv_dequantize_q4(dst, 0, ko, vo)

    outs = (o, lse, w, kept, wo, ko, vo)
    inputs = [torch.randn(x.shape, generator=g, device="cuda").bfloat16() for _ in range(3)]
    want = []
    for y in inputs:
        x.copy_(y)
        step()
        want.append([t.clone() for t in outs])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(2):
        for y, ws_ in zip(inputs, want):
            x.copy_(torch.zeros_like(y))
            step()  # eager work of other inputs in between
            torch.cuda.synchronize()
            x.copy_(y)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(ws_, outs):
                assert torch.equal(a, b), rep
