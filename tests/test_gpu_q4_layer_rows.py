"""The rows that a sparse layer over a 4-bit cache attends by, each step of the decision against the oracle: the cache read back,
the pooled scores on it, the blocks of the largest, and where they lie at later scales."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import csr_rows, note
from paper_2602_04361_amd import sparvar as sv
from paper_2602_04361_amd.pipeline import Q4SparsePath
from q4_helpers import values_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,topk,radius,dilation,projection", [(64, 2, 1, 0, "point"), (128, 3, 1, 1, "cover"), (64, 40, 2, 0, "point")])
def test_rows_of_the_decision(d, topk, radius, dilation, projection):
    note(f"[q4 layer rows] d={d} topk={topk} radius={radius} dilation={dilation} {projection}")
    h, S, steps, B, H = [1, 2, 4, 6, 8, 12, 16], 5, [6, 7], 2, 3
    og, g = O.Geometry(h, h, 4, 2), sv.Geometry(h, h, 4, 2)
    r = np.random.default_rng(d + topk)
    path = Q4SparsePath(g, S, steps, B, H, d, topk, radius, prev_dilation=dilation, projection=projection)
    for l in range(1, len(h) + 1):
        x = torch.from_numpy(r.standard_normal((B, og.N(l), 3 * H, d)).astype(np.float32)).cuda().bfloat16()
        path.step(l, *x.split([H, H, H], 2))
        if l != S:
            continue
        torch.cuda.synchronize()
        kn, vn = values_of(path.q4)
        C1, G_S, NB = og.C(S), og.tiles(S), og.nb_le(S)
        for got, want in zip(path.kv_S, (kn, vn)):  # exact in bf16
            assert np.array_equal(got.double().cpu().numpy(), want[:, :, :C1])
        scores, idx = path.scores.cpu().numpy().reshape(B * H, G_S, NB), path.topk_idx.cpu().numpy().reshape(B * H, G_S, topk)
        q = path.q[S].double().cpu().numpy()
        sizes = np.array([len(og.tile_local_tokens(S, t // og.Tw(S), t % og.Tw(S))) for t in range(G_S)])
        for bh in range(B * H):
            want = O.pooled_scores(q[bh // H, bh % H], kn[bh // H, bh % H, :C1], path.scale, og, S)
            err = np.abs(scores[bh] - want) / sizes[:, None]
            assert err.max() <= 1e-4, f"head {bh}: {err.max():.3e}"  # (the decision's tolerance, by query)
            assert [row.tolist() for row in idx[bh]] == [O.topk_blocks(scores[bh, t], topk) for t in range(G_S)]
        for k in steps:
            rows = O.build_rows(og, S, k, idx, O.local_blocks(og, k, radius, dilation), projection=projection)
            assert csr_rows(*path.csr[k][:2], padded=True) == [row for per in rows for row in per], f"rows of scale {k}"
