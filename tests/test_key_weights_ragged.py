"""Weights of caches whose entries have lengths of their own: what a key had counts up to the length its entry had, and nothing
that was never written does. Bounds as in the tests of sparvar_key_weights."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note, scale_of
from paper_2602_04361_amd import sparvar as sv

CACHES = ["bf16", "f32", "q4"]
FAKE = 1 << 20  # never dereferenced: validation fails first


def test_refusals():
    """The checks of the call without lengths, and the binding's own."""
    a = [2, 4, 2, 10, 100, 64, sv.BF16, FAKE, 640, FAKE, 6400, None, FAKE, None, FAKE, 100, FAKE, 1.0, FAKE, 100, 0.1, None]
    lib = sv.load_library()
    for at, bad, status in ((5, 32, sv.ERR_UNSUPPORTED), (1, 3, sv.ERR_INVALID), (7, None, sv.ERR_INVALID), (9, None, sv.ERR_INVALID),
                            (12, None, sv.ERR_INVALID), (14, None, sv.ERR_INVALID), (15, -1, sv.ERR_INVALID), (15, 101, sv.ERR_INVALID),
                            (17, -0.5, sv.ERR_INVALID), (18, None, sv.ERR_INVALID), (19, 99, sv.ERR_INVALID), (20, 0.0, sv.ERR_INVALID)):
        assert lib.sparvar_key_weights_ragged(*[bad if i == at else x for i, x in enumerate(a)]) == status, (at, bad)
        assert lib.sparvar_last_error()
    q, w = torch.zeros(1, 2, 64, 64).bfloat16(), torch.zeros(1, 2, 64)
    with pytest.raises(sv.SparvarError, match="not on a GPU"):
        sv.sparvar_key_weights(q, 64, w, w, w_old=w, old_len=torch.zeros(1, dtype=torch.int32), q4=sv.Q4Cache.empty(1, 2, 64, 64, device="cpu"))


@pytest.mark.gpu
def test_binding_refusals():
    note("[ragged] refusals")
    q, w = torch.zeros(2, 2, 64, 64, device="cuda").bfloat16(), torch.zeros(2, 2, 64, device="cuda")
    for bad in (torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                torch.zeros(4, dtype=torch.int32, device="cuda")[::2], torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(sv.SparvarError):
            sv.sparvar_key_weights(q, 64, w, w, w_old=w, old_len=bad, k_cache=q)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,nkv,d", [(1, 3000, 128), (40, 300, 64), (200, 300, 64), (130, 900, 128), (200, 3000, 128)])
@pytest.mark.parametrize("cache", CACHES)
def test_ragged(cache, nq, nkv, d):
    """In place: NaN from each entry's old length on, and past its new one."""
    from test_gpu_key_weights import expected, keys

    note(f"[ragged] {cache} nq={nq} nkv={nkv} d={d}")
    old = [0, -4, 1, 31, 32, nkv - 1, nkv, nkv + 9, 100]
    new = [5, 40, 33, 32, nkv, nkv, nkv, nkv, 60]  # (the last entry got shorter)
    B, H, Hkv, limit = len(old), 2, 1, nkv - 3
    args, k = keys(cache, B, Hkv, nkv, d, 5)
    g = torch.Generator(device="cuda").manual_seed(nq)
    q = torch.randn(B, H, nq, d, generator=g, device="cuda")
    q = q if cache == "f32" else q.bfloat16()
    lse = torch.rand(B, H, nq, generator=g, device="cuda") + 6
    w = torch.rand(B, Hkv, nkv + 2, generator=g, device="cuda") * 5
    had = [min(max(n, 0), limit) for n in old]
    for b, n in enumerate(had):
        w[b, :, n:] = float("nan")
    before = w.double().cpu().numpy()
    sv.sparvar_key_weights(q, nkv, lse, w, w_old=w, n_old=limit, old_len=torch.tensor(old, dtype=torch.int32, device="cuda"), decay=0.75,
                           kv_len=torch.tensor(new, dtype=torch.int32, device="cuda"), **args)
    torch.cuda.synchronize()
    got, qn, ln = (t.double().cpu().numpy() for t in (w, q, lse))
    for b in range(B):
        n = min(new[b], nkv)
        prior = np.zeros(n)
        m = min(n, had[b])
        prior[:m] = before[b, 0, :m]
        want, bound = expected(qn[b].reshape(-1, d), k[b, 0, :n], ln[b].reshape(-1), scale_of(d), prior, 0.75)
        assert (np.abs(got[b, 0, :n] - want) <= bound).all(), b
        assert np.array_equal(got[b, 0, n:], before[b, 0, n:], equal_nan=True), b


@pytest.mark.gpu
def test_steps_with_eviction():
    """Entries that grow by numbers of their own, attended, weighed and evicted from again and again, in buffers that hold NaN
    wherever nothing was written: the kept tokens and their weights are those of every entry run by itself."""
    note("[ragged] steps")
    B, H, Hkv, d, budget, first, last = 3, 4, 2, 64, 50, 4, 6
    steps = [[30, 1, 49], [15, 1, 1], [10, 20, 1], [1, 40, 30], [7, 1, 1]]
    cap = budget + 49
    g = torch.Generator(device="cuda").manual_seed(2)

    def run(entries):
        n = len(entries)
        cache = [[torch.full((n, Hkv, cap, d), float("nan"), device="cuda").bfloat16() for _ in range(2)] for _ in range(2)]
        w = [torch.full((n, Hkv, cap), float("nan"), device="cuda") for _ in range(2)]
        order = [[[] for _ in range(Hkv)] for _ in range(n)]
        lens, seen = [0] * n, [0] * n
        for s, counts in enumerate(steps):
            old = list(lens)
            q = torch.stack([queries[s][e] for e in entries])
            for i, e in enumerate(entries):
                m = counts[e]
                for c, x in zip(cache[0], rows[e]):
                    c[i, :, lens[i]:lens[i] + m] = x[:, seen[i]:seen[i] + m]
                for o in order[i]:
                    o.extend(range(seen[i], seen[i] + m))
                lens[i] += m
                seen[i] += m
            top = max(lens)
            dev = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, old)]
            # (LSE in fp32 by elementary operations: attention over an entry's own length)
            lse = torch.empty(n, H, q.shape[2], device="cuda")
            for i in range(n):
                kk = cache[0][0][i, :, :lens[i]].float().repeat_interleave(H // Hkv, 0)
                lse[i] = torch.logsumexp((q[i].float()[:, :, None] * kk[:, None]).sum(3) * scale_of(d), 2)
            sv.sparvar_key_weights(q, top, lse, w[0], w_old=w[0], old_len=dev[1], kv_len=dev[0], decay=0.9, k_cache=cache[0][0])
            kept = torch.empty(n, Hkv, budget, dtype=torch.int32, device="cuda")
            sv.sparvar_kv_evict(w[0], top, budget, first, last, kept, w[1], *cache[0], *cache[1], kv_len=dev[0])
            torch.cuda.synchronize()
            for i in range(n):
                for h in range(Hkv):
                    want = O.kept_tokens(w[0][i, h, :lens[i]].cpu().numpy(), budget, first, last)
                    assert not torch.isnan(w[0][i, h, :lens[i]]).any()
                    assert kept[i, h].tolist() == want + [-1] * (budget - len(want))
                    order[i][h] = [order[i][h][t] for t in want]
                lens[i] = min(lens[i], budget)
            cache.reverse()
            w.reverse()
        return order, [w[0][i, :, :lens[i]] for i in range(n)]

    rows = [torch.randn(2, Hkv, sum(s[e] for s in steps), d, generator=g, device="cuda").bfloat16() for e in range(B)]
    queries = [torch.randn(B, H, 3, d, generator=g, device="cuda").bfloat16() for _ in steps]
    together, weights = run([0, 1, 2])
    for e in range(B):
        alone, w = run([e])
        assert alone[0] == together[e]
        assert torch.equal(w[0], weights[e])
