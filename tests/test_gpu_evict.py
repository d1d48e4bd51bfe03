"""GPU parity of eviction, through the C ABI: kept tokens, weights and rows bit-exact against sorting."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv

pytestmark = pytest.mark.gpu


def weights(kind, shape, g):
    w = torch.rand(*shape, generator=g, device="cuda")
    if kind == "spread":
        return torch.exp(6 * torch.randn(*shape, generator=g, device="cuda")) * (w > 0.1)
    if kind == "ties":  # few values, many of each; both zeros
        return torch.tensor([0.0, -0.0, 1.0, 1.0000001, 2.0, -1.0], device="cuda")[(w * 6).long()]
    if kind == "equal":
        return torch.full(shape, 0.25, device="cuda")
    if kind.startswith("every"):  # one of 128 far above the others, or far below: a sample of some is like none of them
        at = torch.arange(shape[-1], device="cuda") * 128 % (shape[-1] - 3) < 128
        return torch.where(at, w + (9 if kind == "every high" else -9), w)
    if kind == "odd":  # infinities, NaN of both signs, subnormals
        v = torch.tensor([float("inf"), float("-inf"), float("nan"), 1e-42, 2e-42, -1e-42, 0.5], device="cuda")[(w * 7).long()]
        return torch.where(torch.rand(*shape, generator=g, device="cuda") < 0.5, v, -v)
    return w


def run(cache, B, H, n, keep, first, last, d, kind="rand", lens=None, seed=0, pad=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = weights(kind, (B, H, n + pad), g)
    w_out = torch.full((B, H, keep + 2), -7.0, device="cuda")
    kept = torch.full((B, H, keep), 99, dtype=torch.int32, device="cuda")
    if cache == "q4":
        src, dst = sv.Q4Cache.empty(B, H, n + pad, d), sv.Q4Cache.empty(B, H, keep + 1, d)
        for t in (src.k, src.v, src.k_scale, src.v_scale, dst.k, dst.v, dst.k_scale, dst.v_scale):
            t.random_(0, 255, generator=g)
        args = dict(q4_src=src, q4_dst=dst)
        pairs = [(src.k, dst.k), (src.v, dst.v), (src.k_scale, dst.k_scale), (src.v_scale, dst.v_scale)]
    else:
        dt = torch.bfloat16 if cache == "bf16" else torch.float32
        s = [torch.randn(B, H, n + pad, d, generator=g, device="cuda").to(dt) for _ in range(2)]
        t = [torch.full((B, H, keep + 1, d), 3.0, device="cuda").to(dt) for _ in range(2)]
        args = dict(k_src=s[0], v_src=s[1], k_dst=t[0], v_dst=t[1])
        pairs = list(zip(s, t))
    before = [b.clone() for _, b in pairs]
    sv.sparvar_kv_evict(w, n, keep, first, last, kept, w_out,
                        kv_len=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"), **args)
    torch.cuda.synchronize()
    wn = w.cpu().numpy()
    for b in range(B):
        size = n if lens is None else min(max(lens[b], 0), n)
        for h in range(H):
            want = O.kept_tokens(wn[b, h, :size], keep, first, last)
            m = len(want)
            assert kept[b, h].tolist() == want + [-1] * (keep - m), (b, h)
            at = torch.tensor(want, dtype=torch.long, device="cuda")
            assert torch.equal(w_out[b, h, :m].view(torch.int32), w[b, h, at].view(torch.int32))
            assert (w_out[b, h, m:] == -7).all()
            for (s_, t_), old in zip(pairs, before):
                assert torch.equal(t_[b, h, :m], s_[b, h, at]) and torch.equal(t_[b, h, m:], old[b, h, m:])


@pytest.mark.parametrize("B,H,n,keep,first,last,d", [
    (1, 1, 1, 1, 0, 0, 64), (1, 1, 5, 1, 0, 0, 128), (1, 2, 5, 2, 1, 1, 64), (2, 3, 100, 64, 0, 0, 128), (1, 3, 100, 63, 10, 20, 64),
    (2, 1, 1023, 500, 0, 499, 128), (1, 2, 1024, 500, 500, 0, 64), (2, 2, 1025, 900, 121, 64, 128), (1, 2, 777, 777, 5, 5, 64),
    (1, 2, 300, 1000, 0, 0, 128), (1, 1, 8192, 4097, 4, 100, 64), (1, 2, 8193, 100, 0, 0, 128), (1, 1, 9000, 8999, 0, 0, 64),
    (1, 1, 49152, 20000, 121, 1000, 64), (1, 1, 49153, 20000, 0, 0, 64), (1, 1, 70001, 4096, 7, 9, 64), (1, 2, 140000, 70000, 100, 50, 64)])
@pytest.mark.parametrize("cache", ["bf16", "f32", "q4"])
def test_evict(cache, B, H, n, keep, first, last, d):
    note(f"[evict] {cache} B={B} H={H} n={n} keep={keep} first={first} last={last} d={d}")
    run(cache, B, H, n, keep, first, last, d, seed=n + keep)


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("n,keep,first,last", [(50, 20, 0, 0), (1500, 700, 30, 100), (20000, 9000, 0, 500), (66000, 33000, 121, 0)])
def test_weights_of_any_kind(kind, n, keep, first, last):
    note(f"[evict] {kind} n={n} keep={keep}")
    run("bf16", 1, 2, n, keep, first, last, 64, kind=kind, seed=n)


@pytest.mark.parametrize("kind", ["every high", "every low"])
@pytest.mark.parametrize("n,keep", [(20000, 9000), (20000, 100), (20000, 19900), (50001, 25000), (70000, 35000)])
def test_samples_that_mislead(kind, n, keep):
    note(f"[evict] {kind} n={n} keep={keep}")
    run("bf16", 1, 2, n, keep, 0, 0, 64, kind=kind, seed=n)


def test_streams():
    """Two calls side by side on streams of their own, of few tokens and of many, give what each gives alone."""
    note("[evict] two streams")
    jobs = []
    for n in (700, 30000):
        g = torch.Generator(device="cuda").manual_seed(n)
        w = torch.rand(2, 3, n, generator=g, device="cuda")
        x = torch.randn(2, 2, 3, n, 64, generator=g, device="cuda").bfloat16()
        m = n // 2
        outs = [[torch.zeros(2, 3, m, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, m, device="cuda"),
                 torch.zeros(2, 3, m, 64, device="cuda").bfloat16(), torch.zeros(2, 3, m, 64, device="cuda").bfloat16()]
                for _ in range(2)]
        jobs.append((w, n, m, x, torch.cuda.Stream(), *outs))
    for w, n, m, x, _, alone, _ in jobs:
        sv.sparvar_kv_evict(w, n, m, 4, 9, alone[0], alone[1], x[0], x[1], alone[2], alone[3])
    torch.cuda.synchronize()
    for _ in range(10):
        for w, n, m, x, stream, _, o in jobs:
            sv.sparvar_kv_evict(w, n, m, 4, 9, o[0], o[1], x[0], x[1], o[2], o[3], stream=stream)
    torch.cuda.synchronize()
    for *_, alone, o in jobs:
        assert all(torch.equal(a, b) for a, b in zip(alone, o))


@pytest.mark.parametrize("cache", ["bf16", "q4"])
@pytest.mark.parametrize("n,keep,first,last", [(400, 150, 10, 30), (12000, 5000, 121, 64), (60000, 100, 0, 0)])
def test_lengths(cache, n, keep, first, last):
    """Lengths of their own: none, one, around what is kept, past the end."""
    note(f"[evict] lengths {cache} n={n} keep={keep}")
    lens = [0, -5, 1, keep - 1, keep, keep + 1, n - 1, n, n + 50]
    run(cache, len(lens), 2, n, keep, first, last, 64, lens=lens, kind="spread", seed=6)


def test_many_planes():
    """More planes than compute units, and a prefix of a longer cache."""
    note("[evict] 300 planes")
    run("q4", 4, 75, 300, 150, 3, 10, 128, seed=1, pad=40)
