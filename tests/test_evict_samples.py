"""Eviction where the sample that bounds the threshold is like none of the weights: outliers stand at the very tokens that the
kernel samples, 128 of those that compete at even steps, so that the threshold lies outside the bounds and the search goes over
all weights again, in each of the kernels by the number of tokens."""
import numpy as np
import pytest

from gpu_helpers import note

SAMPLE = 128


def sampled(lo, many):
    return lo + np.arange(SAMPLE) * many // SAMPLE


def bounds(w, lo, many, need):
    """The two weights between which the kernel looks first (None: no bound), by its rule in 32 bits: a sample's place is
    three and a half standard deviations and 1.5 from where need of many would be."""
    s = np.sort(w[sampled(lo, many)])[::-1]
    f = np.float32
    share = f(need) / f(many)
    at = share * f(SAMPLE)
    wide = f(1.5) + f(3.5) * np.sqrt(at * (f(1) - share))
    upper = s[int(at - wide)] if at >= wide else None
    lower = s[int(at + wide)] if int(at + wide) < SAMPLE else None
    return lower, upper


def planted(kind, shape, lo, many, rng):
    w = rng.random(shape).astype(np.float32)
    w[..., sampled(lo, many)] += 9 if kind == "high" else -9
    return w


def misled(w, lo, many, need):
    threshold = np.sort(w[lo:lo + many])[::-1][need - 1]
    lower, upper = bounds(w, lo, many, need)
    return (lower is not None and threshold < lower) or (upper is not None and threshold > upper)


# tokens, kept, first, last: one for the kernels of up to 8192, 24576 and 49152 tokens and the one of more
CASES = [(8000, 4000, 0, 0), (8190, 3000, 7, 20), (20000, 9000, 0, 0), (24570, 12000, 121, 300), (45056, 20000, 0, 0),
         (49150, 25001, 3, 4096), (70000, 35000, 0, 0), (50001, 25000, 11, 13)]


@pytest.mark.parametrize("kind", ["high", "low"])
@pytest.mark.parametrize("n,keep,first,last", CASES)
def test_the_sample_misleads(kind, n, keep, first, last):
    many, need = n - first - last, keep - first - last
    for seed in range(5):
        assert misled(planted(kind, (n,), first, many, np.random.default_rng(seed)), first, many, need)
    # and does not where nothing is planted
    assert not misled(np.random.default_rng(9).random(n).astype(np.float32), first, many, need)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["high", "low"])
@pytest.mark.parametrize("n,keep,first,last", CASES)
def test_misleading_sample(kind, n, keep, first, last, monkeypatch):
    import torch

    import test_gpu_evict as E

    note(f"[evict] misled {kind} n={n} keep={keep} first={first} last={last}")
    many, need = n - first - last, keep - first - last

    def weights(_, shape, g):
        w = planted(kind, shape, first, many, np.random.default_rng(n))
        assert all(misled(x, first, many, need) for x in w.reshape(-1, shape[-1])[:, :n])
        return torch.from_numpy(w).cuda()

    monkeypatch.setattr(E, "weights", weights)
    E.run("bf16", 1, 2, n, keep, first, last, 64, seed=n)
