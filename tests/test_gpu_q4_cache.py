"""GPU parity of rows to a 4-bit cache and back, through the C ABI: codes and scale bytes bit-exact against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv

pytestmark = pytest.mark.gpu


def rows(B, H, n, d, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, B, H, n + pad, d, generator=g, device="cuda")
    x *= 2.0 ** torch.randint(-30, 30, (2, B, H, n + pad, d // 32), generator=g, device="cuda").float().repeat_interleave(32, -1)
    # ties, borders of the exponent, zeros and subnormals of 32 bits
    special = torch.tensor([0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -7.0, 6.9999995, 7.0000005, 1e-42, -0.25, -5.0], device="cuda")
    flat = x.view(-1)
    at = torch.randint(0, flat.numel(), (flat.numel() // 8,), generator=g, device="cuda")
    flat[at] = special[torch.randint(0, len(special), at.shape, generator=g, device="cuda")]
    x[:, :, :, 0, :32] = 0.0
    x[:, :, :, n - 1, 32:64] = special.repeat(2)
    return x.to(dtype)[:, :, :, :n]


def check(q4, t0, x):
    for c, s, rows_ in ((q4.k, q4.k_scale, x[0]), (q4.v, q4.v_scale, x[1])):
        n = rows_.shape[2]
        c, s, r = c.cpu().numpy()[:, :, t0:t0 + n], s.cpu().numpy()[:, :, t0:t0 + n], rows_.double().cpu().numpy()
        for b in range(r.shape[0]):
            for h in range(r.shape[1]):
                code, scale = O.encode_rows(r[b, h])
                assert np.array_equal(s[b, h], scale), (b, h)
                assert np.array_equal(O.decode_rows(c[b, h], s[b, h]), O.decode_rows(code, scale)), (b, h)


@pytest.mark.parametrize("B,H,n,t0,cap,d", [(1, 1, 1, 0, 1, 64), (1, 1, 1, 6, 9, 128), (2, 3, 17, 5, 40, 64), (1, 2, 33, 0, 33, 128),
                                            (2, 1, 129, 64, 200, 128), (1, 3, 300, 7, 311, 64), (3, 2, 65, 63, 128, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_and_back(B, H, n, t0, cap, d, dtype):
    note(f"[q4 cache] B={B} H={H} n={n} t0={t0} cap={cap} d={d} {dtype}")
    x = rows(B, H, n, d, dtype, n + t0, pad=3)
    q4 = sv.Q4Cache.empty(B, H, cap, d)
    before = []
    for t in (q4.k, q4.v, q4.k_scale, q4.v_scale):
        t.random_(0, 250)
        before.append(t.clone())
    sv.sparvar_kv_quantize_q4(x[0], x[1], t0, q4)
    out = {}
    for dt in (torch.bfloat16, torch.float32):
        out[dt] = [torch.full((B, H, n + 2, d), 5.0, device="cuda").to(dt) for _ in range(2)]
        sv.sparvar_kv_dequantize_q4(q4, t0, *(t[:, :, 1:n + 1] for t in out[dt]))
    torch.cuda.synchronize()
    check(q4, t0, x)
    for t, old in zip((q4.k, q4.v, q4.k_scale, q4.v_scale), before):  # other tokens are as they were
        assert torch.equal(t[:, :, :t0], old[:, :, :t0]) and torch.equal(t[:, :, t0 + n:], old[:, :, t0 + n:])
    for i, (c, s) in enumerate(((q4.k, q4.k_scale), (q4.v, q4.v_scale))):
        want = O.decode_rows(c.cpu().numpy(), s.cpu().numpy())[:, :, t0:t0 + n]
        for dt, o in out.items():
            assert np.array_equal(o[i][:, :, 1:n + 1].double().cpu().numpy(), want), dt
            assert (o[i][:, :, 0] == 5).all() and (o[i][:, :, n + 1] == 5).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_extremes(dtype):
    """Infinities and the largest values saturate, the smallest vanish, a NaN takes its group with it and no other."""
    note(f"[q4 cache] extremes {dtype}")
    x = torch.ones(2, 1, 1, 4, 64, device="cuda")
    x[:, ..., 0, 3], x[:, ..., 0, 40] = float("nan"), float("-inf")
    x[:, ..., 1, :32], x[:, ..., 1, 32:] = 3e38, 2.0 ** -104
    x[:, ..., 2, 0], x[:, ..., 2, 32] = 2.0 ** 114 * 1.75, -(2.0 ** -98) * 1.75
    x = x.to(dtype)
    q4 = sv.Q4Cache.empty(1, 1, 4, 64)
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, q4)
    for dt in (torch.bfloat16, torch.float32):
        o = [torch.empty(1, 1, 4, 64, device="cuda").to(dt) for _ in range(2)]
        sv.sparvar_kv_dequantize_q4(q4, 0, o[0], o[1])
        torch.cuda.synchronize()
        want = O.decode_rows(*O.encode_rows(x[0, 0, 0].double().cpu().numpy()))
        for t in o:
            got = t[0, 0].double().cpu().numpy()
            assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(want[0, :32]).all() and want[0, 40] == -6 * 2.0 ** 112 and (want[1, :32] == 6 * 2.0 ** 112).all()
    assert q4.k_scale[0, 0, 0].tolist() == [255, 239] and (want[1, 32:] == 0).all()


def test_rows_again_and_out_of_order():
    """Tokens written in any order, one by one or together, are the same; their values written again are themselves."""
    note("[q4 cache] order")
    x = rows(1, 2, 50, 128, torch.bfloat16, 4)
    a, b = sv.Q4Cache.empty(1, 2, 50, 128), sv.Q4Cache.empty(1, 2, 50, 128)
    sv.sparvar_kv_quantize_q4(x[0], x[1], 0, a)
    for t in np.random.default_rng(1).permutation(50).tolist():
        sv.sparvar_kv_quantize_q4(x[0][:, :, t:t + 1].contiguous(), x[1][:, :, t:t + 1].contiguous(), t, b)
    o = [torch.empty(1, 2, 50, 128, device="cuda") for _ in range(2)]
    sv.sparvar_kv_dequantize_q4(b, 0, o[0], o[1])
    sv.sparvar_kv_quantize_q4(o[0], o[1], 0, b)
    torch.cuda.synchronize()
    # (a group's largest is above 3.5 units, so its code is 4 or 6, which no smaller exponent holds)
    for s, t in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)):
        assert torch.equal(s, t)
