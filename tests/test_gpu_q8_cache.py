"""GPU parity of the append (norms, rotation), of the 8-bit cache as it is written and of its way back, through the C ABI,
against the fp64 oracle. Codes and scales are bit-exact; queries and 16- or 32-bit caches are within the rounding of the
32-bit norm and rotation."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import note
from paper_2602_04361_amd import sparvar as sv

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def codes_and_exps(q8):
    """Values of the codes over 2^e and the exponents, as fp64 and int arrays."""
    k = [O.codes_of_bytes(t.view(torch.uint8).cpu().numpy()) for t in (q8.k, q8.v)]
    e = [t.view(torch.uint8).cpu().numpy().astype(np.int64) - 127 for t in (q8.k_scale, q8.v_scale)]
    return k, e


def strided(B, H, n, d, dtype, pad, fill=7.0):
    """[B,H,n,d] inside planes of n + pad rows."""
    return torch.full((B, H, n + pad, d), fill, device="cuda").to(dtype)[:, :, :n]


def fresh(B, H, cap, d, G, pad=3):
    """A cache of sentinel bytes in padded planes: codes 0x2a, scales 0x55."""
    code = [torch.full((B, H, cap + pad, d), 0x2a, dtype=torch.uint8, device="cuda")[:, :, :cap] for _ in range(2)]
    nb = -(-cap // G)
    sc = [torch.full((B, H, nb + 2), 0x55, dtype=torch.uint8, device="cuda")[:, :, :nb] for _ in range(2)]
    return sv.Q8Cache(code[0], code[1], sc[0], sc[1], G)


@pytest.mark.parametrize("dtype,d,G,steps", [
    ("bf16", 128, 64, [1, 4, 16, 36, 64, 144]),  # the first scales of an image, one block over several
    ("bf16", 64, 16, [1, 1, 1, 13, 1, 17, 5]),   # single tokens
    ("f32", 128, 128, [130, 1, 125, 3]),
    ("f32", 64, 32, [31, 1, 1, 95]),
    ("bf16", 128, 16, [16, 16, 33]),
    ("f32", 64, 128, [200, 57]),
    ("f32", 128, 32, [7, 300]),
])
def test_appends_in_steps(dtype, d, G, steps):
    B, H, cap = 2, 3, sum(steps) + 5
    note(f"[q8] quantize {dtype} d={d} G={G} steps={steps}")
    r = np.random.default_rng(d + G)
    q8 = fresh(B, H, cap, d, G)
    want = [[(np.zeros((cap, d)), np.zeros(-(-cap // G), dtype=np.int64)) for _ in range(B * H)] for _ in range(2)]
    t0 = 0
    for i, n in enumerate(steps):
        src = []
        for w in range(2):  # later steps larger, so that blocks are encoded again
            x = r.standard_normal((B, H, n, d)) * 2.0 ** ((i * 5) % 7 - 2 * w)
            t = strided(B, H, n, d, TYPES[dtype], 2)
            t.copy_(torch.from_numpy(x.astype(np.float32)))
            src.append(t)
            xs = t.double().cpu().numpy().reshape(B * H, n, d)
            for p in range(B * H):
                O.append_codes(want[w][p][0], want[w][p][1], xs[p], t0, G)
        sv.sparvar_kv_quantize(src[0], src[1], t0, q8)
        t0 += n
        torch.cuda.synchronize()
        codes, exps = codes_and_exps(q8)
        nb = -(-t0 // G)
        for w in range(2):
            for p in range(B * H):
                b, h = divmod(p, H)
                assert np.array_equal(exps[w][b, h, :nb], want[w][p][1][:nb]), (i, w, p)
                assert np.array_equal(codes[w][b, h, :t0], want[w][p][0][:t0]), (i, w, p)
        # nothing past the tokens and their blocks, nothing between the planes
        for t in (q8.k, q8.v):
            full = t.as_strided((B, H, cap + 3, d), t.stride())
            assert (full[:, :, t0:] == 0x2a).all()
        for t in (q8.k_scale, q8.v_scale):
            full = t.as_strided((B, H, -(-cap // G) + 2), t.stride())
            assert (full[:, :, nb:] == 0x55).all()


def test_special_values():
    """Zeros, blocks at the ends of the exponent range, values on the border of an exponent, saturation, infinities, NaN."""
    G, d, n = 16, 64, 16 * 9
    x = np.zeros((n, d), dtype=np.float32)
    r = np.random.default_rng(3)
    x[16:32] = r.standard_normal((16, d)) * 1e-38        # below 2^-100: encoded at the smallest exponent
    x[32:48] = r.standard_normal((16, d)) * 2.0 ** 121   # beyond 448 * 2^112: saturates
    x[48, 0], x[64, 0], x[80, 1] = 448.0, np.nextafter(np.float32(448.0), np.float32(500)), -1.75 * 2.0 ** -20
    x[96:112] = r.standard_normal((16, d))
    x[97, 3], x[98, 5] = np.inf, -np.inf
    x[112:128] = r.standard_normal((16, d))
    x[113, 7] = np.nan
    x[128:144] = np.linspace(-2.0 ** -8, 2.0 ** -8, 16 * d).reshape(16, d) * 3
    x[130, 0] = 448.0                                    # the rest of its block lies among the subnormals
    note("[q8] special values")
    q8 = fresh(1, 1, n, d, G)
    t = torch.from_numpy(x).cuda()[None, None]
    sv.sparvar_kv_quantize(t, -t, 0, q8)
    torch.cuda.synchronize()
    codes, exps = codes_and_exps(q8)
    for w, y in enumerate((x, -x)):
        v, e = np.zeros((n, d)), np.zeros(n // G, dtype=np.int64)
        O.append_codes(v, e, y, 0, G)
        assert np.array_equal(exps[w][0, 0], e)
        assert np.array_equal(codes[w][0, 0], v, equal_nan=True)
    assert exps[0][0, 0].tolist() == [-100, -100, 112, 0, 1, -28, 112, O.block_exponent(np.abs(x[112:128][~np.isnan(x[112:128])]).max()), 0]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G,t0,n", [(128, 64, 0, 2521), (64, 16, 5, 1), (128, 128, 77, 300), (64, 32, 31, 66)])
def test_way_back_is_exact(dtype, d, G, t0, n):
    B, H, cap = 2, 2, t0 + n + 4
    note(f"[q8] dequantize {dtype} d={d} G={G} t0={t0} n={n}")
    g = torch.Generator(device="cuda").manual_seed(d + n)
    q8 = fresh(B, H, cap, d, G)
    for t in (q8.k, q8.v):  # every code but the NaNs
        b = torch.randint(0, 254, t.shape, generator=g, device="cuda")
        t.copy_((b + (b >= 127).int()).to(torch.uint8))
    for t in (q8.k_scale, q8.v_scale):
        t.copy_(torch.randint(127 - 100, 127 + 113, t.shape, generator=g, device="cuda").to(torch.uint8))
    dst = [strided(B, H, n, d, TYPES[dtype], 1) for _ in range(2)]
    sv.sparvar_kv_dequantize(q8, t0, dst[0], dst[1])
    torch.cuda.synchronize()
    codes, exps = codes_and_exps(q8)
    for w in range(2):
        for b in range(B):
            for h in range(H):
                want = O.cache_values(codes[w][b, h], exps[w][b, h], G)[t0:t0 + n]
                assert np.array_equal(dst[w][b, h].double().cpu().numpy(), want)
        assert (dst[w].as_strided((B, H, n + 1, d), dst[w].stride())[:, :, n:] == 7.0).all()


# y = x r w, then a rotation. In 32 bits with u = 2^-24: the sum of squares is off by at most (8 + 4 + 1) u (eight
# terms a lane, four exchanges, eps), its root by half that and a rounding, the quotient and the two products by one
# each: under 11 u on y; a rotation adds two products and a sum and takes both channels: 14 u (|y_a| + |y_b|).
U32, U16 = 2.0 ** -24, 2.0 ** -8


def map_bound(y, layout, turned):
    a = np.abs(y)
    if turned:
        d = y.shape[-1]
        z = np.empty_like(a)
        i, j = (np.arange(0, d, 2), np.arange(1, d, 2)) if layout == "pairs" else (np.arange(d // 2), np.arange(d // 2, d))
        z[:, i] = z[:, j] = a[:, i] + a[:, j]
        # the length of a pair stays, so the sum before the turn is at most sqrt(2) times the sum after
        a = 1.5 * z
    return 14 * U32 * a + 1e-30


def make_map(r, norm, layout, H, Hkv, d, rows, weights, turn):
    w = [torch.from_numpy((1 + 0.3 * r.standard_normal((h, d))).astype(np.float32)).cuda() if weights else None for h in (H, Hkv)]
    ang = r.uniform(-30, 30, (rows, d // 2))
    cs = torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32)).cuda() if turn else None
    eps = {"rms": 1e-6, "l2": 1e-12, None: 0.0}[norm]
    return sv.NormRope(norm, eps, w[0], w[1], cs, layout), w, cs, float(np.float32(eps))


CASES = [  # B, n, t0, H, Hkv, d, dtype, norm, layout, weights, turn, packed, G
    (2, 1, 0, 4, 4, 128, "bf16", "l2", "pairs", True, True, True, 64),
    (1, 37, 21, 6, 3, 128, "bf16", "rms", "halves", True, True, True, 64),
    (2, 100, 5, 4, 1, 64, "f32", "rms", "pairs", True, True, False, 32),
    (1, 65, 130, 3, 3, 64, "bf16", "l2", "halves", False, True, True, 16),
    (2, 33, 7, 5, 5, 128, "f32", None, "halves", False, True, True, 128),
    (1, 50, 64, 8, 2, 128, "bf16", "rms", "pairs", True, False, False, 16),
    (1, 20, 3, 2, 2, 64, "f32", None, "pairs", False, False, True, 128),
    (3, 129, 0, 2, 1, 128, "f32", "l2", "pairs", True, True, True, 128),
]


@pytest.mark.parametrize("to8", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_append(case, to8):
    B, n, t0, H, Hkv, d, dtype, norm, layout, weights, turn, packed, G = case
    note(f"[append] {case} to8={to8}")
    r = np.random.default_rng(n * 7 + d)
    tdt = TYPES[dtype]
    if packed:  # one fused projection
        x = torch.from_numpy((2 * r.standard_normal((B, n, H + 2 * Hkv, d))).astype(np.float32)).cuda().to(tdt)
        q, k, v = x.split([H, Hkv, Hkv], 2)
    else:       # tokens with padding between them
        q, k, v = (torch.from_numpy((2 * r.standard_normal((B, n, h + 2, d))).astype(np.float32)).cuda().to(tdt)[:, :, :h]
                   for h in (H, Hkv, Hkv))
    heads, w, cs, eps = make_map(r, norm, layout, H, Hkv, d, t0 + n + 3, weights, turn)
    if not (weights or turn or norm):
        heads = None
    qo = torch.full((B, H, n, d), 9.0, device="cuda").to(tdt)
    cap = t0 + n + 2
    xq, xk, xv = (t.double().cpu().numpy() for t in (q, k, v))
    ww = [None if t is None else t.cpu().numpy() for t in w]
    turnrows = None if cs is None else cs[t0:t0 + n].cpu().numpy()

    def mapped(x, b, h, weight):
        return O.norm_rope(x[b, :, h], norm, eps, None if weight is None else weight[h], turnrows, layout)

    half = U16 if dtype == "bf16" else U32
    if to8:
        q8 = fresh(B, Hkv, cap, d, G)
        held = [torch.from_numpy(r.standard_normal((B, Hkv, max(t0, 1), d)).astype(np.float32)).cuda() for _ in range(2)]
        if t0:
            sv.sparvar_kv_quantize(held[0], held[1], 0, q8)
        before = codes_and_exps(q8)
        sv.sparvar_qkv_append(q, k, v, t0, heads, qo, q8=q8)
    else:
        kc, vc = strided(B, Hkv, cap, d, tdt, 1), strided(B, Hkv, cap, d, tdt, 1)
        sv.sparvar_qkv_append(q, k, v, t0, heads, qo, kc, vc)
    torch.cuda.synchronize()
    got = qo.double().cpu().numpy()
    for b in range(B):
        for h in range(H):
            y = mapped(xq, b, h, ww[0])
            assert (np.abs(got[b, h] - y) <= half * np.abs(y) * 1.001 + map_bound(y, layout, turn)).all(), (b, h)
    if not to8:
        gk, gv = kc.double().cpu().numpy(), vc.double().cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                y = mapped(xk, b, h, ww[1])
                assert (np.abs(gk[b, h, t0:t0 + n] - y) <= half * np.abs(y) * 1.001 + map_bound(y, layout, turn)).all(), (b, h)
                assert np.array_equal(gv[b, h, t0:t0 + n], xv[b, :, h])
        for t in (kc, vc):
            full = t.as_strided((B, Hkv, cap + 1, d), t.stride())
            assert (full[:, :, :t0] == 7.0).all() and (full[:, :, t0 + n:] == 7.0).all()
        return
    codes, exps = codes_and_exps(q8)
    nb = -(-(t0 + n) // G)
    for b in range(B):
        for h in range(Hkv):
            v8, e8 = before[0][1][b, h].copy(), before[1][1][b, h].copy()
            O.append_codes(v8, e8, xv[b, :, h], t0, G)  # values are only encoded: exact
            assert np.array_equal(exps[1][b, h, :nb], e8[:nb]) and np.array_equal(codes[1][b, h, :t0 + n], v8[:t0 + n])
            # keys are mapped in 64 bits and rounded once
            k8, e8 = before[0][0][b, h].copy(), before[1][0][b, h].copy()
            O.append_codes(k8, e8, mapped(xk, b, h, ww[1]), t0, G)
            assert np.array_equal(exps[0][b, h, :nb], e8[:nb]) and np.array_equal(codes[0][b, h, :t0 + n], k8[:t0 + n])


@pytest.mark.parametrize("to8", [False, True])
def test_tokens_first(to8):
    """Projections of tokens first, [n, B, heads, d] seen as [B, n, heads, d]: the same bytes as batch first."""
    note(f"[append] tokens first, to8={to8}")
    B, n, H, Hkv, d, t0 = 3, 37, 4, 2, 128, 11
    x = torch.randn(n, B, H + 2 * Hkv, d, device="cuda").bfloat16()
    heads = sv.NormRope("rms", 1e-6, cos_sin=torch.randn(t0 + n, d // 2, 2, device="cuda"))
    got = []
    for y in (x.transpose(0, 1), x.transpose(0, 1).contiguous()):
        q, k, v = y.split([H, Hkv, Hkv], 2)
        qo = torch.full((B, H, n, d), 9.0, device="cuda").bfloat16()
        if to8:
            q8 = fresh(B, Hkv, t0 + n, d, 32)
            sv.sparvar_qkv_append(q, k, v, t0, heads, qo, q8=q8)
            got.append([qo] + [t.clone().view(torch.uint8) for t in (q8.k, q8.v, q8.k_scale, q8.v_scale)])
        else:
            kc, vc = (torch.full((B, Hkv, t0 + n, d), 9.0, device="cuda").bfloat16() for _ in range(2))
            sv.sparvar_qkv_append(q, k, v, t0, heads, qo, kc, vc)
            got.append([qo, kc, vc])
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_norm_of_zero_rows():
    """Rows of zeros: L2 divides by eps, RMS by its root; both give zeros, and a block of them the smallest exponent."""
    note("[append] zero rows")
    x = torch.zeros(1, 3, 6, 64, device="cuda")
    for norm, eps in (("l2", 1e-12), ("rms", 1e-6)):
        q8, qo = fresh(1, 2, 3, 64, 16), torch.full((1, 2, 3, 64), 9.0, device="cuda")
        q, k, v = x.split([2, 2, 2], 2)
        sv.sparvar_qkv_append(q, k, v, 0, sv.NormRope(norm, eps), qo, q8=q8)
        torch.cuda.synchronize()
        assert (qo == 0).all() and (q8.k == 0).all() and (q8.k_scale == 27).all()


@pytest.mark.parametrize("norm,eps", [("l2", 1e-12), ("rms", 1e-6), (None, 0.0)])
def test_a_nan_stays_in_its_row(norm, eps):
    """A NaN makes its row NaN under a norm, itself alone without one, and does not count for its block's exponent."""
    note(f"[append] NaN under {norm}")
    r = np.random.default_rng(5)
    x = r.standard_normal((1, 20, 3, 64)).astype(np.float32)
    x[0, 3, :, 17] = np.nan
    t = torch.from_numpy(x).cuda()
    q8, qo = fresh(1, 1, 20, 64, 16), torch.full((1, 1, 20, 64), 9.0, device="cuda")
    q, k, v = t.split([1, 1, 1], 2)
    sv.sparvar_qkv_append(q, k, v, 0, sv.NormRope(norm, eps), qo, q8=q8)
    torch.cuda.synchronize()
    codes, exps = codes_and_exps(q8)
    y = [O.norm_rope(x[0, :, 0], norm, float(np.float32(eps)), None, None, "pairs"),
         O.norm_rope(x[0, :, 1], norm, float(np.float32(eps)), None, None, "pairs"), x[0, :, 2].astype(np.float64)]
    got = qo[0, 0].double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(y[0]))
    assert np.isnan(got[3]).sum() == (1 if norm is None else 64)
    ok = ~np.isnan(y[0])
    assert (np.abs(got - y[0])[ok] <= (U32 * 1.001 * np.abs(y[0]) + map_bound(y[0], "pairs", False))[ok]).all()
    for w in range(2):
        c, e = np.zeros((20, 64)), np.zeros(2, dtype=np.int64)
        O.append_codes(c, e, y[w + 1], 0, 16)
        assert np.array_equal(exps[w][0, 0], e) and np.array_equal(codes[w][0, 0], c, equal_nan=True)


def test_planes_far_apart():
    """Planes of codes more than 2^32 bytes apart."""
    note("[q8] planes 5 GB apart")
    d, G, n, cap = 64, 16, 20, 40
    gap = 5 << 30
    big = torch.empty(2 * gap + 2 * cap * d, dtype=torch.uint8, device="cuda")
    code = [big[o:].as_strided((1, 3, cap, d), (3 * gap, gap, d, 1)) for o in (0, cap * d)]
    sc = [torch.zeros(1, 3, 3, dtype=torch.uint8, device="cuda") for _ in range(2)]
    far = sv.Q8Cache(code[0], code[1], sc[0], sc[1], G)
    near = fresh(1, 3, cap, d, G)
    x = torch.randn(2, 1, 3, n, d, device="cuda")
    for c in (far, near):
        sv.sparvar_kv_quantize(x[0], x[1], 3, c)
        sv.sparvar_kv_quantize(x[1], x[0], 3 + n - 5, c)
    out = [torch.empty(1, 3, 30, d, device="cuda") for _ in range(4)]
    sv.sparvar_kv_dequantize(far, 3, out[0], out[1])
    sv.sparvar_kv_dequantize(near, 3, out[2], out[3])
    q = torch.randn(1, 3, 7, d, device="cuda").bfloat16()
    o = [torch.empty_like(q) for _ in range(2)]
    for c, y in zip((far, near), o):
        c.k[:, :, :3] = 0x30
        c.v[:, :, :3] = 0x30
        sv.sparvar_dense_attn_q8_fwd(q, c, 33, y)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]) and torch.equal(o[0], o[1])
    assert torch.isfinite(o[0].float()).all() and (o[0] != 0).any()
    del big
    torch.cuda.empty_cache()
