"""Timed cases of the operators around an 8-bit key/value cache, over the range that a VAR inference calls them in.

append      norms of queries and keys for each head and the position rotation, written to a cache (16 bits or 8)
quantize    rows of a cache written in 8 bits, with a power-of-two scale for each block of tokens and head
dequantize  such rows read back
dense       attention of a set of queries over the first tokens of the 8-bit cache
sparse      attention of a scale's query tiles over listed blocks of the 8-bit cache

listed() names the cases, draw(rng) gives more of the same ranges, prepare(case, seed) makes what a program has in hand
before the call, run(state) is one pass, by elementary torch operations or (own) by the library's calls, work(case) the
bytes and operations that it cannot do without, exact(case, seed) the same results in 64 bits.

Codes are e4m3, scales the exponents 2^e of the E8M0 format: e is the smallest integer with max |x| <= 448 * 2^e.
"""
import math

import numpy as np
import torch

own = False

S1024 = "1,2,4,6,8,12,16,20,24,32,40,48,64"  # the 13 scales of a 1024x1024 image
S2048 = S1024 + ",80,96,128"                 # and of a 2048x2048 one
DEV = "cuda"
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
E_MIN, E_MAX = -100, 112


def listed():
    inf = dict(sides=S1024, aspect=1.0, B=2, H=16, Hkv=16, d=128)
    return [
        # the first step of an image: one token a sequence, bound by latency
        dict(inf, name="append_1x1", kind="append", k=1, dtype="bf16", q8=False, norm="l2", layout="pairs", G=64),
        # the last step into a 16-bit cache: 4096 tokens
        dict(inf, name="append_64x64", kind="append", k=13, dtype="bf16", q8=False, norm="l2", layout="pairs", G=64),
        # the same step written in 8 bits as it comes, after 6425 earlier tokens
        dict(inf, name="append_64x64_q8", kind="append", k=13, dtype="bf16", q8=True, norm="l2", layout="pairs", G=64),
        # one early scale of an image, from 32 bits, the narrow head: 36 tokens after 21
        dict(sides=S1024, aspect=1.0, B=2, H=12, Hkv=12, d=64, name="quantize_6x6_f32", kind="quantize", k=4, whole=False,
             dtype="f32", G=32),
        # a whole cache of a 1024x1024 image put into 8 bits
        dict(inf, name="quantize_10521", kind="quantize", k=13, whole=True, dtype="bf16", G=64),
        # the first scales read back to 32 bits, an odd length
        dict(sides=S1024, aspect=1.0, B=2, H=12, Hkv=12, d=64, name="dequantize_521_f32", kind="dequantize", k=7, whole=True,
             dtype="f32", G=32),
        # what a decision step at 32x32 needs in 16 bits: the 2521 tokens up to it
        dict(inf, name="dequantize_2521", kind="dequantize", k=10, whole=True, dtype="bf16", G=64),
        # an early scale, dense: 64 queries, 121 keys
        dict(inf, name="dense_8x8", kind="dense", nq=64, nkv=121, lens=False, lse=False, G=64),
        # one token a sequence against the longest cache, four query heads a key head, lengths of their own
        dict(sides=S2048, aspect=1.0, B=4, H=32, Hkv=8, d=128, name="dense_token_42521", kind="dense", nq=1, nkv=42521,
             lens=True, lse=True, G=64),
        # the last scale in a layer that is kept dense
        dict(inf, name="dense_64x64", kind="dense", nq=4096, nkv=10521, lens=False, lse=True, G=64),
        # a portrait image, the narrow head: tiles cut at the edges
        dict(sides=S1024, aspect=0.75, B=2, H=12, Hkv=12, d=64, name="sparse_portrait_48x36", kind="sparse", k=12, block=8,
             topk=8, G=32),
        # the last sparse step of a 1024x1024 image
        dict(inf, name="sparse_64x64", kind="sparse", k=13, block=8, topk=14, G=64),
    ]


def draw(rng):
    """One more case: any kind, odd sides and ratios, head counts and widths, blocks of 16 to 128 tokens."""
    kind = rng.choice(["append", "append", "quantize", "dequantize", "dense", "dense", "dense", "sparse", "sparse"])
    sides = [int(s) for s in S1024.split(",")]
    for i in range(4, len(sides)):
        if rng.random() < 0.4:
            sides[i] += rng.choice([-1, 1])
    Hkv = rng.choice([4, 6, 8, 12, 16])
    c = dict(sides=",".join(str(s) for s in sides), aspect=rng.choice([1.0, 1.0, 0.75, 0.5625]), B=rng.choice([1, 2]), H=Hkv, Hkv=Hkv,
             d=rng.choice([64, 128, 128]), kind=kind, G=rng.choice([16, 32, 64, 64, 128]))
    if kind == "append":
        c.update(k=rng.randint(1, 13), dtype=rng.choice(["bf16", "bf16", "f32"]), q8=rng.random() < 0.6,
                 norm=rng.choice(["l2", "rms", "rms"]), layout=rng.choice(["pairs", "halves"]))
        if rng.random() < 0.4 and Hkv <= 8:
            c["H"] = 2 * Hkv
    elif kind in ("quantize", "dequantize"):
        c.update(k=rng.randint(2, 13), whole=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]))
    elif kind == "dense":
        few = rng.random() < 0.5  # few rows against a long cache, or a scale against the cache up to it
        nkv = int(math.exp(rng.uniform(math.log(32), math.log(20000 if few else 10000))))
        nq = rng.randint(1, 16) if few else max(1, int(nkv * rng.uniform(0.2, 0.4)))
        c.update(nq=nq, nkv=nkv, lens=rng.random() < 0.4, lse=rng.random() < 0.5)
        if few and Hkv <= 8:
            c["H"] = Hkv * rng.choice([1, 2, 4, 8])
    else:
        c.update(k=rng.randint(10, 13), block=rng.choice([8, 8, 8, 16]), topk=rng.randint(4, 20))
    return c


# ------------------------------------------------------------------------------------------------ geometry of a case
class Grid:
    """The scales of a schedule (1-based), their b x b tiles and the ids of those."""

    def __init__(self, c, block=8):
        self.h = [int(s) for s in c["sides"].split(",")]
        self.w = [max(1, int(s * c["aspect"] + 0.5)) for s in self.h]
        self.n = [a * b for a, b in zip(self.h, self.w)]
        self.C = np.concatenate([[0], np.cumsum(self.n)]).tolist()
        self.eh, self.ew = [min(block, x) for x in self.h], [min(block, x) for x in self.w]
        self.th = [-(-x // e) for x, e in zip(self.h, self.eh)]
        self.tw = [-(-x // e) for x, e in zip(self.w, self.ew)]
        self.NB = np.concatenate([[0], np.cumsum([a * b for a, b in zip(self.th, self.tw)])]).tolist()

    def tile_of_token(self, l):
        x, y = np.divmod(np.arange(self.n[l - 1]), self.w[l - 1])
        return (x // self.eh[l - 1]) * self.tw[l - 1] + y // self.ew[l - 1]

    def block_of_key(self, k):
        return np.concatenate([self.NB[l - 1] + self.tile_of_token(l) for l in range(1, k + 1)])


def rotation_table(grid, d):
    """cos and sin of every cache token's angles [tokens, d / 2, 2]: the first half of the pairs turns with the row, the
    second with the column, both in units of the largest scale's grid."""
    pos = []
    for h, w in zip(grid.h, grid.w):
        x, y = np.divmod(np.arange(h * w), w)
        pos.append(np.stack([(x + 0.5) * grid.h[-1] / h, (y + 0.5) * grid.w[-1] / w], 1))
    pos = np.concatenate(pos)
    freq = 10000.0 ** (-np.arange(d // 4) / (d // 4))
    ang = np.concatenate([pos[:, :1] * freq, pos[:, 1:] * freq], 1)
    return torch.from_numpy(np.stack([np.cos(ang), np.sin(ang)], 2).astype(np.float32)).to(DEV)


def rows_of(c, g, grid):
    """Listed blocks of every query tile of scale k: the sinks (scales 1-4), the tile and its neighbours, and topk drawn ones."""
    k, planes = c["k"], c["B"] * c["H"]
    th, tw, nb, first = grid.th[k - 1], grid.tw[k - 1], grid.NB[k], grid.NB[k - 1]
    keep = torch.zeros(planes, th * tw, nb, dtype=torch.bool)
    keep[:, :, :grid.NB[4]] = True
    a, b = np.divmod(np.arange(th * tw), tw)
    near = (abs(a[:, None] - a[None]) <= 1) & (abs(b[:, None] - b[None]) <= 1)
    keep[:, :, first:] |= torch.from_numpy(near)
    pick = torch.rand(planes, th * tw, nb, generator=g).topk(min(c["topk"], nb), dim=2).indices
    keep.scatter_(2, pick, True)
    n = keep.sum(2)
    stride = int(n.max())
    ids = torch.where(keep, torch.arange(nb), nb).sort(2).values[:, :, :stride]
    ids = torch.where(ids < nb, ids, -1).to(torch.int32)
    return keep.to(DEV), ids.reshape(-1).to(DEV), (torch.arange(planes * th * tw + 1) * stride).to(torch.int32).to(DEV)


# ------------------------------------------------------------------------------------------------ the 8-bit cache
def powers(e):
    return torch.exp2(e.float())


def encode(x, G):
    """x [B, H, n, d] in 32 bits: its codes and the exponents of its blocks of G tokens."""
    B, H, n, d = x.shape
    nb = -(-n // G)
    padded = torch.nn.functional.pad(x, (0, 0, 0, nb * G - n)).reshape(B, H, nb, G * d)
    m, ex = torch.frexp(padded.abs().amax(3))
    e = (ex - 9 + (m > 0.875)).clamp(E_MIN, E_MAX)
    y = (padded * powers(-e)[..., None]).clamp(-448.0, 448.0)
    return y.reshape(B, H, nb * G, d)[:, :, :n].to(F8), (e + 127).to(torch.uint8)


def decode(code, scale, G):
    """The values that codes [B, H, n, d] and exponent bytes [B, H, blocks] stand for, in 32 bits."""
    f = powers(scale.int() - 127).repeat_interleave(G, dim=2)[:, :, :code.shape[2], None]
    return code.float() * f


def write8(s, which, x):
    """Rows [t0, t0 + n) of the cache: the block that t0 lies in is encoded again with the values it holds."""
    G, t0, code, scale = s["G"], s["t0"], s[which + "8"], s[which + "s"]
    j0, end = t0 // G, t0 + x.shape[2]
    j1 = -(-end // G)
    old = decode(code[:, :, j0 * G:t0], scale[:, :, j0:j0 + 1], G)
    cc, ss = encode(torch.cat([old, x.float()], 2), G)
    code[:, :, j0 * G:end] = cc
    scale[:, :, j0:j1] = ss


# ------------------------------------------------------------------------------------------------ inputs
def gen(seed, case, dev=DEV):
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 1000003 + sum(ord(x) for x in case["kind"]))
    return g


def cache8(s, c, n, g):
    """An 8-bit cache of n tokens, as a program holds it: unit normals, keys of the first tokens larger."""
    B, H, d, G = c["B"], c["Hkv"], c["d"], c["G"]
    for which in "kv":
        x = torch.randn(B, H, n, d, generator=g, device=DEV)
        if which == "k":
            x[:, :, :57] += 3.0 * d ** -0.5
        s[which + "8"], s[which + "s"] = encode(x.bfloat16().float(), G)


def tokens_of(c, grid):
    """First token and count of a case's rows: a scale's own, or (whole) everything up to it."""
    t0 = 0 if c.get("whole") else grid.C[c["k"] - 1]
    return t0, grid.C[c["k"]] - t0


def prepare(case, seed):
    c, g = case, gen(seed, case)
    kind, B, H, Hkv, d, G = c["kind"], c["B"], c["H"], c["Hkv"], c["d"], c["G"]
    dt = torch.float32 if c.get("dtype") == "f32" else torch.bfloat16
    s = dict(kind=kind, G=G, d=d, case=dict(c))
    grid = Grid(c, c.get("block", 8))
    if kind == "append":
        s["t0"], n = tokens_of(c, grid)
        x = torch.randn(B, n, H + 2 * Hkv, d, generator=g, device=DEV) * 1.7
        s["qkv"] = x.to(dt)
        s["q"], s["k"], s["v"] = s["qkv"].split([H, Hkv, Hkv], 2)
        s["eps"] = 1e-12 if c["norm"] == "l2" else 1e-6
        if c["norm"] == "l2":  # a learned factor for each head, keys plain
            s["qw"] = (2.0 + torch.rand(H, 1, generator=g, device=DEV)).expand(H, d).contiguous()
            s["kw"] = torch.ones(Hkv, d, device=DEV)
        else:
            s["qw"] = 1.0 + 0.1 * torch.randn(H, d, generator=g, device=DEV)
            s["kw"] = 1.0 + 0.1 * torch.randn(Hkv, d, generator=g, device=DEV)
        s["table"] = rotation_table(grid, d)
        s["qo"] = torch.zeros(B, H, n, d, dtype=dt, device=DEV)
        if c["q8"]:
            cache8(s, c, grid.C[c["k"]], g)
        else:
            s["kc"], s["vc"] = (torch.zeros(B, Hkv, grid.C[c["k"]], d, dtype=dt, device=DEV) for _ in range(2))
    elif kind == "quantize":
        s["t0"], n = tokens_of(c, grid)
        s["k"], s["v"] = (torch.randn(B, Hkv, n, d, generator=g, device=DEV).to(dt) for _ in range(2))
        cache8(s, c, grid.C[c["k"]], g)
    elif kind == "dequantize":
        s["t0"], n = tokens_of(c, grid)
        cache8(s, c, grid.C[c["k"]], g)
        s["ko"], s["vo"] = (torch.zeros(B, Hkv, n, d, dtype=dt, device=DEV) for _ in range(2))
    elif kind == "dense":
        s["q"] = torch.randn(B, H, c["nq"], d, generator=g, device=DEV).bfloat16()
        cache8(s, c, c["nkv"], g)
        s["lens"] = None
        if c["lens"]:
            s["lens"] = torch.randint(max(1, c["nkv"] // 2), c["nkv"] + 1, (B,), generator=g, device=DEV).to(torch.int32)
            s["lens"][0] = c["nkv"]
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, H, c["nq"], device=DEV) if c["lse"] else None
    else:
        k = c["k"]
        s["q"] = torch.randn(B, H, grid.n[k - 1], d, generator=g, device=DEV).bfloat16()
        cache8(s, c, grid.C[k], g)
        s["keep"], s["ids"], s["ptr"] = rows_of(c, gen(seed, c, "cpu"), grid)
        s["qt"] = torch.from_numpy(grid.tile_of_token(k)).to(DEV)
        s["kb"] = torch.from_numpy(grid.block_of_key(k)).to(DEV)
        s["o"] = torch.zeros_like(s["q"])
        s["k"] = k
    if own:
        from paper_2602_04361_amd import sparvar as sv

        if "k8" in s:
            s["q8"] = sv.Q8Cache(s["k8"], s["v8"], s["ks"], s["vs"], G)
        if kind == "append":
            s["heads"] = sv.NormRope(norm=c["norm"], eps=s["eps"], q_weight=s["qw"], k_weight=s["kw"], cos_sin=s["table"],
                                     layout=c["layout"])
        elif kind == "dense":
            size = sv.sparvar_dense_attn_q8_workspace(B, H, Hkv, c["nq"], c["nkv"], d)
            s["ws"] = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
        elif kind == "sparse":
            s["geom"] = sv.Geometry(grid.h, grid.w, c["block"], 4)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def rotate(y, table, layout):
    cos, sin = table[:, None, :, 0], table[:, None, :, 1]
    if layout == "pairs":
        a, b = y[..., 0::2], y[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    a, b = y.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def norm_rotate(x, w, s):
    x, c = x.float(), s["case"]
    ss = x.square().sum(-1, keepdim=True)
    r = 1.0 / ss.sqrt().clamp_min(s["eps"]) if c["norm"] == "l2" else 1.0 / (ss / s["d"] + s["eps"]).sqrt()
    t0 = s["t0"]
    return rotate(x * r * w, s["table"][t0:t0 + x.shape[1]], c["layout"]).transpose(1, 2)


def state8(s):
    return [s["k8"], s["v8"], s["ks"].view(E8), s["vs"].view(E8)]


def run(state):
    return own_pass(state) if own else plain_pass(state)


def own_pass(s):
    from paper_2602_04361_amd import sparvar as sv

    kind = s["kind"]
    if kind == "append":
        if "q8" in s:
            sv.sparvar_qkv_append(s["q"], s["k"], s["v"], s["t0"], s["heads"], s["qo"], q8=s["q8"])
            return [s["qo"]] + state8(s)
        sv.sparvar_qkv_append(s["q"], s["k"], s["v"], s["t0"], s["heads"], s["qo"], s["kc"], s["vc"])
        return [s["qo"], s["kc"], s["vc"]]
    if kind == "quantize":
        sv.sparvar_kv_quantize(s["k"], s["v"], s["t0"], s["q8"])
        return state8(s)
    if kind == "dequantize":
        sv.sparvar_kv_dequantize(s["q8"], s["t0"], s["ko"], s["vo"])
        return [s["ko"], s["vo"]]
    if kind == "dense":
        sv.sparvar_dense_attn_q8_fwd(s["q"], s["q8"], s["case"]["nkv"], s["o"], lse=s["lse"], kv_len=s["lens"],
                                     workspace=s["ws"])
        return [s["o"], s["lse"]] if s["lse"] is not None else [s["o"]]
    sv.sparvar_block_sparse_attn_q8_fwd(s["geom"], s["k"], s["q"], s["q8"], s["o"], s["ptr"], s["ids"])
    return [s["o"]]


def plain_pass(s):
    kind, G, d, t0 = s["kind"], s["G"], s["d"], s.get("t0")
    if kind == "append":
        n = s["q"].shape[1]
        s["qo"].copy_(norm_rotate(s["q"], s["qw"], s))
        k, v = norm_rotate(s["k"], s["kw"], s), s["v"].transpose(1, 2)
        if s["case"]["q8"]:
            write8(s, "k", k)
            write8(s, "v", v)
            return [s["qo"]] + state8(s)
        s["kc"][:, :, t0:t0 + n] = k
        s["vc"][:, :, t0:t0 + n] = v
        return [s["qo"], s["kc"], s["vc"]]
    if kind == "quantize":
        write8(s, "k", s["k"])
        write8(s, "v", s["v"])
        return state8(s)
    if kind == "dequantize":
        n = s["ko"].shape[2]
        s["ko"].copy_(decode(s["k8"], s["ks"], G)[:, :, t0:t0 + n])
        s["vo"].copy_(decode(s["v8"], s["vs"], G)[:, :, t0:t0 + n])
        return [s["ko"], s["vo"]]
    k, v = decode(s["k8"], s["ks"], G), decode(s["v8"], s["vs"], G)
    B, H, nq, _ = s["q"].shape
    rep = H // k.shape[1]
    q = s["q"].float().reshape(B, k.shape[1], rep * nq, d)
    p = torch.matmul(q, k.transpose(2, 3)) * d ** -0.5
    if kind == "dense":
        if s["lens"] is not None:
            p.masked_fill_(torch.arange(k.shape[2], device=DEV) >= s["lens"][:, None, None, None], -math.inf)
    else:
        keep = s["keep"].reshape(B, H, -1, s["keep"].shape[2])
        p.masked_fill_(~keep[:, :, s["qt"]][..., s["kb"]], -math.inf)
    m = p.amax(3, keepdim=True)
    p.sub_(m).exp_()
    total = p.sum(3, keepdim=True)
    o = (torch.matmul(p, v) / total).reshape(B, H, nq, d).to(torch.bfloat16)
    if s.get("lse") is not None:
        return [o, (m + total.log()).reshape(B, H, nq)]
    return [o]


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    c = case
    grid = Grid(c, c.get("block", 8))
    kind, B, H, Hkv, d, G = c["kind"], c["B"], c["H"], c["Hkv"], c["d"], c["G"]
    e = 4 if c.get("dtype") == "f32" else 2
    if kind in ("append", "quantize", "dequantize"):
        t0, n = tokens_of(c, grid)
        blocks = -(-(t0 + n) // G) - t0 // G
        if kind == "append":
            cache = 2 * B * Hkv * (n * d + blocks) if c["q8"] else 2 * B * Hkv * n * d * e
            return {"bytes": B * n * (2 * H + 2 * Hkv) * d * e + n * d * 4 + (H + Hkv) * d * 4 + cache,
                    "flops": 10 * B * n * (H + Hkv) * d}
        return {"bytes": 2 * B * Hkv * (n * d * (e + 1) + blocks), "flops": 4 * B * Hkv * n * d}
    if kind == "dense":
        nq, nkv = c["nq"], c["nkv"]
        # lengths of their own: one entry of the batch is whole, the others three quarters on average
        mean = nkv * (1 + 0.75 * (B - 1)) / B if c["lens"] else nkv
        return {"bytes": B * H * nq * (4 * d + (4 if c["lse"] else 0)) + 2 * B * Hkv * mean * (d + 1.0 / G),
                "flops": 4.0 * B * H * nq * mean * d}
    k = c["k"]
    keep, ids, _ = rows_of(c, gen(1, c, "cpu"), grid)
    size = torch.from_numpy(np.bincount(grid.block_of_key(k), minlength=grid.NB[k])).to(keep.device)
    tile = torch.from_numpy(np.bincount(grid.tile_of_token(k))).to(keep.device)
    pairs = int(((keep * size).sum(2) * tile).sum())
    return {"bytes": B * H * grid.n[k - 1] * 4 * d + 2 * B * Hkv * grid.C[k] * (d + 1.0 / G) + ids.numel() * 4,
            "flops": 4.0 * pairs * d}


# ------------------------------------------------------------------------------------------------ in 64 bits
def e4m3(y):
    """Nearest e4m3 value, ties to the even code, of y in 64 bits with |y| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))).clamp_min(-6.0) - 3.0)
    return torch.round(y / step) * step


def encode64(rows, G, at):
    """Codes and scales (as values) of rows [.., n, d] that start inside a block at offset `at` of it, in 64 bits."""
    codes, scales = [], []
    for a, b in zip([0] + list(range(G - at, rows.shape[2], G)), list(range(G - at, rows.shape[2], G)) + [rows.shape[2]]):
        x = rows[:, :, a:b]
        top = x.abs().amax((2, 3), keepdim=True)
        e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0)).clamp(E_MIN, E_MAX)
        codes.append(e4m3((x / torch.exp2(e)).clamp(-448.0, 448.0)))
        scales.append(torch.exp2(e)[:, :, :, 0])
    return torch.cat(codes, 2), torch.cat(scales, 2)


def value64(s, which):
    blocks = torch.arange(s[which + "8"].shape[2], device=DEV) // s["G"]
    return s[which + "8"].double() * torch.exp2(s[which + "s"].double() - 127.0)[:, :, blocks, None]


def appended64(s, rows):
    """The cache after rows {k, v} were written at t0: its codes and scales, as values."""
    G, t0 = s["G"], s["t0"]
    out = []
    for which in "kv":
        first = t0 // G * G
        c, f = encode64(torch.cat([value64(s, which)[:, :, first:t0], rows[which]], 2), G, 0)
        out.append((torch.cat([s[which + "8"][:, :, :first].double(), c], 2),
                    torch.cat([torch.exp2(s[which + "s"][:, :, :first // G].double() - 127.0), f], 2)))
    return [out[0][0], out[1][0], out[0][1], out[1][1]]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    kind, B, H, Hkv, d = c["kind"], c["B"], c["H"], c["Hkv"], c["d"]
    if kind == "append":
        n, t0 = s["q"].shape[1], s["t0"]
        turn = torch.view_as_complex(s["table"][t0:t0 + n].double().contiguous())

        def heads(x, w):
            x = x.double()
            size = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
            y = x / (size.clamp_min(s["eps"]) if c["norm"] == "l2" else (size * size / d + s["eps"]).sqrt()) * w.double()
            y = y.permute(0, 2, 1, 3)
            y = y.reshape(*y.shape[:3], d // 2, 2) if c["layout"] == "pairs" else y.reshape(*y.shape[:3], 2, d // 2).transpose(3, 4)
            y = torch.view_as_real(torch.view_as_complex(y.contiguous()) * turn)
            return (y if c["layout"] == "pairs" else y.transpose(3, 4)).reshape(*y.shape[:3], d)

        q, k, v = heads(s["q"], s["qw"]), heads(s["k"], s["kw"]), s["v"].double().permute(0, 2, 1, 3)
        if c["q8"]:
            return [q] + appended64(s, dict(k=k, v=v))
        before = torch.zeros(B, Hkv, t0, d, dtype=torch.float64, device=DEV)
        return [q, torch.cat([before, k], 2), torch.cat([before, v], 2)]
    if kind == "quantize":
        return appended64(s, dict(k=s["k"].double(), v=s["v"].double()))
    if kind == "dequantize":
        return [value64(s, w)[:, :, s["t0"]:] for w in "kv"]
    k, v = value64(s, "k"), value64(s, "v")
    o, lse = [], []
    for b in range(B):
        for h in range(H):
            q, kk, vv = s["q"][b, h].double(), k[b, h // (H // Hkv)], v[b, h // (H // Hkv)]
            if kind == "dense":
                if s["lens"] is not None:
                    kk, vv = kk[:int(s["lens"][b])], vv[:int(s["lens"][b])]
                z = q @ kk.T / math.sqrt(d)
                lse.append(torch.logsumexp(z, 1))
            else:
                z = q @ kk.T / math.sqrt(d)
                z[~s["keep"][b * H + h][s["qt"]][:, s["kb"]]] = -math.inf
            o.append(torch.softmax(z, 1) @ vv)
    o = torch.stack(o).reshape(B, H, -1, d)
    return [o, torch.stack(lse).reshape(B, H, -1)] if s.get("lse") is not None else [o]
