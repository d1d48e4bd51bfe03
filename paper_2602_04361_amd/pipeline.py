"""One layer of the SparVAR sparse path on the GPU, as a sequence of C-ABI calls.

SparsePath owns the device buffers (allocated with torch) and issues, on the
current stream:
  decision(): dense attention with LSE at the decision scale S, pooled block
              scores and per-query-tile top-k in one sparvar_decision_step
              call (or, with fused=False, sparvar_dense_attn_fwd followed by
              sparvar_select_blocks);
  step(k):    sparvar_map_index (mapped + local blocks -> CSR + schedule), then
              sparvar_block_sparse_attn_fwd at scale k;
  map_all():  the rows of every step in one sparvar_map_index_steps launch
              (they depend only on the selection at S).
Local rows are geometry-only and built once per step by build_local().
Q8SparsePath runs the same steps from the projections on, over an 8-bit cache,
Q4SparsePath over a 4-bit one. BudgetPath attends densely over a 4-bit cache of
bounded length: what its keys got of the attention decides which ones stay.
All arithmetic runs in libsparvar.so; this module only allocates and calls, but for
the token numbers that BudgetPath keeps beside its cache, which torch writes and gathers.
"""
from __future__ import annotations

import math

import torch

from . import sparvar as sv


class SparsePath:
    def __init__(self, geom: sv.Geometry, S, steps, B, H, d, topk, radius, prev_dilation=0,
                 dtype=torch.bfloat16, device="cuda", use_schedule=False, softmax_scale=None, local_lists=False,
                 fused_decision=True, projection="point"):
        self.g = geom
        self.S, self.steps = int(S), [int(k) for k in steps]
        self.B, self.H, self.d = B, H, d
        self.topk, self.radius, self.dil = topk, radius, prev_dilation
        self.dtype, self.device = dtype, device
        # local_lists: build the sink + local rows once with sparvar_local_blocks and
        # pass them to the mapping; otherwise the mapping generates them itself.
        self.local_lists = local_lists
        self.fused_decision = fused_decision
        # projection of the mapped blocks: "point" (tile origin) or "cover" (every tile of the upsampled span)
        self.projection = sv.PROJECTIONS[projection]
        self.scale = float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)) if softmax_scale is None \
            else float(softmax_scale)
        info = {l: geom.scale_info(l) for l in range(1, len(geom.h) + 1)}
        self.info = info
        iS = info[S]
        G_S, NB_S = iS["tiles_h"] * iS["tiles_w"], iS["n_blocks_le"]
        i32 = dict(dtype=torch.int32, device=device)
        self.o_S = torch.empty(B, H, iS["n_tokens"], d, dtype=dtype, device=device)
        self.lse_S = torch.empty(B, H, iS["n_tokens"], dtype=torch.float32, device=device)
        self.scores = torch.empty(B, H, G_S, NB_S, dtype=torch.float32, device=device)
        self.topk_idx = torch.empty(B, H, G_S, topk, **i32)
        self.local, self.csr, self.out = {}, {}, {}
        for k in self.steps:
            ik = info[k]
            G_k = ik["tiles_h"] * ik["tiles_w"]
            cap_l = sv.sparvar_local_blocks_capacity(geom, k, radius, prev_dilation)
            self.local[k] = (torch.empty(G_k + 1, **i32), torch.empty(max(cap_l, 1), **i32))
            cap = sv.sparvar_map_index_capacity(geom, S, k, B, H, topk, radius, prev_dilation, self.projection)
            rows = B * H * G_k
            self.csr[k] = (torch.empty(rows + 1, **i32), torch.empty(cap, **i32),
                           torch.empty(rows, **i32) if use_schedule else None)
            self.out[k] = torch.empty(B, H, ik["n_tokens"], d, dtype=dtype, device=device)
        self.orders = {}

    # ------------------------------------------------------------------ calls
    def build_local(self):
        for k in self.steps:
            rp, ci = self.local[k]
            sv.sparvar_local_blocks(self.g, k, self.radius, rp, ci, prev_dilation=self.dil)

    def q_slice(self, Q_all, l):
        i = self.info[l]
        return Q_all[:, :, i["token_offset"]:i["n_tokens_le"]]

    def kv_prefix(self, X_all, l):
        return X_all[:, :, :self.info[l]["n_tokens_le"]]

    def decision(self, Q_all, K_all, V_all):
        S = self.S
        q, kk, vv = self.q_slice(Q_all, S), self.kv_prefix(K_all, S), self.kv_prefix(V_all, S)
        if self.fused_decision:
            sv.sparvar_decision_step(self.g, S, q, kk, vv, self.o_S, self.lse_S, self.scores, self.topk,
                                     self.topk_idx, softmax_scale=self.scale)
            return
        sv.sparvar_dense_attn_fwd(q, kk, vv, self.o_S, self.lse_S, softmax_scale=self.scale)
        sv.sparvar_select_blocks(self.g, S, q, kk, self.lse_S, self.topk, self.topk_idx, scores_out=self.scores,
                                 softmax_scale=self.scale)

    def map_step(self, k):
        rp_l, ci_l = self.local[k] if self.local_lists else (None, None)
        rp, ci, sch = self.csr[k]
        sv.sparvar_map_index(self.g, self.S, k, self.B, self.H, self.topk, self.topk_idx, rp_l, ci_l, self.radius,
                             rp, ci, schedule=sch, prev_dilation=self.dil, projection=self.projection)

    def map_all(self, orders=False):
        """The rows of every sparse step in one launch (generated local rows); with orders, also each step's
        attention launch order (longest first inside each XCD's share), used by attn_step(use_order=True)."""
        if orders and not self.orders:
            i32 = dict(dtype=torch.int32, device=self.device)
            self.orders = {k: torch.empty(self.B * self.H * self.info[k]["tiles_h"] * self.info[k]["tiles_w"], **i32)
                           for k in self.steps}
        sv.sparvar_map_index_steps(self.g, self.S, self.steps, self.B, self.H, self.topk, self.topk_idx, self.radius,
                                   [self.csr[k][0] for k in self.steps], [self.csr[k][1] for k in self.steps],
                                   prev_dilation=self.dil, projection=self.projection,
                                   orders=[self.orders[k] for k in self.steps] if orders else None)

    def attn_step(self, k, Q_all, K_all, V_all, lse=None, use_schedule=True, use_order=False):
        rp, ci, sch = self.csr[k]
        if use_order:
            sch, use_schedule = self.orders[k], True
        sv.sparvar_block_sparse_attn_fwd(self.g, k, self.q_slice(Q_all, k), self.kv_prefix(K_all, k),
                                         self.kv_prefix(V_all, k), self.out[k], rp, ci, lse=lse,
                                         schedule=sch if use_schedule else None, softmax_scale=self.scale)

    def step(self, k, Q_all, K_all, V_all):
        self.map_step(k)
        self.attn_step(k, Q_all, K_all, V_all)

    def run(self, Q_all, K_all, V_all):
        """Decision step plus every sparse step (with local_lists, build_local() first)."""
        self.decision(Q_all, K_all, V_all)
        for k in self.steps:
            self.step(k, Q_all, K_all, V_all)


class Cs4aPath:
    """One layer of the token-granular CS^4A path (Sec. 3.2) as C-ABI calls.

    decision(): dense attention with LSE at S, column sums over 1-D query blocks
                of C queries, the top-K tokens of each block, and O_cache at S
                (O_dense minus the attention restricted to those tokens);
    step(k):    the token rows of scale k (sinks + mapped tokens), then the
                gather attention, adding the upsampled O_cache unless
                with_cache is False.
    """

    def __init__(self, geom: sv.Geometry, S, steps, B, H, d, C, K, device="cuda", softmax_scale=None,
                 with_cache=True):
        self.g = geom
        self.S, self.steps = int(S), [int(k) for k in steps]
        self.B, self.H, self.d, self.C, self.K = B, H, d, C, K
        self.with_cache = with_cache
        self.scale = float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)) if softmax_scale is None \
            else float(softmax_scale)
        info = {l: geom.scale_info(l) for l in range(1, len(geom.h) + 1)}
        self.info = info
        iS = info[S]
        G_S = -(-iS["n_tokens"] // C)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.o_S = torch.empty(B, H, iS["n_tokens"], d, **bf)
        self.lse_S = torch.empty(B, H, iS["n_tokens"], dtype=torch.float32, device=device)
        self.colsum = torch.empty(B, H, G_S, iS["n_tokens_le"], dtype=torch.float32, device=device)
        self.inds = torch.empty(B, H, G_S, K, dtype=torch.int32, device=device)
        self.o_cache = torch.empty(B, H, iS["n_tokens"], d, **bf)
        self.M = sv.sparvar_cs4a_row_stride(geom, K)
        self.tokens, self.out = {}, {}
        for k in self.steps:
            G_k = -(-info[k]["n_tokens"] // C)
            self.tokens[k] = torch.empty(B, H, G_k, self.M, dtype=torch.int32, device=device)
            self.out[k] = torch.empty(B, H, info[k]["n_tokens"], d, **bf)

    def q_slice(self, Q_all, l):
        i = self.info[l]
        return Q_all[:, :, i["token_offset"]:i["n_tokens_le"]]

    def kv_prefix(self, X_all, l):
        return X_all[:, :, :self.info[l]["n_tokens_le"]]

    def decision(self, Q_all, K_all, V_all):
        S = self.S
        q, kk, vv = self.q_slice(Q_all, S), self.kv_prefix(K_all, S), self.kv_prefix(V_all, S)
        sv.sparvar_dense_attn_fwd(q, kk, vv, self.o_S, self.lse_S, softmax_scale=self.scale)
        sv.sparvar_cs4a_column_sums(self.g, S, self.C, q, kk, self.lse_S, self.colsum, softmax_scale=self.scale)
        sv.sparvar_cs4a_select_tokens(self.colsum, self.K, self.inds)
        if self.with_cache:
            sv.sparvar_cs4a_attn_fwd(self.g, S, self.C, q, kk, vv, self.o_cache, self.inds, self.K, mode=1,
                                     base=self.o_S, softmax_scale=self.scale)

    def step(self, k, Q_all, K_all, V_all):
        sv.sparvar_cs4a_map_tokens(self.g, self.S, k, self.C, self.B, self.H, self.K, self.inds, self.tokens[k],
                                   self.M)
        sv.sparvar_cs4a_attn_fwd(self.g, k, self.C, self.q_slice(Q_all, k), self.kv_prefix(K_all, k),
                                 self.kv_prefix(V_all, k), self.out[k], self.tokens[k], self.M,
                                 mode=2 if self.with_cache else 0, base=self.o_cache if self.with_cache else None,
                                 base_scale=self.S, softmax_scale=self.scale)

    def run(self, Q_all, K_all, V_all):
        self.decision(Q_all, K_all, V_all)
        for k in self.steps:
            self.step(k, Q_all, K_all, V_all)


class CslaPath:
    """One layer of the paper-literal CSLA block path (Sec. 3.3) as C-ABI calls.

    The block rows of each sparse scale depend only on the geometry, the window
    sizes and the block size, so they are built once (rows()) and reused by every
    layer and head; step(k) runs the block-sparse attention of scale k.
    windows[k] lists one window size per scale 1..k (0: no local keys there).
    """

    def __init__(self, geom: sv.Geometry, steps, windows, block, B, H, d, device="cuda", softmax_scale=None):
        self.g = geom
        self.steps = [int(k) for k in steps]
        self.windows = {int(k): [int(w) for w in windows[k]] for k in self.steps}
        self.block, self.B, self.H, self.d = int(block), B, H, d
        self.scale = float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)) if softmax_scale is None \
            else float(softmax_scale)
        self.info = {l: geom.scale_info(l) for l in range(1, len(geom.h) + 1)}
        self.block_rows, self.out = {}, {}
        for k in self.steps:
            M = sv.sparvar_csla_row_stride(geom, k, self.block)
            G_k = -(-self.info[k]["n_tokens"] // self.block)
            self.block_rows[k] = torch.empty(G_k, M, dtype=torch.int32, device=device)
            self.out[k] = torch.empty(B, H, self.info[k]["n_tokens"], d, dtype=torch.bfloat16, device=device)

    def rows(self):
        for k in self.steps:
            sv.sparvar_csla_block_rows(self.g, k, self.windows[k], self.block, self.block_rows[k])

    def step(self, k, Q_all, K_all, V_all):
        i = self.info[k]
        sv.sparvar_csla_attn_fwd(self.g, k, self.block, Q_all[:, :, i["token_offset"]:i["n_tokens_le"]],
                                 K_all[:, :, :i["n_tokens_le"]], V_all[:, :, :i["n_tokens_le"]], self.out[k],
                                 self.block_rows[k], softmax_scale=self.scale)
        return self.out[k]


class Q8SparsePath(SparsePath):
    """One layer over an 8-bit cache that grows scale by scale, as C-ABI calls.

    step(l, q, k, v) takes scale l's projections [B, N_l, heads, d], scales in order:
      append:    norms, rotation and the scale's tokens into the cache
                 (sparvar_qkv_append);
      l < S:     dense attention over the cache (sparvar_dense_attn_q8_fwd);
      l == S:    the cache up to S read back to 16 bits (sparvar_kv_dequantize), the
                 decision step on it, and the rows of every later step;
      l in steps: block-sparse attention over the cache
                 (sparvar_block_sparse_attn_q8_fwd); any other l > S: dense.
    heads: a NormRope whose table has a row for every cache token, or None.
    block: tokens of a scale of the cache. Queries and outputs are bf16, the decision
    is the fused one, and every step's rows come from one mapping launch: SparsePath's
    options that choose among these (dtype, fused_decision, local_lists, use_schedule)
    are not taken.
    """

    def __init__(self, geom: sv.Geometry, S, steps, B, H, d, topk, radius, heads=None, block=64, device="cuda", *,
                 prev_dilation=0, softmax_scale=None, projection="point"):
        super().__init__(geom, S, steps, B, H, d, topk, radius, prev_dilation=prev_dilation, device=device,
                         softmax_scale=softmax_scale, projection=projection)
        self.heads = heads
        bf = dict(dtype=torch.bfloat16, device=device)
        total = self.info[len(geom.h)]["n_tokens_le"]
        self.q8 = sv.Q8Cache.empty(B, H, total, d, block, device)
        self.kv_S = [torch.empty(B, H, self.info[S]["n_tokens_le"], d, **bf) for _ in range(2)]
        self.q = {l: torch.empty(B, H, i["n_tokens"], d, **bf) for l, i in self.info.items()}
        self.out[self.S] = self.o_S
        need = 0
        for l, i in self.info.items():
            if l != self.S and l not in self.steps:
                self.out[l] = torch.empty(B, H, i["n_tokens"], d, **bf)
                need = max(need, sv.sparvar_dense_attn_q8_workspace(B, H, H, i["n_tokens"], i["n_tokens_le"], d))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None

    def append(self, l, q, k, v):
        sv.sparvar_qkv_append(q, k, v, self.info[l]["token_offset"], self.heads, self.q[l], q8=self.q8)

    def dense(self, l):
        sv.sparvar_dense_attn_q8_fwd(self.q[l], self.q8, self.info[l]["n_tokens_le"], self.out[l],
                                     softmax_scale=self.scale, workspace=self.workspace)

    def decision(self):
        k, v = self.kv_S
        sv.sparvar_kv_dequantize(self.q8, 0, k, v)
        sv.sparvar_decision_step(self.g, self.S, self.q[self.S], k, v, self.o_S, self.lse_S, self.scores, self.topk,
                                 self.topk_idx, softmax_scale=self.scale)
        self.map_all()

    def attn_step(self, k):
        rp, ci, _ = self.csr[k]
        sv.sparvar_block_sparse_attn_q8_fwd(self.g, k, self.q[k], self.q8, self.out[k], rp, ci, softmax_scale=self.scale)

    def step(self, l, q, k, v):
        """Scale l from its projections to its attention output."""
        self.append(l, q, k, v)
        if l == self.S:
            self.decision()
        elif l in self.steps:
            self.attn_step(l)
        else:
            self.dense(l)
        return self.out[l]

    def run(self, projections):
        """Every scale in order; projections: (q, k, v) of each."""
        for l, (q, k, v) in enumerate(projections, 1):
            self.step(l, q, k, v)


class Q4SparsePath(SparsePath):
    """One layer over a 4-bit cache that grows scale by scale, as C-ABI calls: Q8SparsePath's steps, with a scale's rows
    appended to 16 bits first (sparvar_qkv_append), written from there (sparvar_kv_quantize_q4), and attention by
    sparvar_dense_attn_q4_fwd and sparvar_block_sparse_attn_q4_fwd. heads as there. Keys are rounded twice, to bf16 and to codes
    (values once: theirs are bf16 already)."""

    def __init__(self, geom: sv.Geometry, S, steps, B, H, d, topk, radius, heads=None, device="cuda", *, prev_dilation=0,
                 softmax_scale=None, projection="point"):
        super().__init__(geom, S, steps, B, H, d, topk, radius, prev_dilation=prev_dilation, device=device,
                         softmax_scale=softmax_scale, projection=projection)
        bf = dict(dtype=torch.bfloat16, device=device)
        total = self.info[len(geom.h)]["n_tokens_le"]
        self.q4 = sv.Q4Cache.empty(B, H, total, d, device)
        self.kv_S = [torch.empty(B, H, self.info[S]["n_tokens_le"], d, **bf) for _ in range(2)]
        self.q, self.heads, self.new = {}, {}, {}
        most = max(i["n_tokens"] for i in self.info.values())
        rows = [torch.empty(B * H * most * d, **bf) for _ in range(2)]
        need = 0
        self.out[self.S] = self.o_S
        for l, i in self.info.items():
            n = i["n_tokens"]
            self.q[l] = torch.empty(B, H, n, d, **bf)
            self.new[l] = [t[:B * H * n * d].view(B, H, n, d) for t in rows]
            self.heads[l] = None if heads is None else heads.rows(i["token_offset"], n)
            if l != self.S and l not in self.steps:
                self.out[l] = torch.empty(B, H, n, d, **bf)
                need = max(need, sv.sparvar_dense_attn_q4_workspace(B, H, H, n, i["n_tokens_le"], d))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None

    def append(self, l, q, k, v):
        kn, vn = self.new[l]
        sv.sparvar_qkv_append(q, k, v, 0, self.heads[l], self.q[l], kn, vn)
        sv.sparvar_kv_quantize_q4(kn, vn, self.info[l]["token_offset"], self.q4)

    def dense(self, l):
        sv.sparvar_dense_attn_q4_fwd(self.q[l], self.q4, self.info[l]["n_tokens_le"], self.out[l], softmax_scale=self.scale,
                                     workspace=self.workspace)

    def decision(self):
        k, v = self.kv_S
        sv.sparvar_kv_dequantize_q4(self.q4, 0, k, v)
        sv.sparvar_decision_step(self.g, self.S, self.q[self.S], k, v, self.o_S, self.lse_S, self.scores, self.topk,
                                 self.topk_idx, softmax_scale=self.scale)
        self.map_all()

    def attn_step(self, k):
        rp, ci, _ = self.csr[k]
        sv.sparvar_block_sparse_attn_q4_fwd(self.g, k, self.q[k], self.q4, self.out[k], rp, ci, softmax_scale=self.scale)

    def step(self, l, q, k, v):
        """Scale l from its projections to its attention output."""
        self.append(l, q, k, v)
        if l == self.S:
            self.decision()
        elif l in self.steps:
            self.attn_step(l)
        else:
            self.dense(l)
        return self.out[l]

    def run(self, projections):
        """Every scale in order; projections: (q, k, v) of each."""
        for l, (q, k, v) in enumerate(projections, 1):
            self.step(l, q, k, v)


class BudgetPath:
    """One dense layer whose 4-bit cache is held to a budget of tokens, as C-ABI calls.

    step(q, k, v) takes the projections [B, n, heads, d] of the next n tokens (n <= n_max; a scale, or one token):
      append:  norms and rotation to 16 bits (sparvar_qkv_append), rows to the cache (sparvar_kv_quantize_q4): keys are
               rounded twice, to bf16 and to codes;
      attend:  dense attention over the cache (sparvar_dense_attn_q4_fwd);
      weigh:   what each cached key got of it, added to decay times what it had (sparvar_key_weights);
      evict:   where more than `budget` tokens are held, the n_first first, the n_last last and those of largest weight
               move to the other of two caches (sparvar_kv_evict), which is the cache from then on. All that stay
               move, also where one token goes.
    held: tokens in the cache; tokens [B, H_kv, held]: which of the sequence they are, a row for each key head.
    heads: a NormRope whose table has a row for every token of the sequence, or None.
    """

    def __init__(self, B, H, H_kv, d, n_max, budget, n_first=0, n_last=0, heads=None, decay=1.0, device="cuda",
                 softmax_scale=None):
        if min(n_max, budget) < 1 or min(n_first, n_last) < 0 or n_first + n_last > budget:
            raise ValueError("n_max and budget must be >= 1, n_first and n_last >= 0 and at most the budget together")
        self.B, self.H, self.H_kv, self.d = B, H, H_kv, d
        self.n_max, self.budget, self.n_first, self.n_last = int(n_max), int(budget), int(n_first), int(n_last)
        self.heads, self.decay = heads, float(decay)
        self.scale = float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32)) if softmax_scale is None \
            else float(softmax_scale)
        cap = self.budget + self.n_max
        self.caches = [sv.Q4Cache.empty(B, H_kv, cap, d, device) for _ in range(2)]
        self.weights = [torch.empty(B, H_kv, cap, device=device) for _ in range(2)]
        self.order = [torch.empty(B, H_kv, cap, dtype=torch.int64, device=device) for _ in range(2)]
        self.kept = torch.empty(B, H_kv, self.budget, dtype=torch.int32, device=device)
        bf = dict(dtype=torch.bfloat16, device=device)
        self.rows = [torch.empty(B * h * self.n_max * d, **bf) for h in (H, H_kv, H_kv, H)]
        self.lse_rows = torch.empty(B * H * self.n_max, device=device)
        self.workspace = None
        self.held = self.seen = 0

    def _view(self, i, heads, n):
        return self.rows[i][:self.B * heads * n * self.d].view(self.B, heads, n, self.d)

    @property
    def q4(self):
        return self.caches[0]

    @property
    def w(self):
        return self.weights[0]

    @property
    def tokens(self):
        return self.order[0][:, :, :self.held]

    def append(self, q, k, v):
        n = q.shape[1]
        if not 1 <= n <= self.n_max:
            raise ValueError(f"a step of {n} tokens, n_max is {self.n_max}")
        self.q, kn, vn = self._view(0, self.H, n), self._view(1, self.H_kv, n), self._view(2, self.H_kv, n)
        heads = None if self.heads is None else self.heads.rows(self.seen, n)
        sv.sparvar_qkv_append(q, k, v, 0, heads, self.q, kn, vn)
        sv.sparvar_kv_quantize_q4(kn, vn, self.held, self.q4)
        self.order[0][:, :, self.held:self.held + n] = torch.arange(self.seen, self.seen + n, device=self.kept.device)
        self.old, self.held, self.seen = self.held, self.held + n, self.seen + n

    def attend(self):
        n = self.q.shape[2]
        need = sv.sparvar_dense_attn_q4_workspace(self.B, self.H, self.H_kv, n, self.held, self.d)
        if need and (self.workspace is None or self.workspace.numel() < need):
            self.workspace = torch.empty(need, dtype=torch.uint8, device=self.kept.device)
        self.out, self.lse = self._view(3, self.H, n), self.lse_rows[:self.B * self.H * n].view(self.B, self.H, n)
        sv.sparvar_dense_attn_q4_fwd(self.q, self.q4, self.held, self.out, lse=self.lse, softmax_scale=self.scale,
                                     workspace=self.workspace if need else None)

    def weigh(self):
        sv.sparvar_key_weights(self.q, self.held, self.lse, self.w, w_old=self.w, n_old=self.old, decay=self.decay, q4=self.q4,
                               softmax_scale=self.scale)

    def evict(self):
        if self.held <= self.budget:
            return
        sv.sparvar_kv_evict(self.w, self.held, self.budget, self.n_first, self.n_last, self.kept, self.weights[1],
                            q4_src=self.q4, q4_dst=self.caches[1])
        torch.gather(self.order[0], 2, self.kept.long(), out=self.order[1][:, :, :self.budget])
        for pair in (self.caches, self.weights, self.order):
            pair.reverse()
        self.held = self.budget

    def step(self, q, k, v):
        """The next tokens from their projections to their attention output [B, H, n, d] (valid until the next step)."""
        self.append(q, k, v)
        self.attend()
        self.weigh()
        self.evict()
        return self.out
