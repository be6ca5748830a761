"""Paged cache: batches of sequences for the tests, and the three operators in 64 bits."""
import math

import torch

from paper_2607_15498_gb300 import varrate as V

D = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}    # half a rounding step, relative


class Batch:
    """Sequences with (new, context) tokens over shuffled pages. Slots past a sequence's tokens, spare pages and the
    rows that belong to no sequence hold `junk`."""

    def __init__(self, lens, dtype="bf16", G=2, grp=4, ps=16, layers=1, pad=0, lead=0, spare=3, seed=0, junk=float("nan"),
                 device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.G, self.grp, self.H, self.ps, self.layers = lens, G, grp, G * grp, ps, layers
        self.dtype, self.dt, self.pad, self.gen, self.device = dtype, DT[dtype], pad, gen, device
        self.total = sum(n for n, _ in lens)
        self.start = [lead]
        for n, _ in lens:
            self.start.append(self.start[-1] + n)
        self.T = self.start[-1] + pad
        self.len = [n + c for n, c in lens]
        need = [-(-k // ps) for k in self.len]
        self.max_pages = max([1] + need) + 1
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=gen).tolist()
        table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32)   # entries past the last page: never looked at
        at = 0
        for s, p in enumerate(need):
            table[s, :p] = torch.tensor(order[at:at + p], dtype=torch.int32)
            at += p
        self.table_host = table
        pool = torch.full((layers, self.n_pages, 2, G, ps, D), junk, dtype=torch.float64)
        for s, k in enumerate(self.len):
            for u in range(k):
                pool[:, table[s, u // ps], :, :, u % ps] = self.randn(layers, 2, G, D)
        self.pool = pool.to(self.dt).to(device)
        self.table = table.to(device)
        self.row_start = torch.tensor(self.start, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor(self.len, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.pages = V.PagedCache.of(self.pool)
        self.seqs = V.SeqBatch.of(self.row_start, self.kv_len, self.table, self.T)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, dtype=torch.float64)

    def rows(self, heads, fused=None):
        """Random rows [T][heads][d]; `fused`: as a part of wider rows."""
        x = self.randn(self.T, heads + (fused or 0), D).to(self.dt).to(self.device)
        return x[:, (fused or 0) // 2:(fused or 0) // 2 + heads]

    def tokens(self, s, c, layer=0, pool=None):
        """[G][tokens][d] of a sequence's keys (0) or values (1), 64 bits."""
        pool = self.pool if pool is None else pool
        u = torch.arange(self.len[s], device=pool.device)
        page = self.table_host[s].to(pool.device).long()[u // self.ps]
        return pool[layer, page, c, :, u % self.ps].double().transpose(0, 1)

    def workspace(self):
        return V.paged_attn_workspace(self.pages, self.seqs, self.grp)


def form(x, w, eps, freq, rot, pos):
    """Norm and rotation of x [rows][heads][d] in 64 bits, and |y_i| + |y_partner| (what roundings are relative to)."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    size, h = x.abs(), rot // 2
    if h:
        a = pos.double()[:, None, None] * freq.to(x.device)
        a0, a1 = x[..., :h], x[..., h:rot]
        z = torch.cat((a0 * a.cos() - a1 * a.sin(), a1 * a.cos() + a0 * a.sin(), x[..., rot:]), -1)
        pair = a0.abs() + a1.abs()
        return z, torch.cat((pair, pair, size[..., rot:]), -1)
    return x, size


def append_ref(b, q, k, v, wq, wk, eps, freq, rot, layer, before):
    """(queries, pool, allowed error of each) that an append of the batch gives; `before`: the pool as it was."""
    q_out = torch.full((b.T, b.H, D), float("nan"), dtype=torch.float64, device=b.device)
    pool, q_tol, p_tol = before.double(), torch.zeros_like(q_out), torch.zeros(before.shape, dtype=torch.float64, device=b.device)
    # fp32: the sum of squares (12 roundings, halved by the root), its scaling, the root and the two products 13 half
    # steps; the angle's 3.2 and the sine's 2; the two products 2: below 32 half steps of 2^-24 of |y| + |y'|
    fp32 = 32 * 2.0 ** -24
    for s, (n, _) in enumerate(b.lens):
        lo, hi = b.start[s], b.start[s + 1]
        pos = torch.arange(b.len[s] - n, b.len[s], device=b.device)
        if q is not None:
            q_out[lo:hi], size = form(q[lo:hi], wq, eps, freq, rot, pos)
            q_tol[lo:hi] = fp32 * size + HALF[b.dtype] * (q_out[lo:hi].abs() + fp32 * size)
        page = b.table_host[s].to(b.device).long()[pos // b.ps]
        z, size = form(k[lo:hi], wk, eps, freq, rot, pos)
        pool[layer, page, 0, :, pos % b.ps] = z
        p_tol[layer, page, 0, :, pos % b.ps] = fp32 * size + HALF[b.dtype] * (z.abs() + fp32 * size)
        pool[layer, page, 1, :, pos % b.ps] = v[lo:hi].double()
    return q_out, pool, q_tol, p_tol


def attn_ref(b, q, layer=0, pool=None):
    """(attention in 64 bits, allowed error) for every row of a sequence, NaN rows elsewhere. What a token does not see
    is left out of its sums, not multiplied by zero."""
    out = torch.full((b.T, b.H, D), float("nan"), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for s, (n, c) in enumerate(b.lens):
        if n == 0:
            continue
        lo, hi = b.start[s], b.start[s + 1]
        k, v = b.tokens(s, 0, layer, pool), b.tokens(s, 1, layer, pool)
        total = b.len[s]
        seen = torch.arange(total, device=q.device)[None] <= torch.arange(c, total, device=q.device)[:, None]
        vis = seen[None, :, :, None]
        for h in range(b.H):
            g = h // b.grp
            w = (q[lo:hi, h].double() @ k[g].T) / math.sqrt(D)
            w = w.masked_fill(~seen, -math.inf)
            w = torch.exp(w - w.amax(-1, keepdim=True))
            w = w / w.sum(-1, keepdim=True)
            vv = torch.where(vis[0], v[g][None], 0.0) if not torch.isfinite(v[g]).all() else None
            if vv is None:
                out[lo:hi, h], mass = w @ v[g], w @ v[g].abs()
            else:
                out[lo:hi, h], mass = (w[..., None] * vv).sum(1), (w[..., None] * vv.abs()).sum(1)
            # a score: 128 products summed in fp32 (2^-23 a step on the tensor cores), scaled; twice its largest error
            # in the weights and their sum; exp2 2^-21; the sums over the tokens one rounding a token and tile
            size = (q[lo:hi, h].double().abs() @ torch.where(torch.isfinite(k[g]), k[g], 0.0).abs().T) / math.sqrt(D)
            ds = 132 * 2.0 ** -23 * torch.where(seen, size, 0.0).amax(-1, keepdim=True)
            rel = 2 * ds + 2.0 ** -20 + 2 * (total + 8) * 2.0 ** -24
            if b.dtype == "bf16":
                rel = rel + 2.0 ** -8            # weights rounded to bf16
            tol[lo:hi, h] = rel * mass + HALF[b.dtype] * (out[lo:hi, h].abs() + rel * mass)
    return out, tol


def close(got, want, tol):
    """Largest error over what is allowed, with the same infinities and NaN on both sides."""
    got = got.double()
    nan = torch.isnan(want)
    assert torch.equal(nan, torch.isnan(got)), "NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), "infinities in other places"
    fine = ~nan & ~inf
    if not fine.any():
        return 0.0
    err = (got[fine] - want[fine]).abs()
    assert (err <= tol[fine]).all(), (err - tol[fine]).max().item()
    return float((err / tol[fine].clamp_min(1e-300)).max()) if err.any() else 0.0
