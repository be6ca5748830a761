"""Paged cache in 8 bits: batches of sequences for the tests, and the four operators in 64 bits."""
import math

import torch

from paged_helpers import D, form
from paper_2607_15498_gb300 import varrate as V

BLOCK = 16
NAN_CODE = 0x7F


def round8(x):
    """64-bit numbers to the nearest e4m3 number, ties to even, 448 at most."""
    step = torch.exp2(torch.frexp(x).exponent.clamp(min=-5).double() - 4)
    return (torch.round(x / step) * step).clamp(-448, 448)


def least_byte(most):
    """Scale byte of a block whose largest element is `most` (64 bits)."""
    e = torch.ceil(torch.log2(most / 448))
    e = e + (most > 448 * torch.exp2(e)).double() - (most <= 448 * torch.exp2(e - 1)).double()
    return torch.where(most == 0, 0.0, (e + 127).clamp(1, 246))


def factor(byte):
    return torch.exp2(byte.double() - 127)


def quantise(x):
    """(codes uint8, scale bytes) of x [..., tokens (of whole blocks), d], 64 bits."""
    b = x.unflatten(-2, (-1, BLOCK))
    byte = least_byte(b.abs().amax((-1, -2)))
    codes = round8(b / factor(byte)[..., None, None]).flatten(-3, -2).float().to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), byte.to(torch.uint8)


class Batch8:
    """Sequences with (new, context) tokens over shuffled pages. Codes, scales and weights past a sequence's tokens, spare pages
    and the rows that belong to no sequence hold junk: NaN codes, any scale, NaN."""

    def __init__(self, lens, G=2, grp=4, ps=16, layers=1, pad=0, lead=0, spare=3, seed=0, spread=1.0, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.G, self.grp, self.H, self.ps, self.layers = lens, G, grp, G * grp, ps, layers
        self.pad, self.gen, self.device, self.dtype = pad, gen, device, "bf16"
        self.total = sum(n for n, _ in lens)
        self.start = [lead]
        for n, _ in lens:
            self.start.append(self.start[-1] + n)
        self.T = self.start[-1] + pad
        self.len = [n + c for n, c in lens]
        need = [-(-k // ps) for k in self.len]
        self.max_pages, self.n_pages = max([1] + need) + 1, sum(need) + spare
        order = torch.randperm(self.n_pages, generator=gen).tolist()
        table = torch.full((len(lens), self.max_pages), -7, dtype=torch.int32)
        at = 0
        for s, p in enumerate(need):
            table[s, :p] = torch.tensor(order[at:at + p], dtype=torch.int32)
            at += p
        self.table_host = table
        codes = torch.full((layers, self.n_pages, 2, G, ps, D), NAN_CODE, dtype=torch.uint8)
        scale = torch.randint(1, 247, (layers, self.n_pages, 2, G, ps // BLOCK), generator=gen).to(torch.uint8)
        mass = torch.full((layers, self.n_pages, G, ps), float("nan"))
        for s, k in enumerate(self.len):
            for page in range(need[s]):
                n = min(ps, k - page * ps)
                x = self.randn(layers, 2, G, ps, D)
                x[..., n:, :] = 0
                # blocks differ in size
                x *= torch.exp2(spread * self.randn(layers, 2, G, ps // BLOCK, 1, 1)).expand(-1, -1, -1, -1, BLOCK, 1).flatten(3, 4)
                q, b = quantise(x)
                t = int(table[s, page])
                codes[:, t, :, :, :n] = q[..., :n, :]
                whole = -(-n // BLOCK)
                scale[:, t, :, :, :whole] = b[..., :whole]
                m = torch.rand((layers, G, n), generator=gen)
                mass[:, t, :, :n] = torch.where(m < 0.1, 0.0, m ** 4)
        self.codes, self.scale, self.mass = codes.to(device), scale.to(device), mass.to(device)
        self.table = table.to(device)
        self.row_start = torch.tensor(self.start, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor(self.len, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.pages = V.Paged8Cache.of(self.codes, self.scale, self.mass)
        self.seqs = V.SeqBatch.of(self.row_start, self.kv_len, self.table, self.T)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, dtype=torch.float64)

    def rows(self, heads, fused=None):
        """Random rows [T][heads][d]; `fused`: as a part of wider rows."""
        x = self.randn(self.T, heads + (fused or 0), D).bfloat16().to(self.device)
        return x[:, (fused or 0) // 2:(fused or 0) // 2 + heads]

    def place(self, s, u):
        """Pages and slots of places u of a sequence."""
        return self.table_host[s].to(u.device).long()[u // self.ps], u % self.ps

    def values(self, codes=None, scale=None):
        """The cache in 64 bits."""
        codes, scale = self.codes if codes is None else codes, self.scale if scale is None else scale
        return codes.view(torch.float8_e4m3fn).float().double() * factor(scale).repeat_interleave(BLOCK, -1)[..., None]

    def tokens(self, s, c, layer=0, pool=None):
        """[G][tokens][d] of a sequence's keys (0) or values (1), 64 bits."""
        pool = self.values() if pool is None else pool
        p, i = self.place(s, torch.arange(self.len[s], device=pool.device))
        return pool[layer, p, c, :, i].transpose(0, 1)

    def workspace(self):
        return V.paged8_attn_workspace(self.pages, self.seqs, self.grp)


def append8_check(b, args, layer, before, q_out, lens=None):
    """Compares the cache and queries after an append of the whole batch with the formulas; `before`: (codes, scale, mass) as they
    were. Returns nothing; asserts."""
    q, k, v, wq, wk, eps, freq, rot, gone = args
    codes0, scale0, mass0 = (t.clone() for t in before)
    dev = b.device
    fp32 = 32 * 2.0 ** -24                   # as for the append of the uncompressed cache
    got_codes, got_scale = b.codes.clone(), b.scale.clone()
    touched = torch.zeros(b.codes.shape[:-1], dtype=torch.bool, device=dev)
    blocks = torch.zeros(b.scale.shape, dtype=torch.bool, device=dev)
    fresh = torch.zeros(b.mass.shape, dtype=torch.bool, device=dev)
    for s, (n, _) in enumerate(b.lens):
        if n == 0:
            continue
        lo, hi, first = b.start[s], b.start[s + 1], b.len[s] - n
        u = torch.arange(first, b.len[s], device=dev)
        pos = u + (0 if gone is None else int(gone[s]))
        if q is not None:
            want, size = form(q[lo:hi], wq, eps, freq, rot, pos)
            tol = fp32 * size + 2.0 ** -8 * (want.abs() + fp32 * size)
            assert ((q_out[lo:hi].double() - want).abs() <= tol).all()
        zk, size = form(k[lo:hi], wk, eps, freq, rot, pos)
        z = torch.stack((zk, v[lo:hi].double()))                     # [2][n][G][d]
        sz = torch.stack((size, torch.zeros_like(size)))
        p, i = b.place(s, u)
        fresh[layer, p, :, i] = True
        for block in range(first // BLOCK, -(-b.len[s] // BLOCK)):
            a, e = max(first, block * BLOCK), min(b.len[s], (block + 1) * BLOCK)
            page, at = int(b.table_host[s, block * BLOCK // b.ps]), block * BLOCK % b.ps
            old = a - block * BLOCK
            new, new_size = (t[:, a - first:e - first].transpose(1, 2) for t in (z, sz))   # [2][G][tokens][d]
            most = torch.where(torch.isfinite(new), new.abs(), 0.0).amax((-1, -2))
            byte = least_byte(most)
            near = (most / (448 * factor(least_byte(most))) - 1).abs() < 1e-5   # a last place of fp32 may decide
            was = scale0[layer, page, :, :, at // BLOCK].double()
            if old:
                byte = torch.maximum(byte, was)
            got = got_scale[layer, page, :, :, at // BLOCK].double()
            assert torch.equal(torch.where(near, got, byte), got), (s, block, byte, got)
            f = factor(got)[..., None, None]
            if old:
                held = codes0[layer, page, :, :, at:at + old].view(torch.float8_e4m3fn).float().double()
                want = round8(held * (factor(was) / factor(got))[..., None, None])
                have = got_codes[layer, page, :, :, at:at + old].view(torch.float8_e4m3fn).float().double()
                assert torch.equal(torch.nan_to_num(want, nan=9e9), torch.nan_to_num(have, nan=9e9)), (s, block)
            have = got_codes[layer, page, :, :, at + old:at + e - block * BLOCK].view(torch.float8_e4m3fn).float().double()
            assert torch.equal(torch.isnan(have), ~torch.isfinite(new)), (s, block)
            ok = torch.isfinite(new)
            err = fp32 * new_size
            z1 = new.clamp(-448 * f, 448 * f)
            tol = err + torch.maximum(2.0 ** -4 * (z1.abs() + err), 2.0 ** -10 * f)
            assert ((have * f - z1).abs() <= tol)[ok].all(), (s, block, ((have * f - z1).abs() - tol)[ok].max())
            touched[layer, page, :, :, at:at + e - block * BLOCK] = True
            blocks[layer, page, :, :, at // BLOCK] = True
    assert torch.equal(got_codes[~touched], codes0[~touched]), "codes of other tokens"
    assert torch.equal(got_scale[~blocks], scale0[~blocks]), "scales of other blocks"
    assert (b.mass[fresh] == 0).all()
    same = torch.nan_to_num(b.mass, nan=-1.0)[~fresh] == torch.nan_to_num(mass0, nan=-1.0)[~fresh]
    assert same.all(), "weights of other tokens"


def logits(b, q, s, g, layer=0, pool=None):
    """Scores [new][group][tokens] of a sequence and KV head in 64 bits, -infinity where a token is not seen, and |q| |k| sums."""
    n, c = b.lens[s]
    k = b.tokens(s, 0, layer, pool)[g]
    x = q[b.start[s]:b.start[s + 1], g * b.grp:(g + 1) * b.grp].double()
    w = torch.einsum("ihd,td->iht", x, k) / math.sqrt(D)
    size = torch.einsum("ihd,td->iht", x.abs(), torch.where(torch.isfinite(k), k, 0.0).abs()) / math.sqrt(D)
    seen = torch.arange(n + c, device=q.device)[None] <= torch.arange(c, n + c, device=q.device)[:, None]
    return w.masked_fill(~seen[:, None], -math.inf), torch.where(seen[:, None], size, 0.0), seen


def score_error(size):
    """What a score may be off: 128 exact products summed in fp32 (2^-23 a step on the tensor cores) and four multiplications."""
    return 132 * 2.0 ** -23 * size.amax(-1, keepdim=True)


def attn8_ref(b, q, layer=0, pool=None):
    """(attention, its allowed error, lse, its allowed error), in 64 bits; NaN where a row is of no sequence."""
    pool = b.values() if pool is None else pool
    out = torch.full((b.T, b.H, D), float("nan"), dtype=torch.float64, device=q.device)
    lse = torch.full((b.T, b.H), float("nan"), dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for s, (n, c) in enumerate(b.lens):
        if n == 0:
            continue
        rows = slice(b.start[s], b.start[s + 1])
        for g in range(b.G):
            heads = slice(g * b.grp, (g + 1) * b.grp)
            w, size, seen = logits(b, q, s, g, layer, pool)
            v = b.tokens(s, 1, layer, pool)[g]
            y = torch.logsumexp(w, -1)
            a = torch.softmax(w, -1)
            if torch.isfinite(v).all():
                o, mass = torch.einsum("iht,td->ihd", a, v), torch.einsum("iht,td->ihd", a, v.abs())
            else:
                vv = torch.where(seen[..., None], v[None], 0.0)
                o, mass = (a[..., None] * vv[:, None]).sum(2), (a[..., None] * vv[:, None].abs()).sum(2)
            # twice a score's error in the weights and their sum; exp2 2^-21; sums a rounding a token; weights to bf16 at worst
            ds = score_error(size)
            rel = 2 * ds + 2.0 ** -20 + 2 * (n + c + 8) * 2.0 ** -24 + 2.0 ** -8
            out[rows, heads], lse[rows, heads] = o, y
            tol[rows, heads] = rel * mass + 2.0 ** -8 * (o.abs() + rel * mass)
            tol_lse[rows, heads] = ds[..., 0] + 2.0 ** -20 + (n + c + 8) * 2.0 ** -24 + 4 * 2.0 ** -24 * (1 + y.abs())
    return out, tol, lse, tol_lse


def mass8_ref(b, q, lse, before, layer=0):
    """(weights of every token after varrate_paged8_mass, their allowed error), 64 bits."""
    out, tol = before.double().clone(), torch.zeros(before.shape, dtype=torch.float64, device=q.device)
    pool = b.values()
    for s, (n, c) in enumerate(b.lens):
        if n == 0:
            continue
        p, i = b.place(s, torch.arange(n + c, device=q.device))
        for g in range(b.G):
            w, size, _ = logits(b, q, s, g, layer, pool)
            y = lse[b.start[s]:b.start[s + 1], g * b.grp:(g + 1) * b.grp].double()
            a = torch.exp(w - torch.where(torch.isfinite(y), y, math.inf)[..., None])
            # a score's error, that of lse log2 e (a rounding, and one of the difference), exp2 2^-21; the sum a rounding a row
            err = score_error(size) + 2.0 ** -23 * (torch.nan_to_num(y, 0, 0, 0).abs()[..., None] * 2 + 1) + 2.0 ** -20
            err = err + n * b.grp * 2.0 ** -24
            out[layer, p, g, i] += a.sum((0, 1))
            # a weight below 2^-126 is no normal number of fp32 and counts as 0: n rows of the group lose less than that each
            tol[layer, p, g, i] = (a * err).sum((0, 1)) + 2.0 ** -24 * out[layer, p, g, i].abs() + n * b.grp * 2.0 ** -126
    return out, tol


def evict8_ref(b, layer, n_layers, budget, n_first, n_last):
    """(codes, scale, mass, kept, new_len) after an eviction, exact."""
    codes, scale, mass = b.codes.clone(), b.scale.clone(), b.mass.clone()
    S = len(b.lens)
    kept = torch.full((S, n_layers, b.G, budget), -1, dtype=torch.int32)
    for s, n in enumerate(b.len):
        for l in range(layer, layer + n_layers):
            for g in range(b.G):
                if n <= budget:
                    kept[s, l - layer, g, :n] = torch.arange(n)
                    continue
                p, i = b.place(s, torch.arange(n, device=b.device))
                m = b.mass[l, p, g, i].double().cpu()
                m = torch.where(torch.isnan(m), math.inf, m).tolist()   # (of inputs without infinities)
                by = sorted(range(n_first, n - n_last), key=lambda u: (-m[u], u))[:budget - n_first - n_last]
                src = torch.tensor(list(range(n_first)) + sorted(by) + list(range(n - n_last, n)), device=b.device)
                kept[s, l - layer, g] = src.int().cpu()
                (ps, sl), (pd, dl) = b.place(s, src), b.place(s, torch.arange(budget, device=b.device))
                mass[l, pd, g, dl] = b.mass[l, ps, g, sl]
                for c in range(2):
                    byte = b.scale[l, ps, c, g, sl // BLOCK].double()
                    pad = torch.nn.functional.pad(byte, (0, -budget % BLOCK)).unflatten(0, (-1, BLOCK)).amax(1)
                    new = pad.repeat_interleave(BLOCK)[:budget]
                    x = b.codes[l, ps, c, g, sl].view(torch.float8_e4m3fn).float().double()
                    x = round8(x * torch.exp2(byte - new)[:, None])
                    codes[l, pd, c, g, dl] = x.float().to(torch.float8_e4m3fn).view(torch.uint8)
                    scale[l, pd, c, g, dl // BLOCK] = new.to(torch.uint8)
    return codes, scale, mass, kept.to(b.device), b.kv_len.clamp(max=budget)
