"""Performance cases of the paged cache: the calls that bring a sequence up to the codec and past it.

A serving program keeps the keys and values of tokens that are not coded yet in pages
``pool [layers][pages][2][kv_heads][page][128]`` (0: keys, 1: values). A batch is described by
``row_start [seqs + 1]`` (rows of each sequence's new tokens), ``kv_len [seqs]`` (tokens of a sequence, the
new ones included) and ``table [seqs][pages of a sequence]``. Three operators, each through the public entry
points of ``paper_2607_15498_gb300.varrate``:

* ``append``  varrate_paged_append: norm of every query and key head (where the model has one), position
              rotation, queries out, keys and values into their pages.
* ``attn``    varrate_paged_attn: causal attention of the new tokens over the pages; one new token of a
              sequence is a decode step, many are a chunk of its prompt.
* ``gather``  varrate_paged_gather: a range of tokens out of the pages, dense, as varrate_encode (a whole
              prompt, several layers) and the exact tail of varrate_decode_attn (one layer) take it.

The first ``chunks`` sequences bring ``new_lo`` to ``new_hi`` new tokens, the others one; each has ``ctx_lo`` to
``ctx_hi`` tokens before them. These lengths are drawn from ``mix``, so they belong to the case. ``pad`` rows
stand behind the last sequence's, as in a batch that is padded to a captured size. Queries and keys have
logits of a few units and a share of keys of 4 times the size.
"""
import math
import random

import torch

own = False

D = 128
OPS = ("append", "attn", "gather")


def _case(op, **kw):
    c = {"op": op, "dtype": "bf16", "kv_heads": 8, "group": 4, "page": 64, "layers": 1, "seqs": 1, "chunks": 0,
         "new_lo": 1, "new_hi": 1, "ctx_lo": 0, "ctx_hi": 0, "pad": 0, "norm": False, "rot": 128, "fused": True, "n": 0,
         "mix": 1}
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of eight sequences, one layer: a launch and a few kilobytes
        dict(_case("append", seqs=8, ctx_lo=2000, ctx_hi=8000), name="append_step_batch8"),
        # a small fp32 model with head norms, a chunk of a few prompts
        dict(_case("append", dtype="f32", kv_heads=1, seqs=3, chunks=3, new_lo=100, new_hi=700, ctx_hi=1400, norm=True, page=16, fused=False), name="append_chunk_f32"),
        # an 8192-token prompt in one piece, keys and values straight out of the joint projection
        dict(_case("append", chunks=1, new_lo=8192, new_hi=8192), name="append_prompt_8k"),
        # prompts of many lengths at once, group 7, head norms, half of each head rotated, a padded batch
        dict(_case("append", kv_heads=4, group=7, seqs=24, chunks=23, new_lo=300, new_hi=4000, ctx_hi=2000, norm=True, rot=64, page=32, pad=37), name="append_prompts_ragged"),
        # one token of one short sequence: latency
        dict(_case("attn", ctx_lo=899, ctx_hi=899), name="attn_step_short"),
        # one decode step of eight 32k sequences: bandwidth
        dict(_case("attn", seqs=8, ctx_lo=32767, ctx_hi=32767), name="attn_step_batch8_32k"),
        # a serving step of group 7: a chunk of one prompt beside the single tokens of running sequences
        dict(_case("attn", kv_heads=4, group=7, seqs=24, chunks=1, new_lo=383, new_hi=383, ctx_lo=60, ctx_hi=7800, page=16, pad=11), name="attn_mixed_step"),
        # an 8192-token prompt in one piece: tensor cores
        dict(_case("attn", chunks=1, new_lo=8192, new_hi=8192), name="attn_prompt_8k"),
        # a chunk of 512 tokens at the end of a 131072-token context
        dict(_case("attn", chunks=1, new_lo=512, new_hi=512, ctx_lo=130560, ctx_hi=130560, page=128), name="attn_chunk_131k"),
        # the small fp32 model: two chunks, one of odd length
        dict(_case("attn", dtype="f32", kv_heads=1, seqs=2, chunks=2, new_lo=500, new_hi=1100, ctx_hi=1000, page=32), name="attn_chunk_f32"),
        # the exact tails of eight sequences, for the decode calls of one layer
        dict(_case("gather", seqs=8, ctx_lo=2000, ctx_hi=4000, n=160), name="gather_tail_batch8"),
        # a finished 32k prompt, four layers of it, on its way to the encode
        dict(_case("gather", layers=4, ctx_lo=32767, ctx_hi=32767, n=32768), name="gather_prompt_32k"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    f32 = rng.random() < 0.2
    G, grp = rng.randint(1, 8), rng.randint(1, 8)
    kw = dict(dtype="f32" if f32 else "bf16", kv_heads=G, group=grp, page=rng.choice([16, 32, 64, 128, 256]),
              mix=rng.randint(1, 1 << 20), pad=rng.choice([0, 0, rng.randint(1, 40)]))
    if op == "append":
        seqs = _log(rng, 1, 64)
        rows = _log(rng, seqs, 8192 if f32 else 24000)            # new rows in all, about
        most = max(2, min(8192, 2 * rows // seqs))
        ctx = _log(rng, 16, max(17, min(8000, (1 << 18) // seqs)))
        kw.update(seqs=seqs, chunks=rng.choice([seqs, max(0, seqs - 1)]), new_lo=1, new_hi=most, ctx_lo=0, ctx_hi=ctx,
                  norm=rng.random() < 0.5, rot=rng.choice([128, 128, 64, 32, 0]), fused=rng.random() < 0.5)
    elif op == "attn":
        seqs, room = _log(rng, 1, 64), 1 << (28 if f32 else 31)
        # a padded batch holds no more (query, key, head) triples than the largest listed prompt, 8192 x 8192 x 32
        new = rng.choice([1, _log(rng, 2, 8192)])
        new = max(1, min(new, math.isqrt(room // (seqs * G * grp))))
        most = min(131072, room // (seqs * G * grp * new), (1 << (18 if f32 else 21)) // (seqs * G))
        new = min(new, most)
        ctx = _log(rng, max(16, new), max(17, most))
        kw.update(seqs=seqs, chunks=rng.randint(1, seqs) if new > 1 else 0, new_lo=max(1, new // 3), new_hi=new,
                  ctx_lo=max(0, (ctx - new) // 50), ctx_hi=max(0, ctx - new))
    else:
        seqs, n = _log(rng, 1, 16), _log(rng, 1, 32768)
        layers = max(1, min(_log(rng, 1, 8), (1 << (19 if f32 else 20)) // (seqs * n * G)))
        seqs = max(1, min(seqs, (1 << (19 if f32 else 20)) // (layers * n * G)))
        n = max(1, min(n, (1 << (19 if f32 else 20)) // (layers * seqs * G)))
        kw.update(seqs=seqs, layers=layers, n=n, ctx_lo=n, ctx_hi=n + rng.randint(0, 1000), pad=0)
    return _case(op, **kw)


# ------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """[(new tokens, tokens in all)] of every sequence."""
    rng = random.Random(case["mix"])
    out = []
    for s in range(case["seqs"]):
        new = _log(rng, case["new_lo"], case["new_hi"]) if s < case["chunks"] else 1
        ctx = rng.randint(case["ctx_lo"], case["ctx_hi"]) if case["ctx_hi"] < 16 else _log(rng, max(1, case["ctx_lo"]), case["ctx_hi"])
        out.append((new, ctx + new))
    return out


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + salt)
    return g


def prepare(case, seed):
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    G, grp, ps, L, S = (case[k] for k in ("kv_heads", "group", "page", "layers", "seqs"))
    H = G * grp
    lens = _lengths(case)
    total = sum(n for n, _ in lens)
    T = total + case["pad"]
    need = [-(-k // ps) for _, k in lens]
    max_pages, n_pages = max(need), sum(need) + 3
    g = _gen(seed, 1)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((S, max_pages), dtype=torch.int32, device="cuda")
    used = 0
    for s, p in enumerate(need):
        table[s, :p] = order[used:used + p]
        used += p
    starts = [0]
    for n, _ in lens:
        starts.append(starts[-1] + n)
    pool = torch.empty((L, n_pages, 2, G, ps, D), dtype=dt, device="cuda")
    for l in range(L):
        pool[l] = torch.randn(pool.shape[1:], generator=g, device="cuda", dtype=torch.float32).to(dt)
        big = torch.rand((n_pages, G, ps, 1), generator=g, device="cuda") < 0.005
        pool[l, :, 0] *= torch.where(big, 4.0, 1.0).to(dt)
    st = {"op": case["op"], "S": S, "G": G, "grp": grp, "ps": ps, "T": T, "total": total, "rot": case["rot"],
          "nmax": max(n for n, _ in lens), "lmax": max(k for _, k in lens), "layer": L - 1, "L": L, "n": case["n"],
          "pool": pool, "table": table, "eps": 1e-6, "dt": dt,
          "row_start": torch.tensor(starts, dtype=torch.int32, device="cuda"),
          "kv_len": torch.tensor([k for _, k in lens], dtype=torch.int32, device="cuda"),
          "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if case["op"] == "append":
        width = (H + 2 * G) * D if case["fused"] else 0
        if width:
            x = torch.randn((T, width), generator=g, device="cuda", dtype=torch.float32).to(dt)
            q, k, v = x.split((H * D, G * D, G * D), dim=1)
        else:
            q, k, v = (torch.randn((T, h * D), generator=g, device="cuda", dtype=torch.float32).to(dt) for h in (H, G, G))
        st.update(q=q.unflatten(1, (H, D)), k=k.unflatten(1, (G, D)), v=v.unflatten(1, (G, D)),
                  q_out=torch.zeros((T, H, D), dtype=dt, device="cuda"), wq=None, wk=None,
                  freq=None if not case["rot"] else
                  500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"]))
        if case["norm"]:
            st["wq"], st["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dt) for _ in range(2))
    elif case["op"] == "attn":
        st.update(q=(2.0 * torch.randn((T, H, D), generator=g, device="cuda")).to(dt),
                  out=torch.zeros((T, H, D), dtype=dt, device="cuda"))
    else:
        first = [_gen_int(seed, s, k - case["n"]) for s, (_, k) in enumerate(lens)]
        st.update(first=torch.tensor(first, dtype=torch.int32, device="cuda"),
                  k_out=torch.zeros((S, L, G, case["n"], D), dtype=dt, device="cuda"),
                  v_out=torch.zeros((S, L, G, case["n"], D), dtype=dt, device="cuda"))
    if own:   # the descriptions and the scratch that a serving program keeps
        from paper_2607_15498_gb300 import varrate as V
        st["V"] = V
        st["pages"] = V.PagedCache.of(pool)
        st["seqs"] = V.SeqBatch.of(st["row_start"], st["kv_len"], table, T)
        if case["op"] == "attn":
            st["ws"] = V.paged_attn_workspace(st["pages"], st["seqs"], grp)
    return st


def _gen_int(seed, salt, most):
    return random.Random(seed * 1000003 + salt).randint(0, most)


# ------------------------------------------------------------------------------------ the operators

def run(st):
    return {"append": _append, "attn": _attn, "gather": _gather}[st["op"]](st)


def _append(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged_append(st["pages"], st["seqs"], st["layer"], st["q"], st["k"], st["v"], st["wq"],
                                       st["wk"], st["eps"], st["freq"], st["rot"], st["q_out"], st["status"]))
    else:
        row = torch.arange(st["total"], device="cuda")
        seq = (row[:, None] >= st["row_start"][None, 1:]).sum(1)
        pos = (st["kv_len"] - st["row_start"][1:])[seq] + row
        page = st["table"][seq, pos // st["ps"]].long()
        cos = sin = None
        if st["rot"]:
            angle = pos[:, None].double() * st["freq"]
            cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        st["q_out"][:st["total"]] = _turn(st, st["q"][:st["total"]], st["wq"], cos, sin)
        st["pool"][st["layer"], page, 0, :, pos % st["ps"]] = _turn(st, st["k"][:st["total"]], st["wk"], cos, sin)
        st["pool"][st["layer"], page, 1, :, pos % st["ps"]] = st["v"][:st["total"]]
    return {"q": st["q_out"], "pool": st["pool"]}


def _turn(st, x, w, cos, sin):
    x, h = x.float(), st["rot"] // 2
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * w.float()
    if h:
        a, b = x[..., :h], x[..., h:2 * h]
        x = torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., 2 * h:]), -1)
    return x.to(st["dt"])


def _attn(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged_attn(st["pages"], st["seqs"], st["layer"], st["grp"], st["q"], st["out"], st["status"],
                                     st["ws"]))
    else:
        S, G, grp, n, ps = (st[k] for k in ("S", "G", "grp", "nmax", "ps"))
        kv = st["pool"][st["layer"]][st["table"].long()]                     # [S][pages][2][G][page][d]
        k, v = (kv[:, :, c].transpose(1, 2).flatten(2, 3).float() for c in (0, 1))
        first = st["row_start"][:-1, None]
        row = first + torch.arange(n, device="cuda")                         # [S][n]
        there = row < st["row_start"][1:, None]
        pos = st["kv_len"][:, None] - st["row_start"][1:, None] + row
        q = st["q"][row.clamp(max=st["T"] - 1).long()].unflatten(2, (G, grp)).permute(0, 2, 1, 3, 4)
        s = q.flatten(2, 3).float() @ k.transpose(2, 3) * (1 / math.sqrt(D))
        later = torch.arange(k.shape[2], device="cuda") > pos.repeat_interleave(grp, 1)[:, None, :, None]
        s.masked_fill_(later, -math.inf)
        s.sub_(s.amax(-1, keepdim=True)).exp_()
        o = (s @ v) / s.sum(-1, keepdim=True)
        o = o.unflatten(2, (n, grp)).permute(0, 2, 1, 3, 4).flatten(2, 3).to(st["dt"])
        st["out"][:st["total"]] = o[there]
    return st["out"]


def _gather(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged_gather(st["pages"], st["seqs"], 0, st["L"], st["first"], st["n"], st["k_out"], st["v_out"],
                                       st["status"]))
    else:
        pos = st["first"][:, None] + torch.arange(st["n"], device="cuda")    # [S][n]
        page = torch.gather(st["table"].long(), 1, (pos // st["ps"]).long())
        x = st["pool"].transpose(0, 1)[page, :, :, :, pos % st["ps"]]        # [S][n][L][2][G][d]
        x = x.permute(3, 0, 2, 4, 1, 5)
        st["k_out"].copy_(x[0])
        st["v_out"].copy_(x[1])
    return {"k": st["k_out"], "v": st["v_out"]}


# ------------------------------------------------------------------------------------ work and exact results

def work(case):
    lens = _lengths(case)
    e = 4 if case["dtype"] == "f32" else 2
    G, H = case["kv_heads"], case["kv_heads"] * case["group"]
    rows = sum(n for n, _ in lens)
    if case["op"] == "append":
        return {"bytes": 2 * rows * (H + 2 * G) * D * e, "flops": rows * (H + G) * ((4 * D if case["norm"] else 0) + 3 * case["rot"])}
    if case["op"] == "attn":
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in lens)
        return {"bytes": 2 * rows * H * D * e + 2 * sum(k for _, k in lens) * G * D * e, "flops": 4 * D * H * pairs}
    return {"bytes": 4 * case["seqs"] * case["layers"] * G * case["n"] * D * e, "flops": 0}


def exact(case, seed):
    """One sequence after another, in 64 bits on the inputs of ``prepare``."""
    st = prepare(case, seed)
    pool, ps, l, G, grp = st["pool"], st["ps"], st["layer"], st["G"], st["grp"]
    start, length, table = st["row_start"].tolist(), st["kv_len"].tolist(), st["table"].long()

    def tokens(s, c, layer, lo, hi):
        """[G][hi - lo][d] of a sequence's keys (c = 0) or values."""
        t = torch.arange(lo, hi, device="cuda")
        return pool[layer, table[s, t // ps], c, :, t % ps].double().transpose(0, 1)

    if case["op"] == "gather":
        out = {"k": st["k_out"].double(), "v": st["v_out"].double()}
        for s, f in enumerate(st["first"].tolist()):
            for layer in range(st["L"]):
                for c, name in enumerate("kv"):
                    out[name][s, layer] = tokens(s, c, layer, f, f + st["n"])
        return out
    if case["op"] == "attn":
        out = st["out"].double()
        for s in range(st["S"]):
            n, total = start[s + 1] - start[s], length[s]
            for g in range(G):
                q = st["q"][start[s]:start[s + 1], g * grp:(g + 1) * grp].double()
                w = torch.einsum("ihd,td->hit", q, tokens(s, 0, l, 0, total)[g]) / math.sqrt(D)
                seen = torch.ones((n, total), dtype=torch.bool, device="cuda").tril(total - n)
                w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
                out[start[s]:start[s + 1], g * grp:(g + 1) * grp] = torch.einsum("hit,td->ihd", w, tokens(s, 1, l, 0, total)[g])
        return out
    q_out, pages, h = st["q_out"].double(), pool.double(), st["rot"] // 2
    for s in range(st["S"]):
        lo, hi = start[s], start[s + 1]
        t = torch.arange(length[s] - (hi - lo), length[s], device="cuda")

        def formed(x, w):
            x = x[lo:hi].double()
            if w is not None:
                x = x * w.double() / (x.pow(2).sum(-1, keepdim=True) / D + st["eps"]).sqrt()
            if h:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), t[:, None] * st["freq"])[:, None]
                z = torch.complex(x[..., :h], x[..., h:2 * h]) * turn
                x = torch.cat((z.real, z.imag, x[..., 2 * h:]), -1)
            return x

        q_out[lo:hi] = formed(st["q"], st["wq"])
        pages[l, table[s, t // ps], 0, :, t % ps] = formed(st["k"], st["wk"])
        pages[l, table[s, t // ps], 1, :, t % ps] = st["v"][lo:hi].double()
    return {"q": q_out, "pool": pages}
