"""Performance cases of the paged cache in 8 bits: append, attention, attention weight per token, eviction.

Keys and values stand in pages as e4m3 codes with one power of two for each block of 16 tokens of a head,
``codes [layers][pages][2][kv_heads][page][128]`` and ``scale [layers][pages][2][kv_heads][page / 16]`` (0: keys,
1: values), an element being code times scale; ``mass [layers][pages][kv_heads][page]`` holds the attention weight that
each cached token has had. A batch is described by ``row_start [seqs + 1]`` (rows of each sequence's new tokens),
``kv_len [seqs]`` (tokens of a sequence, the new ones included) and ``table [seqs][pages of a sequence]``. Four
operators, each through the public entry points of ``paper_2607_15498_gb300.varrate``:

* ``append``  varrate_paged8_append: norm of every query and key head (where the model has one), position rotation,
              queries out, keys and values as codes into their pages; a block that holds older tokens gets a scale that
              is enough for all of it.
* ``attn``    varrate_paged8_attn: causal attention of the new tokens over the pages, with the logarithm of each row's sum.
* ``mass``    varrate_paged8_mass: the weights that the new tokens give to every cached token, added up over the new
              tokens and the query heads of a KV head.
* ``evict``   varrate_paged8_evict: per layer and KV head the first and the last tokens of a sequence and those of the
              others with most weight are kept and move together, up to a budget.

The first ``chunks`` sequences bring ``new_lo`` to ``new_hi`` new tokens, the others one; each has ``ctx_lo`` to
``ctx_hi`` tokens before them. These lengths are drawn from ``mix``, so they belong to the case. ``pad`` rows stand
behind the last sequence's, as in a batch that is padded to a captured size. Queries and keys have logits of a few units
and a share of keys of 4 times the size; heads and tokens differ in size, so that neighbouring blocks have other scales.
"""
import math
import random

import torch

own = False

D = 128
BLOCK = 16
OPS = ("append", "attn", "mass", "evict")


def _case(op, **kw):
    c = {"op": op, "kv_heads": 8, "group": 4, "page": 64, "layers": 1, "seqs": 1, "chunks": 0, "new_lo": 1, "new_hi": 1,
         "ctx_lo": 0, "ctx_hi": 0, "pad": 0, "norm": False, "rot": 128, "fused": True, "gone": False, "budget": 0,
         "first": 0, "last": 0, "mix": 1}
    c.update(kw)
    return c


def listed():
    return [
        # one decode step of eight sequences, one layer: latency
        dict(_case("append", seqs=8, ctx_lo=2000, ctx_hi=8000), name="append8_step_batch8"),
        # an 8192-token prompt in one piece, keys and values straight out of the joint projection
        dict(_case("append", chunks=1, new_lo=8192, new_hi=8192), name="append8_prompt_8k"),
        # chunks of many lengths of sequences that lost tokens before, group 7, head norms, half of each head rotated, a padded batch
        dict(_case("append", kv_heads=4, group=7, seqs=24, chunks=23, new_lo=30, new_hi=900, ctx_lo=100, ctx_hi=2000, norm=True, rot=64, page=16, pad=37, gone=True), name="append8_chunks_ragged"),
        # one token of one short sequence: latency
        dict(_case("attn", ctx_lo=899, ctx_hi=899), name="attn8_step_short"),
        # one decode step of eight 32k sequences: bandwidth
        dict(_case("attn", seqs=8, ctx_lo=32767, ctx_hi=32767), name="attn8_step_batch8_32k"),
        # a serving step of group 7: a chunk of one prompt beside the single tokens of running sequences
        dict(_case("attn", kv_heads=4, group=7, seqs=24, chunks=1, new_lo=383, new_hi=383, ctx_lo=60, ctx_hi=7800, page=16, pad=11), name="attn8_mixed_step"),
        # an 8192-token prompt in one piece: tensor cores
        dict(_case("attn", chunks=1, new_lo=8192, new_hi=8192), name="attn8_prompt_8k"),
        # the weights of one decode step of eight 32k sequences: bandwidth
        dict(_case("mass", seqs=8, ctx_lo=32767, ctx_hi=32767), name="mass8_step_batch8_32k"),
        # the weights that the last 512 tokens of a 131072-token context give
        dict(_case("mass", chunks=1, new_lo=512, new_hi=512, ctx_lo=130560, ctx_hi=130560, page=128), name="mass8_chunk_131k"),
        # one layer of a few short sequences back to 1024 tokens: latency
        dict(_case("evict", seqs=4, ctx_lo=900, ctx_hi=1500, budget=1024, first=4, last=256), name="evict8_short_batch4"),
        # one layer of a 131072-token context down to half of it
        dict(_case("evict", ctx_lo=131071, ctx_hi=131071, page=128, budget=65536, first=16, last=4096), name="evict8_131k"),
        # four layers of eight sequences of many lengths down to 12288 tokens
        dict(_case("evict", layers=4, seqs=8, ctx_lo=9000, ctx_hi=32000, budget=12288, first=4, last=1024), name="evict8_layers_ragged"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(OPS)
    G, grp = rng.randint(1, 8), rng.randint(1, 8)
    kw = dict(kv_heads=G, group=grp, page=rng.choice([16, 32, 64, 128, 256]), mix=rng.randint(1, 1 << 20),
              pad=rng.choice([0, 0, rng.randint(1, 40)]))
    if op == "append":
        seqs = _log(rng, 1, 64)
        rows = _log(rng, seqs, 8192)                              # new rows in all, at most
        kw.update(seqs=seqs, chunks=rng.choice([seqs, max(0, seqs - 1)]), new_lo=1, new_hi=max(2, rows // seqs), ctx_lo=0,
                  ctx_hi=_log(rng, 16, max(17, min(8000, (1 << 18) // seqs))), norm=rng.random() < 0.5,
                  rot=rng.choice([128, 128, 64, 32, 0]), fused=rng.random() < 0.5, gone=rng.random() < 0.3)
    elif op in ("attn", "mass"):
        seqs, room = _log(rng, 1, 64), 1 << 31
        # a padded batch holds no more (query, key, head) triples than the largest listed prompt, 8192 x 8192 x 32
        new = rng.choice([1, _log(rng, 2, 8192)])
        new = max(1, min(new, math.isqrt(room // (seqs * G * grp))))
        most = min(131072, room // (seqs * G * grp * new), (1 << 21) // (seqs * G))
        new = min(new, most)
        ctx = _log(rng, max(16, new), max(17, most))
        kw.update(seqs=seqs, chunks=rng.randint(1, seqs) if new > 1 else 0, new_lo=max(1, new // 3), new_hi=new,
                  ctx_lo=max(0, (ctx - new) // 50), ctx_hi=max(0, ctx - new))
    else:
        seqs, layers = _log(rng, 1, 16), _log(rng, 1, 8)
        most = max(32, min(131072, (1 << 22) // (seqs * layers * G)))
        ctx = _log(rng, 20, most)
        budget = rng.randint(1, ctx)
        first = rng.choice([0, rng.randint(0, min(64, budget))])
        kw.update(seqs=seqs, layers=layers, ctx_lo=max(1, ctx // 3), ctx_hi=ctx, budget=budget, first=first,
                  last=rng.choice([0, rng.randint(0, budget - first)]), pad=0)
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


def _exponent(amax):
    """The scale byte of a block whose largest element is amax: 2^(byte - 127) times 448 is the first not below it."""
    m, x = torch.frexp(amax)
    return torch.where(amax == 0, 0, (x - 9 + (m > 0.875) + 127).clamp(1, 246))


def _codes(x, byte):
    """x / 2^(byte - 127) as e4m3."""
    return (x * torch.exp2(127.0 - byte.float())).clamp(-448, 448).to(torch.float8_e4m3fn)


def prepare(case, seed):
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
    codes = torch.empty((L, n_pages, 2, G, ps, D), dtype=torch.uint8, device="cuda")
    scale = torch.empty((L, n_pages, 2, G, ps // BLOCK), dtype=torch.uint8, device="cuda")
    for l in range(L):
        for c in range(2):
            x = torch.randn((n_pages, G, ps // BLOCK, BLOCK, D), generator=g, device="cuda")
            if c == 0:
                x *= torch.where(torch.rand((n_pages, G, ps // BLOCK, BLOCK, 1), generator=g, device="cuda") < 0.005, 4.0, 1.0)
            else:
                x *= torch.exp2(torch.randn((n_pages, G, ps // BLOCK, 1, 1), generator=g, device="cuda"))
            byte = _exponent(x.abs().amax((-1, -2)))
            scale[l, :, c] = byte.to(torch.uint8)
            codes[l, :, c] = _codes(x, byte[..., None, None]).view(torch.uint8).flatten(2, 3)
    # weight so far: a few tokens have most of it, some have none
    mass = torch.rand((L, n_pages, G, ps), generator=g, device="cuda")
    mass = torch.where(mass < 0.05, 0.0, (mass - 0.05) ** 6 * 100)
    st = {"op": case["op"], "S": S, "G": G, "grp": grp, "ps": ps, "T": T, "total": total, "rot": case["rot"],
          "nmax": max(n for n, _ in lens), "tokens": sum(k for _, k in lens), "layer": L - 1, "L": L,
          "codes": codes.view(torch.float8_e4m3fn), "scale": scale.view(torch.float8_e8m0fnu), "mass": mass, "table": table, "eps": 1e-6,
          "budget": case["budget"], "first": case["first"], "last": case["last"], "gone": None,
          "row_start": torch.tensor(starts, dtype=torch.int32, device="cuda"),
          "kv_len": torch.tensor([k for _, k in lens], dtype=torch.int32, device="cuda"),
          "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if case["op"] == "append":
        width = (H + 2 * G) * D if case["fused"] else 0
        if width:
            x = torch.randn((T, width), generator=g, device="cuda", dtype=torch.float32).bfloat16()
            q, k, v = x.split((H * D, G * D, G * D), dim=1)
        else:
            q, k, v = (torch.randn((T, h * D), generator=g, device="cuda", dtype=torch.float32).bfloat16() for h in (H, G, G))
        st.update(q=q.unflatten(1, (H, D)), k=k.unflatten(1, (G, D)), v=v.unflatten(1, (G, D)),
                  q_out=torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda"), wq=None, wk=None,
                  freq=None if not case["rot"] else
                  500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") / case["rot"]))
        if case["norm"]:
            st["wq"], st["wk"] = ((1 + 0.2 * torch.randn(D, generator=g, device="cuda")).bfloat16() for _ in range(2))
        if case["gone"]:
            st["gone"] = torch.randint(0, 100000, (S,), generator=g, device="cuda", dtype=torch.int32)
    elif case["op"] == "attn":
        st.update(q=(2.0 * torch.randn((T, H, D), generator=g, device="cuda")).bfloat16(),
                  out=torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.zeros((T, H), dtype=torch.float32, device="cuda"))
    elif case["op"] == "mass":
        st.update(q=(2.0 * torch.randn((T, H, D), generator=g, device="cuda")).bfloat16(),
                  lse=torch.zeros((T, H), dtype=torch.float32, device="cuda"))
        s, there = _scores(st)
        st["lse"][:total] = torch.logsumexp(s, -1).unflatten(2, (st["nmax"], grp)).permute(0, 2, 1, 3).flatten(2, 3)[there]
    else:
        st.update(kept=torch.zeros((S, L, G, case["budget"]), dtype=torch.int32, device="cuda"),
                  new_len=torch.zeros(S, dtype=torch.int32, device="cuda"))
    if own:   # the descriptions and the scratch that a serving program keeps
        from paper_2607_15498_gb300 import varrate as V
        st["V"] = V
        st["pages"] = V.Paged8Cache.of(st["codes"], st["scale"], mass)
        st["seqs"] = V.SeqBatch.of(st["row_start"], st["kv_len"], table, T)
        if case["op"] == "attn":
            st["ws"] = V.paged8_attn_workspace(st["pages"], st["seqs"], grp)
    return st


# ------------------------------------------------------------------------------------ the operators

def run(st):
    return {"append": _append, "attn": _attn, "mass": _mass, "evict": _evict}[st["op"]](st)


def _append(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged8_append(st["pages"], st["seqs"], st["layer"], st["q"], st["k"], st["v"], st["wq"], st["wk"],
                                        st["eps"], st["freq"], st["rot"], st["gone"], st["q_out"], st["status"]))
    else:
        l, ps, n = st["layer"], st["ps"], st["total"]
        row = torch.arange(n, device="cuda")
        seq = (row[:, None] >= st["row_start"][None, 1:]).sum(1)
        at = (st["kv_len"] - st["row_start"][1:])[seq] + row                 # place in the sequence
        page, block = st["table"][seq, at // ps].long(), at % ps // BLOCK
        cos = sin = None
        if st["rot"]:
            pos = at if st["gone"] is None else at + st["gone"][seq]
            angle = pos[:, None].double() * st["freq"]
            cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        st["q_out"][:n] = _turn(st, st["q"][:n], st["wq"], cos, sin).bfloat16()
        x = torch.stack((_turn(st, st["k"][:n], st["wk"], cos, sin), st["v"][:n].float()), 1)   # [rows][2][G][d]
        # scales: of the new tokens, and where a block holds older ones also theirs
        nb = ps // BLOCK
        scale, codes = st["scale"].view(torch.uint8)[l], st["codes"].view(torch.uint8)[l]
        fresh = torch.zeros((scale.shape[0] * nb, 2, st["G"]), dtype=torch.int32, device="cuda")
        where = page * nb + block
        fresh.index_reduce_(0, where, _exponent(x.abs().amax(-1)).int(), "amax")
        start = (st["kv_len"] - st["row_start"][1:] + st["row_start"][:-1]).long()   # a sequence's first new token
        page0 = torch.gather(st["table"].long(), 1, (start // ps)[:, None])[:, 0]
        block0, old = start % ps // BLOCK, start % BLOCK
        before = scale[page0, :, :, block0].int()                            # [S][2][G]
        fresh.index_reduce_(0, page0 * nb + block0, before * (old > 0)[:, None, None], "amax")
        after = fresh[page0 * nb + block0]
        slot = block0[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")  # [S][16]
        held = codes[page0[:, None], :, :, slot]                             # [S][16][2][G][d]
        moved = held.view(torch.float8_e4m3fn).float() * torch.exp2((before - after).float())[:, None, :, :, None]
        keep = (torch.arange(BLOCK, device="cuda") >= old[:, None])[..., None, None, None]
        codes[page0[:, None], :, :, slot] = torch.where(keep, held, moved.to(torch.float8_e4m3fn).view(torch.uint8))
        scale[page, :, :, block] = fresh[where].to(torch.uint8)
        codes[page, :, :, at % ps] = _codes(x, fresh[where][..., None]).view(torch.uint8)
        st["mass"][l][page, :, at % ps] = 0
    return {"q": st["q_out"], "codes": st["codes"], "scale": st["scale"], "mass": st["mass"]}


def _turn(st, x, w, cos, sin):
    x, h = x.float(), st["rot"] // 2
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * w.float()
    if h:
        a, b = x[..., :h], x[..., h:2 * h]
        x = torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., 2 * h:]), -1)
    return x


def _tokens(st, c):
    """[S][G][tokens][d], 32 bits: the keys (c = 0) or values of every sequence."""
    pages = st["table"].long()
    x = st["codes"].view(torch.uint8)[st["layer"], :, c][pages].view(torch.float8_e4m3fn).float()   # [S][pages][G][page][d]
    f = torch.exp2(st["scale"].view(torch.uint8)[st["layer"], :, c][pages].float() - 127)
    x = x.unflatten(3, (-1, BLOCK)).mul_(f[..., None, None])
    return x.flatten(3, 4).transpose(1, 2).flatten(2, 3)


def _scores(st):
    """[S][G][new tokens x group][tokens], -infinity where a row does not see a token, and which rows [S][new tokens] there are."""
    G, grp, n = st["G"], st["grp"], st["nmax"]
    k = _tokens(st, 0)
    row = st["row_start"][:-1, None] + torch.arange(n, device="cuda")        # [S][n]
    there = row < st["row_start"][1:, None]
    pos = st["kv_len"][:, None] - st["row_start"][1:, None] + row
    q = st["q"][row.clamp(max=st["T"] - 1).long()].unflatten(2, (G, grp)).permute(0, 2, 1, 3, 4)
    s = q.flatten(2, 3).float() @ k.transpose(2, 3) * (1 / math.sqrt(D))
    s.masked_fill_(torch.arange(k.shape[2], device="cuda") > pos.repeat_interleave(grp, 1)[:, None, :, None], -math.inf)
    return s, there


def _rows(st, x, there):
    """x [S][G][new tokens x group][...] as rows [T][H][...]."""
    return x.unflatten(2, (st["nmax"], st["grp"])).transpose(1, 2).flatten(2, 3)[there]


def _attn(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged8_attn(st["pages"], st["seqs"], st["layer"], st["grp"], st["q"], st["out"], st["lse"],
                                      st["status"], st["ws"]))
    else:
        s, there = _scores(st)
        top = s.amax(-1, keepdim=True)
        s.sub_(top).exp_()
        total = s.sum(-1, keepdim=True)
        st["out"][:st["total"]] = _rows(st, (s @ _tokens(st, 1)) / total, there).bfloat16()
        st["lse"][:st["total"]] = _rows(st, (top + total.log())[..., 0], there)
    return {"out": st["out"], "lse": st["lse"]}


def _mass(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged8_mass(st["pages"], st["seqs"], st["layer"], st["grp"], st["q"], st["lse"], st["status"]))
    else:
        s, there = _scores(st)
        row = (st["row_start"][:-1, None] + torch.arange(st["nmax"], device="cuda")).clamp(max=st["T"] - 1).long()
        lse = st["lse"][row].masked_fill(~there[..., None], math.inf)        # [S][n][H]
        lse = lse.unflatten(2, (st["G"], st["grp"])).transpose(1, 2).flatten(2, 3)
        w = s.sub_(lse[..., None]).exp_().sum(2)                             # [S][G][tokens]
        seq = torch.repeat_interleave(torch.arange(st["S"], device="cuda"), st["kv_len"], output_size=st["tokens"])
        at = torch.arange(st["tokens"], device="cuda") - (st["kv_len"].cumsum(0) - st["kv_len"])[seq]
        page = st["table"][seq, at // st["ps"]].long()
        st["mass"][st["layer"]][page, :, at % st["ps"]] += w[seq, :, at]
    return st["mass"]


def _evict(st):
    if own:
        V = st["V"]
        V.check(V.varrate_paged8_evict(st["pages"], st["seqs"], 0, st["L"], st["budget"], st["first"], st["last"],
                                       st["kept"], st["new_len"], None, st["status"]))
    else:
        ps, G, b = st["ps"], st["G"], st["budget"]
        pages, n = st["table"].long(), st["kv_len"].long()[:, None, None, None]
        at = torch.arange(pages.shape[1] * ps, device="cuda")
        mass = st["mass"][:, pages].permute(1, 0, 3, 2, 4).flatten(3, 4)     # [S][L][G][tokens]
        always = (at < st["first"]) | (at >= n - st["last"])
        rank = torch.where(at >= n, -1.0, torch.where(always, math.inf, mass))
        best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :b]
        best = torch.where(torch.arange(best.shape[-1], device="cuda") < n, best, at.numel())
        best = torch.nn.functional.pad(best, (0, b - best.shape[-1]), value=at.numel()).sort(-1).values
        st["kept"].copy_(torch.where(best < at.numel(), best, -1))
        st["new_len"].copy_(st["kv_len"].clamp(max=b))
        # from where each kept token moves to where; entries past the new length repeat the first token's move
        ok = best < at.numel()
        src, to = (torch.where(ok, x, best[..., :1]) for x in (best, torch.arange(b, device="cuda")))
        to = torch.where(ok, to, 0)
        s, l, g = (torch.arange(m, device="cuda").view([-1 if i == d else 1 for i in range(4)]).expand(best.shape)
                   for d, m in enumerate(best.shape[:3]))
        src_page, to_page = pages[s, src // ps], pages[s, to // ps]
        codes, scale, mass = st["codes"].view(torch.uint8), st["scale"].view(torch.uint8), st["mass"]
        for c in range(2):
            byte = scale[l, src_page, c, g, src % ps // BLOCK].int()
            wide = torch.nn.functional.pad(byte * ok, (0, -b % BLOCK)).unflatten(-1, (-1, BLOCK)).amax(-1)
            wide = torch.gather(wide, -1, to // BLOCK)
            x = codes[l, src_page, c, g, src % ps].view(torch.float8_e4m3fn).float()
            x = x * torch.exp2((byte - wide).float())[..., None]
            codes[l, to_page, c, g, to % ps] = x.to(torch.float8_e4m3fn).view(torch.uint8)
            scale[l, to_page, c, g, to % ps // BLOCK] = wide.to(torch.uint8)
        mass[l, to_page, g, to % ps] = mass[l, src_page, g, src % ps]
    return {"codes": st["codes"], "scale": st["scale"], "mass": st["mass"], "kept": st["kept"], "new_len": st["new_len"]}



# ------------------------------------------------------------------------------------ work and exact results

def work(case):
    lens = _lengths(case)
    G, H = case["kv_heads"], case["kv_heads"] * case["group"]
    rows, tokens = sum(n for n, _ in lens), sum(k for _, k in lens)
    code = D + 1 / BLOCK                                          # a token's codes and its share of a scale
    if case["op"] == "append":
        return {"bytes": 2 * rows * (2 * H + 2 * G) * D + rows * G * (2 * code + 4),
                "flops": rows * ((H + G) * ((4 * D if case["norm"] else 0) + 3 * case["rot"]) + 4 * G * D)}
    if case["op"] == "evict":
        kept = sum(min(case["budget"], k) for n, k in lens if k > case["budget"])
        seen = sum(k for n, k in lens if k > case["budget"])
        listed_ = case["seqs"] * case["budget"]
        return {"bytes": case["layers"] * G * (4 * seen + kept * (4 * code + 4) + 4 * listed_), "flops": 0}
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in lens)
    if case["op"] == "attn":
        return {"bytes": rows * H * (4 * D + 4) + 2 * tokens * G * code, "flops": 4 * D * H * pairs}
    return {"bytes": rows * H * (2 * D + 4) + tokens * G * (code + 8), "flops": 2 * D * H * pairs}


def _round8(x):
    """64-bit numbers of at most 448 in absolute value to the nearest e4m3 number, ties to even."""
    step = torch.exp2(torch.frexp(x).exponent.clamp(min=-5).double() - 4)
    return torch.round(x / step) * step


def exact(case, seed):
    """One sequence after another, in 64 bits on the inputs of ``prepare``."""
    st = prepare(case, seed)
    ps, layer, G, grp = st["ps"], st["layer"], st["G"], st["grp"]
    start, length, table = st["row_start"].tolist(), st["kv_len"].tolist(), st["table"].long()
    codes, factor = st["codes"].double(), st["scale"].double()

    def place(s, t):
        return table[s, t // ps], t % ps

    def tokens(s, c, g):
        """[tokens][d] of a sequence's keys (c = 0) or values of one head."""
        p, i = place(s, torch.arange(length[s], device="cuda"))
        return codes[layer, p, c, g, i] * factor[layer, p, c, g, i // BLOCK][:, None]

    def logits(s, g):
        """[new tokens][group][tokens], -infinity where a token is not seen."""
        n, total = start[s + 1] - start[s], length[s]
        q = st["q"][start[s]:start[s + 1], g * grp:(g + 1) * grp].double()
        w = torch.einsum("ihd,td->iht", q, tokens(s, 0, g)) / math.sqrt(D)
        seen = torch.ones((n, total), dtype=torch.bool, device="cuda").tril(total - n)
        return w.masked_fill(~seen[:, None], -math.inf)

    if case["op"] == "attn":
        out, lse = st["out"].double(), st["lse"].double()
        for s in range(st["S"]):
            for g in range(G):
                w, rows, heads = logits(s, g), slice(start[s], start[s + 1]), slice(g * grp, (g + 1) * grp)
                lse[rows, heads] = torch.logsumexp(w, -1)
                out[rows, heads] = torch.einsum("iht,td->ihd", torch.softmax(w, -1), tokens(s, 1, g))
        return {"out": out, "lse": lse}
    mass = st["mass"].double()
    if case["op"] == "mass":
        for s in range(st["S"]):
            p, i = place(s, torch.arange(length[s], device="cuda"))
            for g in range(G):
                lse = st["lse"][start[s]:start[s + 1], g * grp:(g + 1) * grp].double()
                mass[layer, p, g, i] += torch.exp(logits(s, g) - lse[..., None]).sum((0, 1))
        return mass
    if case["op"] == "evict":
        b, kept = case["budget"], torch.full_like(st["kept"], -1)
        for s, n in enumerate(length):
            for l in range(st["L"]):
                for g in range(G):
                    new = torch.arange(min(n, b), device="cuda")
                    src = new
                    if n > b:
                        lo, hi = case["first"], n - case["last"]
                        p, i = place(s, torch.arange(lo, hi, device="cuda"))
                        by = torch.sort(st["mass"][l, p, g, i], dim=-1, descending=True, stable=True).indices
                        some = lo + by[:b - lo - case["last"]].sort().values
                        src = torch.cat((torch.arange(lo, device="cuda"), some, torch.arange(hi, n, device="cuda")))
                    kept[s, l, g, :len(src)] = src
                    (p, i), (q, j) = place(s, src), place(s, new)
                    mass[l, q, g, j] = mass[l, p, g, i]
                    for c in range(2):
                        f = factor[l, p, c, g, i // BLOCK]
                        most = torch.zeros(-(-len(src) // BLOCK), dtype=torch.float64, device="cuda")
                        most = most.scatter_reduce(0, new // BLOCK, f, "amax")[new // BLOCK]
                        codes[l, q, c, g, j] = _round8(codes[l, p, c, g, i] * (f / most)[:, None])
                        factor[l, q, c, g, j // BLOCK] = most
        return {"codes": codes, "scale": factor, "mass": mass, "kept": kept, "new_len": st["kv_len"].clamp(max=b)}
    q_out, h, gone = st["q_out"].double(), st["rot"] // 2, st["gone"].tolist() if st["gone"] is not None else [0] * st["S"]
    for s in range(st["S"]):
        lo, hi, first = start[s], start[s + 1], length[s] - (start[s + 1] - start[s])
        t = torch.arange(first, length[s], device="cuda")

        def formed(x, w):
            x = x[lo:hi].double()
            if w is not None:
                x = x * w.double() / (x.pow(2).sum(-1, keepdim=True) / D + st["eps"]).sqrt()
            if h:
                turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (t + gone[s])[:, None] * st["freq"])[:, None]
                z = torch.complex(x[..., :h], x[..., h:2 * h]) * turn
                x = torch.cat((z.real, z.imag, x[..., 2 * h:]), -1)
            return x

        q_out[lo:hi] = formed(st["q"], st["wq"])
        x = torch.stack((formed(st["k"], st["wk"]), st["v"][lo:hi].double()))        # [2][new][G][d]
        p, i = place(s, t)
        mass[layer, p, :, i] = 0
        for block in range(first // BLOCK, -(-length[s] // BLOCK)):
            a, z = max(first, block * BLOCK), min(length[s], (block + 1) * BLOCK)
            page, at = int(table[s, block * BLOCK // ps]), block * BLOCK % ps
            new, old = x[:, a - first:z - first].transpose(1, 2), a - block * BLOCK      # [2][G][tokens][d]
            most = new.abs().amax((-1, -2))
            e = torch.ceil(torch.log2(most / 448))
            e = e + (most > 448 * torch.exp2(e)).double() - (most <= 448 * torch.exp2(e - 1)).double()
            f = torch.exp2(e.clamp(-126, 119))
            before = factor[layer, page, :, :, at // BLOCK].clone()
            if old:
                f = torch.maximum(f, before)
                held = codes[layer, page, :, :, at:at + old]
                codes[layer, page, :, :, at:at + old] = _round8(held * (before / f)[..., None, None])
            factor[layer, page, :, :, at // BLOCK] = f
            codes[layer, page, :, :, at + old:at + z - block * BLOCK] = _round8(new / f[..., None, None])
    return {"q": q_out, "codes": codes, "scale": factor, "mass": mass}
