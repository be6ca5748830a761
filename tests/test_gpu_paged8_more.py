"""Paged cache in 8 bits: calls of the kinds that its other tests do not make."""
import pytest
import torch

from paged8_helpers import Batch8, attn8_ref, mass8_ref
from paged_helpers import Batch, close
from paper_2607_15498_gb300 import varrate as V

pytestmark = pytest.mark.gpu


def attn(b, q, ws=None, layer=0):
    out = torch.full((b.T, b.H, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, b.H), float("nan"), device="cuda")
    V.check(V.varrate_paged8_attn(b.pages, b.seqs, layer, b.grp, q, out, lse, b.status, b.workspace() if ws is None else ws))
    return out, lse


@pytest.mark.parametrize("lens, grp", [([(9 + i % 24, 1500 + 37 * i) for i in range(40)], 4), ([(17 + i % 40, 700) for i in range(60)], 2)])
def test_weights_of_many_chunks_of_one_query_tile(lens, grp):
    """Units of a single query tile, many a CTA: their warps run as far apart as they may."""
    b = Batch8(lens, G=8, grp=grp, ps=64)
    b.mass.nan_to_num_(0.5)
    before = b.mass.clone()
    q = b.rows(b.H)
    _, lse = attn(b, q)
    for i in range(300):
        b.mass.copy_(before)
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
        if i == 0:
            first = b.mass.clone()
    assert b.status.item() == 0 and torch.equal(first, b.mass)
    want, tol = mass8_ref(b, q, lse, before)
    close(b.mass, want, tol)


def test_one_workspace_for_every_group_and_cache():
    """A workspace that is large enough serves calls of any shape, also of the uncompressed cache, one after another."""
    kinds = [([(1, 3000)] * 3 + [(40, 700)], 4), ([(150, 3000), (1, 900), (0, 4), (9, 2000)], 3), ([(1, 4000)] * 8, 1),
             ([(200, 900), (2, 3000)], 5), ([(64, 2000), (1, 700)], 8), ([(20, 1500)] + [(0, 5)] * 30, 6), ([(90, 3000)], 2)]
    batches = [Batch8(lens, G=2, grp=grp, ps=64, seed=i) for i, (lens, grp) in enumerate(kinds)]
    plain = [Batch([(1, 3000), (33, 2000)], "bf16", 2, grp, seed=grp) for grp in (4, 3)]
    q = [b.rows(b.H) for b in batches]
    want = [attn(b, x) for b, x in zip(batches, q)]
    for b, x, (out, lse) in zip(batches, q, want):
        o, tol, y, tol_lse = attn8_ref(b, x)
        close(out, o, tol)
        close(lse, y, tol_lse)
    q_plain = [b.rows(b.H) for b in plain]
    ws = torch.zeros(max(b.workspace().numel() for b in batches + plain), dtype=torch.uint8, device="cuda")
    out_plain = [torch.empty_like(x) for x in q_plain]
    want_plain = []
    for b, x, o in zip(plain, q_plain, out_plain):
        V.check(V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, x, o, b.status, b.workspace()))
        want_plain.append(o.clone())
    for order in (range(len(batches)), [3, 0, 1, 4, 0, 3, 6, 2, 5, 1, 0, 4]):
        for n, i in enumerate(order):
            out, lse = attn(batches[i], q[i], ws)
            assert batches[i].status.item() == 0, (i, n)
            assert torch.equal(out.view(torch.int16), want[i][0].view(torch.int16)) and torch.equal(lse, want[i][1]), (i, n)
            j = n % len(plain)
            V.check(V.varrate_paged_attn(plain[j].pages, plain[j].seqs, 0, plain[j].grp, q_plain[j], out_plain[j], plain[j].status, ws))
            assert plain[j].status.item() == 0 and torch.equal(out_plain[j].view(torch.int16), want_plain[j].view(torch.int16))


def set_codes(b, s, u, c, codes):
    """Codes of places u of a sequence (keys 0, values 1; the same for every head): numbers that e4m3 holds."""
    p, i = b.place(s, u)
    b.codes[0, p, c, :, i] = codes[:, None].to(torch.float8_e4m3fn).view(torch.uint8).expand(-1, b.G, -1)


def set_bytes(b, s, u, c, byte):
    p, i = b.place(s, u)
    b.scale[0, p, c, :, i // 16] = byte


# sequences enough that each of their blocks is one unit, and a warp has one step of 16 keys after the other
MANY = 40


@pytest.mark.parametrize("fraction", [0, 1, 2, 3, 5, 8, 13])
def test_scores_a_place_apart_at_2_27(fraction):
    """Scores of 2^27 log2 units and more, where neighbouring numbers of fp32 are 16 apart: each run of 128 keys is a place above
    the one before, so the last 128 keys have all the weight."""
    ctx = 1023
    b = Batch8([(1, ctx)] * MANY, G=16, grp=1, ps=128)
    u = torch.arange(ctx + 1, device="cuda")
    k = torch.zeros((ctx + 1, 128), device="cuda")
    k[:, 0], k[:, 1], k[:, 2] = 448.0, u // 128, fraction
    for s in range(MANY):
        set_codes(b, s, u, 0, k)
        set_bytes(b, s, u, 0, 127)
    q = torch.zeros((MANY, b.H, 128), device="cuda")
    # in the kernel's units 448 * 1.5 * 2^14, 1 a step and 2^-3 a `fraction`, times 16.3: all of it exact but for the last product
    q[..., 0], q[..., 1], q[..., 2] = 1.5 * 2.0 ** 21, 2.0 ** 7, 2.0 ** 4
    out, lse = attn(b, q.bfloat16())
    assert b.status.item() == 0
    top = (448 * 1.5 * 2.0 ** 21 + 7 * 2.0 ** 7 + fraction * 2.0 ** 4) / 128 ** 0.5
    # sum 1, log2 e / sqrt(d) 1.5, product 1, log2 of the sum 1, product 1 half step of 2^-24; log 128 is below one
    assert ((lse.double() - top).abs() <= 8 * 2.0 ** -24 * top).all()
    pool = b.values()
    for s in range(MANY):
        v = b.tokens(s, 1, pool=pool)
        want = v[:, 896:].mean(1)
        # the keys of the run before are at least 16 - 1 below in exact arithmetic and, two roundings apart, no less than a place in
        # fp32: 2^-16 of the weight; the average's sums and the output's rounding
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -15 + 200 * 2.0 ** -24) * v.abs().amax()
        assert ((out[s].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("size", [8.0, 30.0, 300.0])
def test_values_for_large_queries(size):
    """Rows that few tokens decide, for both kernels."""
    b = Batch8([(1, 200), (9, 50), (1, 3000), (70, 300)], G=2, grp=4)
    q = (size * b.rows(b.H).double()).bfloat16()
    out, lse = attn(b, q)
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    assert b.status.item() == 0
    # fp32 ends at 2^-126, and the reference of many rows stands up to 2^40 above the largest weight: what is lighter than 2^-86 of it
    # counts as nothing, less than that of the largest value for each token
    close(out, want, tol + max(b.len) * 2.0 ** -86 * b.values().nan_to_num(0).abs().amax())
    close(lse, want_lse, tol_lse)


@pytest.mark.parametrize("new, ctx, n", [(1, 1200, MANY), (2, 30, 1), (1, 15, 1), (4, 1000, MANY)])
@pytest.mark.parametrize("lighter, up", [(5, 0), (18, 0), (24, 0), (35, 0), (60, 0), (80, 0), (5, 10), (20, 10), (20, 3), (30, 11), (30, 40)])
def test_a_heavy_token_without_a_value(new, ctx, n, lighter, up):
    """As attention sinks have it: the first token has all the weight and a value of zeros, the others 2^-lighter of it; its block's
    scale is 2^up times theirs. What there is comes from the light ones, each with its weight rounded to 16 bits at worst."""
    b = Batch8([(new, ctx)] * n, G=8, grp=4, ps=64, spread=0.0)
    u = torch.arange(new + ctx, device="cuda")
    for s in range(n):
        set_bytes(b, s, u, 0, 120)
        set_bytes(b, s, u, 1, 120)
        p, i = b.place(s, u)
        b.codes[0, p, 0, :, i, 0] = 0                   # no other key has an element 0
        b.codes[0, p[0], 0, :, i[0]] = 0
        b.codes[0, p[0], 0, :, i[0], 0] = 0x7E          # 448
        if n > 1:
            b.codes[0, p[:16], 1, :, i[:16]] = 0        # the first block's values
            b.scale[0, p[0], 1, :, i[0] // 16] = 120 + up
        else:                                           # other tokens of the first step have values as well
            b.codes[0, p[0], 1, :, i[0]] = 0
    q = 0.5 * b.rows(b.H).float()
    q[..., 0] = lighter * 0.6931472 * 128 ** 0.5 / (448 * 2.0 ** -7)
    q = q.bfloat16()
    out, lse = attn(b, q)
    assert b.status.item() == 0
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    assert (want.abs() > 2.0 ** -(lighter + 30)).any()
    close(out, want, tol)
    close(lse, want_lse, tol_lse)


@pytest.mark.parametrize("byte", [1, 2, 3, 4, 9])
@pytest.mark.parametrize("new", [1, 3])
def test_values_of_the_smallest_scales_behind_zeros(new, byte):
    """The first 128 tokens' values are zeros, of scale byte 0; the others' have the smallest scales there are."""
    b = Batch8([(new, 300)] * MANY, G=8, grp=4, ps=64)
    u = torch.arange(300 + new, device="cuda")
    for s in range(MANY):
        set_bytes(b, s, u, 1, byte)
        p, i = b.place(s, u[:128])
        b.codes[0, p, 1, :, i] = 0
        b.scale[0, p, 1, :, i // 16] = 0
    q = b.rows(b.H)
    out, lse = attn(b, q)
    want, tol, _, _ = attn8_ref(b, q)
    assert (want.abs() > 2.0 ** -130).any()
    # half a step of bf16's numbers below 2^-126, and the kernel's sums below it, a rounding a warp
    close(out, want, tol + 2.0 ** -134 + 20 * 2.0 ** -150)


@pytest.mark.parametrize("order", ["rising", "falling", "jumps"])
@pytest.mark.parametrize("size", [20.0, 60.0, 300.0])
def test_scores_that_drift(order, size):
    """Scores that rise or fall by `size` log2 units over the context, or jump by as much from key to key."""
    ctx = 1100
    b = Batch8([(1, ctx)] * MANY + [(2, ctx)], G=8, grp=4, ps=64)
    ramp = torch.linspace(-1, 1, ctx + 2, device="cuda")
    if order == "falling":
        ramp = -ramp
    if order == "jumps":
        ramp = ramp[torch.randperm(ctx + 2, generator=b.gen).cuda()]
    for s in range(MANY + 1):
        u = torch.arange(b.len[s], device="cuda")
        set_bytes(b, s, u, 0, 121)
        p, i = b.place(s, u)
        codes = (448 * ramp[:len(u)]).to(torch.float8_e4m3fn).view(torch.uint8)
        b.codes[0, p, 0, :, i, 0] = codes[:, None].expand(-1, b.G)
    q = 0.5 * b.rows(b.H).float()
    q[..., 0] = 0.5 * size * 0.6931472 * 128 ** 0.5 / (448 * 2.0 ** -6)
    q = q.bfloat16()
    out, lse = attn(b, q)
    assert b.status.item() == 0
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    # weights that fp32 does not hold beside the largest count as nothing (as in the test of large queries)
    close(out, want, tol + max(b.len) * 2.0 ** -86 * b.values().nan_to_num(0).abs().amax())
    close(lse, want_lse, tol_lse)


@pytest.mark.parametrize("new, ctx, at", [(20, 300, 200), (40, 300, 200), (40, 9000, 6000), (20, 9000, 6000), (12, 700, 3), (100, 3000, 2900)])
@pytest.mark.parametrize("first", [True, False])
def test_scores_past_2_24_of_many_rows(new, ctx, at, first):
    """One key has a score of 2^30 log2 units, one far from it 2^23.5: the first has all the weight, wherever the two stand, and is lse."""
    b = Batch8([(new, ctx)], G=1, grp=4, ps=64)
    u = torch.arange(new + ctx, device="cuda")
    k = torch.zeros((new + ctx, 128), device="cuda")
    big, small = (1, at) if first else (at, 1)
    k[big, 0], k[small, 0] = 448.0, 5.0
    set_codes(b, 0, u, 0, k)
    set_bytes(b, 0, u, 0, 127)
    q = torch.zeros((new, 4, 128), device="cuda")
    q[..., 0] = 1.02 * 2.0 ** 30 * 0.6931472 * 128 ** 0.5 / 448
    q = q.bfloat16()
    out, lse = attn(b, q)
    assert b.status.item() == 0
    v = b.tokens(0, 1)[0][big].expand_as(out)
    assert ((out.double() - v).abs() <= (2 * 2.0 ** -8 + 2.0 ** -16) * v.abs()).all()   # the weight and the output in bf16
    top = q[..., 0].double() * 448 / 128 ** 0.5
    # log2 e / sqrt(d) 1.5, product 1, the reference's distance on and off 2, log2 of the sum 1, product 1 half step of 2^-24
    assert ((lse.double() - top).abs() <= 8 * 2.0 ** -24 * top).all()


@pytest.mark.parametrize("new, ctx", [(40, 600), (20, 900), (3, 900)])
@pytest.mark.parametrize("low", [-2.0 ** 30, -2.0 ** 25])
def test_scores_far_below_the_others(new, ctx, low):
    """The first 200 keys' scores are -2^25 or -2^30 log2 units, the others' ordinary: those decide as if they stood alone."""
    b = Batch8([(new, ctx)], G=1, grp=4, ps=64)
    u = torch.arange(new + ctx, device="cuda")
    set_bytes(b, 0, u, 0, 121)
    p, i = b.place(0, u)
    b.codes[0, p, 0, :, i, 0] = 0
    b.codes[0, p[:200], 0, :, i[:200]] = 0
    b.codes[0, p[:200], 0, :, i[:200], 0] = 0xFE        # -448
    q = b.rows(4).float()
    q[..., 0] = -low * 0.6931472 * 128 ** 0.5 / (448 * 2.0 ** -6)
    q = q.bfloat16()
    out, lse = attn(b, q)
    assert b.status.item() == 0
    # the same without the first keys: what is left has the same keys and values, positions do not matter to it
    x = q.clone()
    x[..., 0] = 0
    pool = b.values()
    k, v = (b.tokens(0, c, pool=pool)[0][200:] for c in (0, 1))
    w = torch.einsum("ihd,td->iht", x.double(), k) / 128 ** 0.5
    size = torch.einsum("ihd,td->iht", x.double().abs(), k.abs()) / 128 ** 0.5
    seen = torch.arange(200, new + ctx, device="cuda")[None] <= torch.arange(ctx, ctx + new, device="cuda")[:, None]
    w = w.masked_fill(~seen[:, None], -float("inf"))
    a, y = torch.softmax(w, -1), torch.logsumexp(w, -1)
    # as attn8_ref; the elements beside the large one are fp16 times a power of two, off by 2^-39 of it
    ds = (132 * 2.0 ** -23 * size + 2.0 ** -39 * q[..., :1].abs().double() * k.abs().sum(-1) / 128 ** 0.5).amax(-1, keepdim=True)
    rel = 2 * ds + 2.0 ** -20 + 2 * (new + ctx + 8) * 2.0 ** -24 + 2.0 ** -8
    mass, o = torch.einsum("iht,td->ihd", a, v.abs()), torch.einsum("iht,td->ihd", a, v)
    close(out, o, rel * mass + 2.0 ** -8 * (o.abs() + rel * mass))
    close(lse, y, ds[..., 0] + 2.0 ** -20 + (new + ctx + 8) * 2.0 ** -24 + 4 * 2.0 ** -24 * (1 + y.abs()))


@pytest.mark.parametrize("call", ["attn", "mass"])
def test_a_chunk_among_empty_slots_takes_no_longer(call):
    """60 new tokens on 32768 of one sequence beside 63 that have nothing new: the time of the chunk alone, or a little more."""
    times, outs = [], []
    for slots in (1, 64):
        b = Batch8([(60, 300)] + [(0, 40)] * (slots - 1), G=8, grp=4, ps=64)
        n, pages = 32768, 32768 // 64
        gen = torch.Generator(device="cuda").manual_seed(3)
        codes = torch.randint(0, 0x60, (1, pages, 2, 8, 64, 128), generator=gen, dtype=torch.uint8, device="cuda")
        scale = torch.full((1, pages, 2, 8, 4), 122, dtype=torch.uint8, device="cuda")
        table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(slots, pages).contiguous()
        length = torch.tensor([n] + [40] * (slots - 1), dtype=torch.int32, device="cuda")
        cache = V.Paged8Cache.of(codes, scale, torch.zeros((1, pages, 8, 64), device="cuda"))
        seqs = V.SeqBatch.of(b.row_start, length, table, 60)
        q = torch.randn((60, 32, 128), generator=gen, device="cuda").bfloat16()
        out, lse, ws = torch.empty_like(q), torch.empty((60, 32), device="cuda"), V.paged8_attn_workspace(cache, seqs, 4)

        def run():
            if call == "attn":
                V.check(V.varrate_paged8_attn(cache, seqs, 0, 4, q, out, lse, b.status, ws))
            else:
                V.check(V.varrate_paged8_mass(cache, seqs, 0, 4, q, lse, b.status))

        V.check(V.varrate_paged8_attn(cache, seqs, 0, 4, q, out, lse, b.status, ws))
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = float("inf")
        for _ in range(8):
            start.record()
            for _ in range(10):
                run()
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        assert b.status.item() == 0
        times.append(best)
        outs.append((out, lse))
    assert times[1] < 2 * times[0], times               # (6 to 7 times where every row is one of the kernel of few)
    assert (outs[0][0].float() - outs[1][0].float()).abs().max() <= 2.0 ** -6 * outs[0][0].abs().max()
