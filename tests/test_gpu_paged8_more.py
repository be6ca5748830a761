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
