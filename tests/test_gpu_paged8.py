"""Paged cache in 8 bits on the GPU against the formulas in 64 bits: append, attention, weights, eviction."""
import pytest
import torch

from paged8_helpers import BLOCK, Batch8, append8_check, attn8_ref, evict8_ref, mass8_ref
from paged_helpers import D, close
from paper_2607_15498_gb300 import varrate as V

pytestmark = pytest.mark.gpu


def freqs(rot, device="cuda"):
    return None if rot == 0 else 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)


def run_append(b, q=True, norm=False, rot=128, gone=None, layer=0, k=None, v=None, fused=None, eps=1e-6):
    q = b.rows(b.H, fused) if q else None
    k = b.rows(b.G, fused) if k is None else k
    v = b.rows(b.G, fused) if v is None else v
    wq, wk = ((1 + 0.2 * b.randn(D)).bfloat16().cuda() for _ in range(2)) if norm else (None, None)
    g = None if gone is None else torch.tensor(gone, dtype=torch.int32, device="cuda")
    out = None if q is None else torch.full((b.T, b.H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    before = b.codes.clone(), b.scale.clone(), b.mass.clone()
    f = freqs(rot)
    V.check(V.varrate_paged8_append(b.pages, b.seqs, layer, q, k, v, wq, wk, eps, f, rot, g, out, b.status))
    torch.cuda.synchronize()
    assert b.status.item() == 0
    append8_check(b, (q, k, v, wq, wk, eps, f, rot, gone), layer, before, out)
    if q is not None:                                   # rows of no sequence are left alone
        assert torch.isnan(out[:b.start[0]]).all() and torch.isnan(out[b.start[-1]:]).all()


@pytest.mark.parametrize("kw, ap", [
    (dict(lens=[(1, 0)]), dict()),
    (dict(lens=[(1, 0), (1, 7), (1, 15), (1, 16), (1, 31)], ps=16), dict(norm=True)),
    (dict(lens=[(40, 0), (0, 9), (17, 13), (1, 100), (3, 46)], G=3, grp=7, ps=32, pad=5, lead=2), dict(norm=True, rot=64, gone=[0, 5, 100000, 1, 2 ** 31 - 200])),
    (dict(lens=[(300, 5)], G=1, grp=1, ps=256), dict(rot=0, fused=2)),
    (dict(lens=[(33, 2)] * 3, G=8, grp=8, ps=64, layers=2), dict(rot=32, layer=1, fused=6)),
    (dict(lens=[(20, 20)], G=2, grp=5), dict(q=False, norm=True)),
    (dict(lens=[(2, k) for k in range(40)], G=1, grp=2, ps=16), dict()),
    (dict(lens=[(5000, 11)], G=1, grp=1, ps=128), dict(norm=True))])
def test_append(kw, ap):
    run_append(Batch8(**kw), **ap)


def test_append_of_nan_infinities_zeros_and_extremes():
    b = Batch8([(20, 6), (16, 0), (5, 0), (18, 0)], G=2, grp=1, ps=16)
    k, v = b.rows(2), b.rows(2)
    v[3, 0, 5], v[4, 0, 6], v[4, 1, 7] = float("nan"), float("inf"), -float("inf")
    v[20:36, 0] = 0                                     # a block of zeros
    v[36:41] *= 3e38 / v[36:41].abs().max()             # above what a scale holds
    v[41:57, 0] = 1e-40
    k[41:57, 1] = 2.0 ** -133
    run_append(b, q=False, k=k, v=v, rot=0)
    assert b.scale.view(torch.uint8).max() <= 246
    p, i = b.place(1, torch.arange(16, device="cuda"))
    assert (b.scale[0, p, 1, 0, i // BLOCK] == 0).all() and (b.codes[0, p, 1, 0, i] == 0).all()


def test_a_block_grows_token_by_token():
    """The scale of a block is enough for its largest token so far, and older codes come down with it."""
    b = Batch8([(1, 0)], G=2, grp=1, ps=32)
    for n in range(1, 33):
        b.lens, b.len, b.start, b.T = [(1, n - 1)], [n], [0, 1], 1
        b.kv_len.fill_(n)
        b.table_host = b.table.cpu()
        b.table_host[0, 0] = 1
        b.table.copy_(b.table_host)
        k, v = ((2.0 ** ((n * 7) % 11 - 5)) * b.rows(2) for _ in range(2))
        run_append(b, q=False, k=k.bfloat16(), v=v.bfloat16(), rot=128)


ATTN = [
    dict(lens=[(1, 0)]),
    dict(lens=[(1, c) for c in (0, 1, 14, 15, 16, 17, 127, 128, 129, 1000)], ps=16),
    dict(lens=[(1, 4000), (0, 70), (1, 130)], G=4, grp=8, ps=64, pad=3, lead=1),
    dict(lens=[(2, 30), (3, 200), (9, 64), (17, 5), (1, 300)], G=2, grp=7, ps=32, pad=2),
    dict(lens=[(1, 9000)], G=1, grp=1, ps=256),
    dict(lens=[(130, 0), (1, 5), (70, 61)], G=2, grp=3, ps=128),
    dict(lens=[(300, 700)], G=1, grp=4, ps=64, spread=4.0),
    dict(lens=[(64, 64), (1, 500)], G=2, grp=5, ps=16),
    dict(lens=[(31, 1), (5, 2), (260, 3)], G=1, grp=6, ps=16),
    dict(lens=[(257, 0)], G=2, grp=2, ps=32, layers=2),
    dict(lens=[(1, 33), (8, 120)], G=3, grp=1, ps=16),
    dict(lens=[(40, 3000), (24, 2500), (1, 3300), (90, 1800), (4, 2000)], G=8, grp=4, ps=64),
    dict(lens=[(17, 900)] * 40, G=2, grp=7, ps=128),
    dict(lens=[(1, 13 * i % 90) for i in range(100)], G=1, grp=2, ps=16, pad=4),
    dict(lens=[(1, 7 * i % 60) for i in range(40)] + [(30, 50), (0, 9)] + [(2, 5)] * 30 + [(150, 10)], G=2, grp=4, ps=16),
    dict(lens=[(20, 100)] + [(0, 5)] * 30, G=2, grp=5, ps=32),          # many tokens of one sequence, but no more rows than sequences
    dict(lens=[(0, 3)] * 20 + [(9, 0)], G=1, grp=8, ps=16),
]


def run_attn(b, q=None, layer=0, ws=None):
    q = b.rows(b.H) if q is None else q
    out = torch.full((b.T, b.H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b.T, b.H), float("nan"), device="cuda")
    ws = b.workspace() if ws is None else ws
    V.check(V.varrate_paged8_attn(b.pages, b.seqs, layer, b.grp, q, out, lse, b.status, ws))
    torch.cuda.synchronize()
    assert b.status.item() == 0
    return q, out, lse, ws


def check_attn(b, q, out, lse, layer=0):
    want, tol, want_lse, tol_lse = attn8_ref(b, q, layer)
    return close(out, want, tol), close(lse, want_lse, tol_lse)


@pytest.mark.parametrize("i", range(len(ATTN)))
def test_attention(i):
    kw = dict(ATTN[i])
    b = Batch8(**kw)
    layer = b.layers - 1
    q, out, lse, ws = run_attn(b, layer=layer)
    check_attn(b, q, out, lse, layer)
    q, again, lse2, _ = run_attn(b, q, layer, ws)       # one workspace for many calls; the same bits
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))


def test_attention_without_lse_gives_the_same():
    b = Batch8([(1, 700), (40, 3)])
    q, out, _, ws = run_attn(b)
    other = torch.empty_like(out)
    V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, other, None, b.status, ws))
    assert torch.equal(out, other)


@pytest.mark.parametrize("new", [1, 3, 200])
def test_scales_far_apart(new):
    """Values of blocks that differ by up to 2^200: what the large ones add up to is right, and nothing becomes infinite or NaN."""
    b = Batch8([(new, 400)], G=2, grp=4, ps=64)
    b.scale[:, :, 1] = torch.randint(20, 247, b.scale[:, :, 1].shape, generator=b.gen).to(torch.uint8).cuda()
    q, out, lse, _ = run_attn(b)
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    big = want.abs().amax()
    close(lse, want_lse, tol_lse)
    close(out, want, tol + 2.0 ** -85 * big)


@pytest.mark.parametrize("new, ctx", [(1, 40), (2, 47), (5, 60), (150, 20)])
def test_nan_of_some_tokens(new, ctx):
    """A NaN value reaches the rows that see its token, and no others."""
    b = Batch8([(new, ctx), (1, 50)], G=1, grp=2, ps=32)
    for u, d in ((ctx + new - 1, 3), (ctx + new // 2, 77), (ctx + new // 3, 77)):
        p, i = b.place(0, torch.tensor([u], device="cuda"))
        b.codes[0, p, 1, 0, i, d] = 0xFF
    q, out, lse, _ = run_attn(b)
    check_attn(b, q, out, lse)
    p, i = b.place(0, torch.tensor([ctx + new - 1], device="cuda"))
    b.codes[0, p, 0, 0, i, 9] = 0x7F                    # a key: the last token's rows are NaN
    q, out, lse, _ = run_attn(b, q)
    check_attn(b, q, out, lse)
    assert torch.isnan(out[new - 1]).all() and torch.isnan(lse[new - 1]).all()


@pytest.mark.parametrize("size", [0.0, 1e-30, 30.0, 1e30])
def test_queries_of_any_size(size):
    b = Batch8([(1, 200), (9, 50)], G=1, grp=4)
    q = (size * b.rows(4).double()).bfloat16()
    q, out, lse, _ = run_attn(b, q)
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    if size <= 1.0:
        close(out, want, tol)
        close(lse, want_lse, tol_lse)
    else:                                               # scores of a size where their error decides: finite all the same
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("i", range(len(ATTN)))
def test_weights(i):
    b = Batch8(**ATTN[i])
    layer = b.layers - 1
    q, _, lse, _ = run_attn(b, layer=layer)
    b.mass[torch.isnan(b.mass)] = 0.5                   # (places of no token: left alone)
    before = b.mass.clone()
    V.check(V.varrate_paged8_mass(b.pages, b.seqs, layer, b.grp, q, lse, b.status))
    want, tol = mass8_ref(b, q, lse, before, layer)
    close(b.mass, want, tol)
    assert b.status.item() == 0
    # every row's weights sum to 1
    assert abs(float((b.mass - before).double().sum()) - b.total * b.H) < 1e-4 * b.total * b.H
    first = b.mass.clone()
    b.mass.copy_(before)
    V.check(V.varrate_paged8_mass(b.pages, b.seqs, layer, b.grp, q, lse, b.status))
    assert torch.equal(first, b.mass)


def test_weights_of_rows_without_a_finite_lse():
    b = Batch8([(5, 60), (1, 30)], G=2, grp=2)
    q, _, lse, _ = run_attn(b)
    lse[1, 0], lse[2, 3], lse[5] = float("nan"), -float("inf"), float("inf")
    before = b.mass.nan_to_num(0.25)
    b.mass.copy_(before)
    V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
    want, tol = mass8_ref(b, q, lse, before)
    close(b.mass, want, tol)


def run_evict(b, budget, n_first=0, n_last=0, layer=0, n_layers=1, gone=None):
    S = len(b.lens)
    kept = torch.full((S, n_layers, b.G, budget), 9, dtype=torch.int32, device="cuda")
    new_len = torch.full((S,), 9, dtype=torch.int32, device="cuda")
    want = evict8_ref(b, layer, n_layers, budget, n_first, n_last)
    V.check(V.varrate_paged8_evict(b.pages, b.seqs, layer, n_layers, budget, n_first, n_last, kept, new_len, gone, b.status))
    torch.cuda.synchronize()
    assert b.status.item() == 0
    assert torch.equal(kept, want[3]) and torch.equal(new_len, want[4])
    assert torch.equal(torch.nan_to_num(b.mass, nan=-1), torch.nan_to_num(want[2], nan=-1))
    assert torch.equal(b.scale.view(torch.uint8), want[1].view(torch.uint8))
    x, y = (t.view(torch.float8_e4m3fn).float() for t in (b.codes, want[0]))
    assert torch.equal(torch.nan_to_num(x, nan=-999), torch.nan_to_num(y, nan=-999))


@pytest.mark.parametrize("kw, ev", [
    (dict(lens=[(1, 0)]), dict(budget=1)),
    (dict(lens=[(1, 1), (0, 0), (1, 30)]), dict(budget=1)),
    (dict(lens=[(1, 99), (0, 40), (7, 50)], G=3, ps=32), dict(budget=41, n_first=4, n_last=8)),
    (dict(lens=[(1, 2047)], G=1, ps=64, layers=3), dict(budget=1500, n_first=3, n_last=100, layer=1, n_layers=2)),
    (dict(lens=[(1, 3000), (1, 1023), (1, 1024), (1, 1025)], G=2, ps=128, spread=3.0), dict(budget=1024)),
    (dict(lens=[(1, 500)], G=1), dict(budget=300, n_first=300)),
    (dict(lens=[(1, 500)], G=1), dict(budget=300, n_last=300)),
    (dict(lens=[(1, 500)], G=1), dict(budget=300, n_first=100, n_last=200)),
    (dict(lens=[(1, 500)], G=1), dict(budget=500)),
    (dict(lens=[(1, 500)], G=1, ps=256), dict(budget=499)),
    (dict(lens=[(1, 50)], G=1), dict(budget=7000)),
    (dict(lens=[(1, 9000)], G=1, ps=256, spread=8.0), dict(budget=7000, n_first=16, n_last=64))])
def test_evict(kw, ev):
    run_evict(Batch8(**kw), **ev)


def test_evict_equal_weights_and_nan():
    b = Batch8([(1, 600)], G=3)
    b.mass[:, :, 0] = 1.0                               # all equal: the lowest places
    b.mass[:, :, 1] = (b.mass[:, :, 1] * 3).floor()     # few different ones
    b.mass[:, :, 2, 5] = float("nan")                   # a NaN is kept
    run_evict(b, 200, 2, 30)


def test_evict_counts_what_is_gone():
    b = Batch8([(1, 99), (1, 20)])
    gone = torch.tensor([7, 8], dtype=torch.int32, device="cuda")
    run_evict(b, 40, gone=gone)
    assert gone.tolist() == [67, 8]


@pytest.mark.parametrize("n, budget", [(360000, 30000), (360000, 300000), (900000, 100000)])
def test_evict_more_than_shared_memory_holds(n, budget):
    """A head of more tokens than a cluster keeps the weights of, or of more tiles than the move knows the first tokens of."""
    pages = n // 256 + 1
    codes = torch.randint(0, 127, (1, pages, 2, 1, 256, D), dtype=torch.uint8, device="cuda")
    scale = torch.full((1, pages, 2, 1, 16), 120, dtype=torch.uint8, device="cuda")
    mass = torch.randint(0, 1 << 20, (1, pages, 1, 256), device="cuda").float()
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    cache, length = V.Paged8Cache.of(codes, scale, mass), torch.tensor([n], dtype=torch.int32, device="cuda")
    seqs = V.SeqBatch.of(None, length, table, 0)
    kept, new = torch.zeros((1, 1, 1, budget), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    m = mass.flatten()[:n].clone()
    k, v = (codes[0, :, c, 0].flatten(0, 1)[:n].clone() for c in range(2))
    V.check(V.varrate_paged8_evict(cache, seqs, 0, 1, budget, 10, 1000, kept, new, None, st))
    rank = m.clone()
    rank[:10], rank[n - 1000:] = 1e30, 1e30
    want = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:budget].sort().values
    assert st.item() == 0 and new.item() == budget and torch.equal(kept.flatten().long(), want)
    assert torch.equal(mass.flatten()[:budget], m[want])
    for c, x in enumerate((k, v)):
        assert torch.equal(codes[0, :, c, 0].flatten(0, 1)[:budget], x[want])
