"""The operators of the 8-bit paged cache together, as a serving program runs them: steps, graphs, streams, wrong tables, large pools."""
import pytest
import torch

from paged8_helpers import Batch8, append8_check, attn8_ref, evict8_ref, mass8_ref
from paged_helpers import D, close
from paper_2607_15498_gb300 import varrate as V

pytestmark = pytest.mark.gpu


class Serving:
    """Sequences that grow step by step, with every call checked against the formulas in 64 bits on the cache as it stands."""

    def __init__(self, contexts, G=2, grp=4, ps=16, most=400, seed=3):
        self.b = Batch8([(0, 0)] * len(contexts), G=G, grp=grp, ps=ps, seed=seed, spare=len(contexts) * (most // ps + 1))
        b, per = self.b, most // ps + 1
        order = torch.randperm(b.n_pages, generator=b.gen)[:len(contexts) * per].to(torch.int32)
        b.table_host = order.view(len(contexts), per).contiguous()
        b.table, b.max_pages = b.table_host.cuda(), per
        self.n = [0] * len(contexts)
        self.gone = torch.zeros(len(contexts), dtype=torch.int32, device="cuda")
        self.freq = 10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device="cuda") / 128)
        self.step(contexts)

    def step(self, new):
        b = self.b
        b.lens = [(n, k) for n, k in zip(new, self.n)]
        self.n = [n + k for n, k in zip(new, self.n)]
        b.len, b.start = list(self.n), [0]
        for n in new:
            b.start.append(b.start[-1] + n)
        b.T = b.total = b.start[-1]
        b.row_start = torch.tensor(b.start, dtype=torch.int32, device="cuda")
        b.kv_len = torch.tensor(b.len, dtype=torch.int32, device="cuda")
        b.seqs = V.SeqBatch.of(b.row_start, b.kv_len, b.table, b.T)
        q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
        out, lse = torch.empty_like(q), torch.empty((b.T, b.H), device="cuda")
        q_out = torch.empty_like(q)
        before = b.codes.clone(), b.scale.clone(), b.mass.clone()
        V.check(V.varrate_paged8_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, self.freq, 128, self.gone, q_out, b.status))
        append8_check(b, (q, k, v, None, None, 0.0, self.freq, 128, self.gone.tolist()), 0, before, q_out)
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q_out, out, lse, b.status, b.workspace()))
        want, tol, want_lse, tol_lse = attn8_ref(b, q_out)
        close(out, want, tol)
        close(lse, want_lse, tol_lse)
        before = b.mass.clone()
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q_out, lse, b.status))
        for s, n in enumerate(self.n):                      # places of no token hold anything
            p, i = b.place(s, torch.arange(n, device="cuda"))
            assert torch.isfinite(b.mass[0, p, :, i]).all()
        want, tol = mass8_ref(b, q_out, lse, before)
        close(b.mass, want, tol)
        assert b.status.item() == 0

    def evict(self, budget, n_first, n_last):
        b, S = self.b, len(self.n)
        kept = torch.empty((S, 1, b.G, budget), dtype=torch.int32, device="cuda")
        new = torch.empty(S, dtype=torch.int32, device="cuda")
        want = evict8_ref(b, 0, 1, budget, n_first, n_last)
        V.check(V.varrate_paged8_evict(b.pages, b.seqs, 0, 1, budget, n_first, n_last, kept, new, self.gone, b.status))
        for got, ref in zip((b.codes, b.scale, b.mass, kept, new), want):
            got, ref = (t.view(torch.float8_e4m3fn).float() if t.dtype == torch.uint8 and t.dim() == 6 else t for t in (got, ref))
            assert torch.equal(torch.nan_to_num(got.float(), nan=-9), torch.nan_to_num(ref.float(), nan=-9))
        self.n = new.tolist()
        assert b.status.item() == 0


def test_prompt_steps_and_evictions():
    s = Serving([150, 37, 260, 1])
    s.step([1, 1, 1, 1])
    s.evict(120, 4, 30)
    s.step([1, 1, 1, 1])
    s.step([3, 20, 1, 0])
    s.evict(100, 4, 16)
    for _ in range(3):
        s.step([1, 1, 1, 1])
    assert s.gone.tolist()[1] == 0 and s.gone.tolist()[0] > 50


def test_a_captured_step_follows_its_tables():
    """One capture of append, attention, weights and eviction; replayed with other lengths, rows and tables."""
    b = Batch8([(1, 100), (1, 30), (40, 80)], G=2, grp=4, ps=32, pad=6)
    q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
    freq = 10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device="cuda") / 128)
    q_out, out, lse, ws = torch.empty_like(q), torch.empty_like(q), torch.empty((b.T, b.H), device="cuda"), b.workspace()
    kept, new = torch.empty((3, 1, 2, 60), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")

    def run():
        V.check(V.varrate_paged8_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, freq, 128, None, q_out, b.status))
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q_out, out, lse, b.status, ws))
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q_out, lse, b.status))
        V.check(V.varrate_paged8_evict(b.pages, b.seqs, 0, 1, 60, 2, 20, kept, new, None, b.status))

    start = [t.clone() for t in (b.codes, b.scale, b.mass)]

    def reset():
        for t, x in zip((b.codes, b.scale, b.mass), start):
            t.copy_(x)

    def state():
        return [t.clone() for t in (b.codes, b.scale, b.mass, q_out[:b.start[-1]], out[:b.start[-1]], lse[:b.start[-1]], kept, new)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph):
        run()
    for lengths, starts in (([101, 31, 120], [0, 1, 2, 42]), ([60, 44, 90], [0, 3, 3, 40]), ([17, 2, 128], [1, 2, 4, 48])):
        b.kv_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        b.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
        b.start = starts
        q.normal_(), k.normal_(), v.normal_()
        reset()
        out.zero_(), q_out.zero_(), lse.zero_()
        run()
        torch.cuda.synchronize()
        want = state()
        reset()
        out.zero_(), q_out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(state(), want):
            assert torch.equal(x.view(torch.uint8) if x.dtype == torch.bfloat16 else torch.nan_to_num(x.float(), nan=-9),
                               y.view(torch.uint8) if y.dtype == torch.bfloat16 else torch.nan_to_num(y.float(), nan=-9))
        assert b.status.item() == 0


def test_two_graphs_and_an_eager_call_share_a_workspace():
    b = Batch8([(1, 900), (50, 400)], G=2, grp=4, ps=64)
    q = [b.rows(b.H) for _ in range(3)]
    ws = b.workspace()
    outs = [torch.empty_like(q[0]) for _ in range(3)]
    call = lambda i: V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q[i], outs[i], None, b.status, ws))   # noqa: E731
    graphs = []
    for i in range(2):
        call(i)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    call(2)
    want = []
    for i in range(3):
        call(i)
        want.append(outs[i].clone())
    for t in outs:
        t.zero_()
    for i in (1, 0, 1, 0):
        graphs[i].replay()
        call(2)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want)) and b.status.item() == 0


def test_on_another_stream():
    b = Batch8([(1, 500), (33, 70)], G=2, grp=4, ps=64)
    q = b.rows(b.H)
    out, lse, ws = torch.empty_like(q), torch.empty((b.T, b.H), device="cuda"), b.workspace()
    mass = b.mass.nan_to_num(0.5)
    b.mass.copy_(mass)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, out, lse, b.status, ws))
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
    side.synchronize()
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    close(out, want, tol)
    close(lse, want_lse, tol_lse)
    want, tol = mass8_ref(b, q, lse, mass)
    close(b.mass, want, tol)


def test_queries_may_be_rotated_in_place():
    b = Batch8([(20, 3)], G=2, grp=4)
    q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
    freq = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device="cuda") / 64)
    keep, out = q.clone(), torch.empty_like(q)
    start = b.codes.clone(), b.scale.clone()
    V.check(V.varrate_paged8_append(b.pages, b.seqs, 0, keep, k, v, None, None, 0.0, freq, 64, None, out, b.status))
    b.codes.copy_(start[0]), b.scale.copy_(start[1])
    V.check(V.varrate_paged8_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, freq, 64, None, q, b.status))
    assert torch.equal(q, out)


def clean(b):
    """A batch whose places hold no NaN, for comparisons of whole caches."""
    b.mass.nan_to_num_(0.5)
    b.codes[b.codes == 0x7F] = 0
    return b


@pytest.mark.parametrize("wrong", ["length", "row", "page", "gone", "short"])
def test_a_wrong_table_spoils_its_sequence_alone(wrong):
    """Lengths, rows and pages out of range raise the status; the other sequences' results are those of a batch without it."""
    def run(broken):
        b = clean(Batch8([(1, 80), (30, 40), (1, 200), (12, 0)], G=2, grp=4, ps=16, layers=1))
        gone = torch.zeros(4, dtype=torch.int32, device="cuda")
        if broken:
            if wrong == "length":
                b.kv_len[1] = 100000
            elif wrong == "row":
                b.row_start[4] = b.T + 1
            elif wrong == "page":
                b.table[1, 2] = b.n_pages
            elif wrong == "gone":
                gone[1] = -1
            else:
                b.kv_len[1] = 29                            # fewer tokens than new ones
        q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
        q_out, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((b.T, b.H), device="cuda")
        freq = 10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device="cuda") / 128)
        kept, new = torch.zeros((4, 1, 2, 50), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        status = []
        for f in (lambda: V.varrate_paged8_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, freq, 128, gone, q_out, b.status),
                  lambda: V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q_out, out, lse, b.status, b.workspace()),
                  lambda: V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q_out, lse, b.status),
                  lambda: V.varrate_paged8_evict(b.pages, b.seqs, 0, 1, 50, 2, 10, kept, new, None, b.status)):
            b.status.zero_()
            V.check(f())
            torch.cuda.synchronize()
            status.append(b.status.item())
        return b, q_out, out, lse, kept, new, status

    a, x = run(False), run(True)
    assert a[-1] == [0, 0, 0, 0]
    by_rows = wrong in ("row",)                             # evict does not look at rows; the others not at gone
    assert x[-1][0] == V.ERR_CORRUPT
    if wrong != "gone":
        assert x[-1][1] == x[-1][2] == V.ERR_CORRUPT
    assert x[-1][3] == (0 if by_rows or wrong in ("gone", "short") else V.ERR_CORRUPT)
    bad = 3 if wrong == "row" else 1
    for s in range(4):
        if s == bad:
            continue
        rows = slice(a[0].start[s], a[0].start[s + 1])
        for i in (1, 2, 3):
            assert torch.equal(a[i][rows], x[i][rows]), (s, i)
        assert torch.equal(a[4][s], x[4][s]) and a[5][s] == x[5][s]
        p, u = a[0].place(s, torch.arange(min(a[0].len[s], 50), device="cuda"))
        assert torch.equal(a[0].codes[0, p, :, :, u], x[0].codes[0, p, :, :, u])
        assert torch.equal(a[0].mass[0, p, :, u], x[0].mass[0, p, :, u])


def test_row_ranges_out_of_order_stay_in_range():
    b = clean(Batch8([(5, 30), (40, 10), (7, 90)], G=1, grp=2))
    for starts in ([0, 45, 5, 52], [50, 40, 30, 0], [0, 5, 45, 2 ** 31 - 1], [-5, 5, 45, 52], [2 ** 31 - 1] * 4):
        b.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
        q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
        out, lse = torch.zeros_like(q), torch.zeros((b.T, b.H), device="cuda")
        b.status.zero_()
        V.check(V.varrate_paged8_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, None, 0, None, out, b.status))
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, out, lse, b.status, b.workspace()))
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
        torch.cuda.synchronize()
        assert b.status.item() == V.ERR_CORRUPT


def test_a_layer_far_into_a_large_pool():
    """Offsets past 2^32 bytes: the last layer of 6 GB of codes gives what the same pages give alone."""
    G, grp, ps, pages, layers = 8, 4, 64, 4096, 12
    big = V.Paged8Cache.allocate(layers, pages, G, ps)
    small = V.Paged8Cache.allocate(1, 40, G, ps)
    small.codes.view(torch.uint8).random_(0, 127)
    small.scale.view(torch.uint8).fill_(120)
    small.mass.uniform_()
    for name in ("codes", "scale", "mass"):
        x, y = (getattr(c, name) for c in (big, small))
        x, y = (t.view(torch.uint8) if t.dtype != torch.float32 else t for t in (x, y))
        x[layers - 1, pages - 40:] = y[0]
    length = torch.tensor([1200, 1000], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 1, 131], dtype=torch.int32, device="cuda")
    got = []
    for cache, layer, first in ((big, layers - 1, pages - 40), (small, 0, 0)):
        table = torch.arange(first, first + 40, dtype=torch.int32, device="cuda").view(2, 20).contiguous()
        seqs = V.SeqBatch.of(start, length, table, 131)
        gen = torch.Generator(device="cuda").manual_seed(5)
        q, k, v = (torch.randn((131, h, D), generator=gen, device="cuda").bfloat16() for h in (G * grp, G, G))
        out, q_out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((131, G * grp), device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        kept, new = torch.empty((2, 1, G, 500), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        V.check(V.varrate_paged8_append(cache, seqs, layer, q, k, v, None, None, 0.0, None, 0, None, q_out, st))
        V.check(V.varrate_paged8_attn(cache, seqs, layer, grp, q_out, out, lse, st, V.paged8_attn_workspace(cache, seqs, grp)))
        V.check(V.varrate_paged8_mass(cache, seqs, layer, grp, q_out, lse, st))
        V.check(V.varrate_paged8_evict(cache, seqs, layer, 1, 500, 4, 100, kept, new, None, st))
        assert st.item() == 0
        got.append([out, lse, kept, cache.codes.view(torch.uint8)[layer, first:first + 40].clone(),
                    cache.scale.view(torch.uint8)[layer, first:first + 40].clone(), cache.mass[layer, first:first + 40].clone()])
    for x, y in zip(*got):
        assert torch.equal(x, y)
