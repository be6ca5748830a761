"""The paged cache on the GPU (varrate_paged_append, varrate_paged_attn, varrate_paged_gather) against the
same operators in 64 bits. Tolerances are derived in paged_helpers."""
import pytest
import torch

from paged_helpers import D, DT, V, Batch, append_ref, attn_ref, close

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu(vlib):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


def freqs(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot) if rot else None


def status(b):
    torch.cuda.synchronize()
    return int(b.status.item())


# ------------------------------------------------------------------------------------ append

def run_append(b, norm=False, rot=128, fused=False, layer=0, queries=True, in_place=False, eps=1e-5):
    q = b.rows(b.H, 2 * b.G if fused else None)
    k, v = b.rows(b.G, 3 if fused else None), b.rows(b.G, 5 if fused else None)
    wq, wk = ((1 + 0.3 * b.randn(D)).to(b.dt).cuda() if norm else None for _ in range(2))
    before = b.pool.clone()
    want = append_ref(b, q if queries else None, k, v, wq, wk, eps, freqs(rot), rot, layer, before)
    q_out = q if in_place else torch.full((b.T, b.H, D), NAN, dtype=b.dt, device="cuda")
    rest = q.clone()
    st = V.varrate_paged_append(b.pages, b.seqs, layer, q if queries else None, k, v, wq, wk, eps, freqs(rot), rot,
                                q_out if queries else None, b.status)
    assert st == V.OK
    if queries:
        q_want = want[0]
        if in_place:   # rows of no sequence stay as they were
            out = torch.ones(b.T, dtype=torch.bool, device="cuda")
            out[b.start[0]:b.start[-1]] = False
            q_want = torch.where(out[:, None, None], rest.double(), q_want)
        close(q_out, q_want, want[2])
    written = want[3] > 0
    close(b.pool, want[1], want[3])
    # every other bit of the pool as it was (a value that the append stores has no allowed error of 0)
    bits = torch.int16 if b.dtype == "bf16" else torch.int32
    same = b.pool.view(bits) == before.view(bits)
    for s, (n, c) in enumerate(b.lens):
        for u in range(c, c + n):
            same[layer, b.table_host[s, u // b.ps], :, :, u % b.ps] = True
    assert same.all() and (written.any() or b.total == 0)
    assert status(b) == V.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[(1, 0)], [(1, 31), (1, 15), (1, 16)], [(5, 0), (0, 9), (37, 3), (1, 64)], [(130, 7)]])
@pytest.mark.parametrize("norm, rot, fused", [(False, 128, False), (True, 128, True), (True, 64, False), (False, 0, True),
                                              (True, 16, False), (False, 112, True)])
def test_append(dtype, lens, norm, rot, fused):
    run_append(Batch(lens, dtype, pad=3, lead=2), norm, rot, fused)


@pytest.mark.parametrize("G, grp", [(1, 1), (1, 8), (3, 7), (8, 4), (5, 3)])
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_append_head_layouts(G, grp, ps):
    run_append(Batch([(19, 250), (2, 0)], "bf16", G, grp, ps, layers=2), True, 128, True, layer=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_in_place_and_without_queries(dtype):
    run_append(Batch([(9, 4), (1, 77)], dtype, pad=2), True, in_place=True)
    run_append(Batch([(9, 4), (1, 77)], dtype, pad=2), queries=False)


def test_append_many_sequences():
    """More sequences than one or two warps look up at once, empty ones among them."""
    run_append(Batch([(s % 3, s % 5) for s in range(1300)], "bf16", 1, 2, pad=5))


def test_append_far_positions():
    """Positions near 2^31 / 8: the angle keeps its precision (64-bit reference: the product in double)."""
    b = Batch([(3, 5)], "f32", 1, 2)
    far = (1 << 28) - 3
    table = torch.zeros((1, (far + 3) // b.ps + 1), dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([far + 3], dtype=torch.int32, device="cuda")
    seqs = V.SeqBatch.of(b.row_start, kv_len, table, b.T)
    q, k, v = b.rows(b.H), b.rows(b.G), b.rows(b.G)
    q_out = torch.empty_like(q)
    assert V.varrate_paged_append(b.pages, seqs, 0, q, k, v, None, None, 0.0, freqs(128), 128, q_out, b.status) == V.OK
    pos = torch.arange(far, far + 3, dtype=torch.float64, device="cuda")
    a = pos[:, None, None] * freqs(128)
    x0, x1 = q.double()[..., :64], q.double()[..., 64:]
    want = torch.cat((x0 * a.cos() - x1 * a.sin(), x1 * a.cos() + x0 * a.sin()), -1)
    pair = (x0.abs() + x1.abs()).repeat(1, 1, 2)
    # 2^28 positions times a rounding of 2^-53 of the angle on each side: 2^-24, beside the fp32 roundings
    close(q_out, want, pair * (2.0 ** -23 + 32 * 2.0 ** -24))
    assert status(b) == V.OK


# ------------------------------------------------------------------------------------ attention

def run_attn(b, layer=0, ws=None, q=None):
    q = 2 * b.rows(b.H) if q is None else q
    out = torch.full((b.T, b.H, D), NAN, dtype=b.dt, device="cuda")
    want, tol = attn_ref(b, q, layer)
    assert V.varrate_paged_attn(b.pages, b.seqs, layer, b.grp, q, out, b.status, b.workspace() if ws is None else ws) == V.OK
    close(out, want, tol)          # rows of no sequence are NaN on both sides: not written
    assert status(b) == V.OK
    return out


LENS = [[(1, 0)], [(1, 127)], [(1, 128)], [(1, 700), (1, 3), (1, 129)], [(7, 0)], [(64, 64), (0, 5), (3, 200)],
        [(129, 0)], [(300, 0), (1, 1000), (33, 95)], [(40, 1500)]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("G, grp", [(2, 4), (1, 7), (3, 1), (1, 8)])
def test_attn(dtype, lens, G, grp):
    run_attn(Batch(lens, dtype, G, grp, pad=2, lead=1))


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_page_sizes(dtype, ps):
    run_attn(Batch([(1, 600), (150, 300), (1, ps - 1), (1, ps), (2 * ps, 0)], dtype, 2, 4, ps, layers=2), layer=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["keys", "values"])
@pytest.mark.parametrize("what", [NAN, float("inf"), -float("inf")])
@pytest.mark.parametrize("grp", [1, 4, 7])
def test_attn_later_tokens_have_no_part(dtype, where, what, grp):
    """A later token of the chunk holds NaN or infinities: the tokens before it do not see them, those from it on do
    (values: in the result as 64-bit arithmetic has it; keys: only tokens before it are compared)."""
    b = Batch([(200, 77), (1, 40)], dtype, 2, grp)
    at = 77 + 90
    b.pool[0, b.table_host[0, at // b.ps], 0 if where == "keys" else 1, 1, at % b.ps, 5:9] = what
    q = b.rows(b.H)
    out = torch.zeros((b.T, b.H, D), dtype=b.dt, device="cuda")
    want, tol = attn_ref(b, q)
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, b.workspace()) == V.OK
    if where == "values":
        close(out, want, tol)
    else:
        sees = slice(90, 200)
        close(out[:90], want[:90], tol[:90])
        close(out[200:], want[200:], tol[200:])
        close(out[sees, :b.grp], want[sees, :b.grp], tol[sees, :b.grp])
    assert status(b) == V.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_large_scores(dtype):
    """Scores of some hundreds: the running maximum moves, weights underflow."""
    b = Batch([(150, 600), (1, 900)], dtype, 2, 4)
    b.pool[:, :, 0] *= 16
    run_attn(b, q=6 * b.rows(b.H))
    b.pool[:, :, 0] = b.pool[:, :, 0].sort(dim=-1).values   # rising maxima along a page
    run_attn(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_one_workspace_for_many_calls(dtype):
    big = Batch([(1, 3000)] * 3, dtype, 2, 4)
    ws = big.workspace()
    first = run_attn(big, ws=ws, q=(q := big.rows(big.H)))
    for lens in ([(1, 5)], [(2, 1000)], [(1, 2999)] * 2):
        b = Batch(lens, dtype, 2, 4, seed=3)
        if V.varrate_paged_attn_ws_bytes(b.pages, b.seqs, b.grp) <= ws.numel():
            run_attn(b, ws=ws)
    assert torch.equal(run_attn(big, ws=ws, q=q), first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_from_a_graph_and_on_a_stream(dtype):
    """A captured step: lengths, rows and pages refilled in place between replays, a batch padded with empty sequences."""
    b = Batch([(3, 200), (1, 900), (1, 64)], dtype, 2, 4, pad=4)
    q = b.rows(b.H)
    out, ws = torch.zeros_like(q), b.workspace()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
    torch.cuda.synchronize()
    want, tol = attn_ref(b, q)
    close(out[:5], want[:5], tol[:5])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
    for lens in ([(3, 200), (1, 900), (1, 64)], [(1, 100), (2, 700), (0, 64)], [(1, 50), (0, 3), (0, 3)]):
        b.lens, b.len = lens, [n + c for n, c in lens]
        b.start = [0]
        for n, _ in lens:
            b.start.append(b.start[-1] + n)
        b.row_start.copy_(torch.tensor(b.start, dtype=torch.int32))
        b.kv_len.copy_(torch.tensor(b.len, dtype=torch.int32))
        out.fill_(7)
        g.replay()
        want, tol = attn_ref(b, q)
        n = b.start[-1]
        close(out[:n], want[:n], tol[:n])
        assert (out[n:] == 7).all()
        assert status(b) == V.OK


# ------------------------------------------------------------------------------------ gather

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [16, 128])
@pytest.mark.parametrize("n, first", [(1, [0, 40, 299]), (100, [0, 13, 200]), (300, None), (129, [171, 0, 7])])
def test_gather(dtype, ps, n, first):
    b = Batch([(1, 299), (3, 297), (0, 300)], dtype, 3, 2, ps, layers=3)
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    for layer, layers in ((0, 3), (1, 1), (1, 2)):
        out = [torch.full((3, layers, 3, n, D), NAN, dtype=b.dt, device="cuda") for _ in range(2)]
        assert V.varrate_paged_gather(b.pages, b.seqs, layer, layers, f, n, *out, b.status) == V.OK
        for c in range(2):
            for s in range(3):
                at = 0 if first is None else first[s]
                for l in range(layers):
                    want = b.tokens(s, c, layer + l)[:, at:at + n]
                    assert torch.equal(out[c][s, l].double(), want)
    keep = out[1].clone()
    out[1].fill_(3)
    assert V.varrate_paged_gather(b.pages, b.seqs, 1, 2, f, n, None, out[1], b.status) == V.OK
    assert torch.equal(out[1], keep)
    assert status(b) == V.OK


# ------------------------------------------------------------------------------------ tables out of range

def bad_tables():
    def page(b): b.table[1, 1:3] = b.n_pages
    def negative(b): b.table[1, 1:3] = -1
    def short(b): b.kv_len[1] = 4
    def long(b): b.kv_len[1] = b.max_pages * b.ps + 1
    def below(b): b.kv_len[1] = -3
    def order(b): b.row_start[2] = 1
    def past(b): b.row_start[3] = b.T + 1
    return [page, negative, short, long, below, order, past]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spoil", bad_tables(), ids=lambda f: f.__name__)
def test_tables_out_of_range(dtype, spoil):
    """Marked in the status word; a sequence that the spoilt entry does not touch is right all the same."""
    b = Batch([(4, 30), (5, 40), (6, 50)], dtype, 2, 4)
    q = b.rows(b.H)
    want, tol = attn_ref(b, q)
    spoil(b)
    out = torch.full_like(q, NAN)
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, b.workspace()) == V.OK
    assert status(b) == V.ERR_CORRUPT
    if spoil.__name__ == "order":   # the rows of the third sequence then cover the first one's
        return
    close(out[:4], want[:4], tol[:4])
    if spoil.__name__ != "past":
        close(out[9:], want[9:], tol[9:])
    b.status.zero_()
    k, v = b.rows(b.G), b.rows(b.G)
    q_out = torch.full_like(q, NAN)
    assert V.varrate_paged_append(b.pages, b.seqs, 0, q, k, v, None, None, 0.0, None, 0, q_out, b.status) == V.OK
    assert status(b) == V.ERR_CORRUPT
    assert torch.equal(q_out[:4], q[:4])
    if spoil.__name__ in ("page", "negative", "long"):
        b.status.zero_()
        outs = [torch.full((3, 1, 2, 30, D), NAN, dtype=b.dt, device="cuda") for _ in range(2)]
        assert V.varrate_paged_gather(b.pages, b.seqs, 0, 1, None, 30, *outs, b.status) == V.OK
        assert status(b) == V.ERR_CORRUPT
        for s in (0, 2):
            assert torch.equal(outs[0][s, 0].double(), b.tokens(s, 0)[:, :30])


def test_gather_range_out_of_sequence():
    b = Batch([(1, 99), (1, 99)], "bf16", 2, 4)
    for first in ([0, 51], [-1, 3], [90, 2 ** 31 - 10]):
        b.status.zero_()
        outs = [torch.full((2, 1, 2, 50, D), 5.0, dtype=b.dt, device="cuda") for _ in range(2)]
        f = torch.tensor(first, dtype=torch.int32, device="cuda")
        assert V.varrate_paged_gather(b.pages, b.seqs, 0, 1, f, 50, *outs, b.status) == V.OK
        assert status(b) == V.ERR_CORRUPT
        for s in range(2):
            if 0 <= first[s] and first[s] + 50 <= 100:
                assert torch.equal(outs[1][s, 0].double(), b.tokens(s, 1)[:, first[s]:first[s] + 50])
            else:
                assert (outs[1][s] == 5).all()


def test_gather_of_more_tokens_than_a_sequence_may_have():
    """As many as the argument holds, which no sequence has: nothing is written."""
    b = Batch([(1, 99), (1, 30)], "bf16", 2, 4)
    out = torch.full((2, 1, 2, 50, D), 5.0, dtype=b.dt, device="cuda")
    for n in (2 ** 31 - 1, 2 ** 31 - 63, 2 ** 31 - 255):
        b.status.zero_()
        assert V.lib().varrate_paged_gather(b.pages.ref, b.seqs.ref, 0, 1, None, n, out.data_ptr(), None, b.status.data_ptr(),
                                            b.pages.stream(None)) == V.OK
        assert status(b) == V.ERR_CORRUPT and (out == 5).all()


# ------------------------------------------------------------------------------------ offsets past 32 bits

def test_pool_of_more_than_2_to_the_32_elements():
    G, ps, n = 8, 256, 9000
    b = Batch([(40, 700), (1, 500)], "bf16", G, 4, ps)
    pool = torch.empty((1, n, 2, G, ps, D), dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 1 << 32
    used = sorted({int(x) for x in b.table_host.flatten() if x >= 0})
    place = {x: n - 1 - i * 7 for i, x in enumerate(used)}
    for x, y in place.items():
        pool[0, y] = b.pool[0, x]
    pages = V.PagedCache.of(pool)
    table = torch.tensor([[place.get(int(x), -7) for x in row] for row in b.table_host], dtype=torch.int32, device="cuda")
    seqs = V.SeqBatch.of(b.row_start, b.kv_len, table, b.T)
    q, k, v = b.rows(b.H), b.rows(G), b.rows(G)
    outs, q_outs = [], []
    for pg, sq, bb in ((b.pages, b.seqs, b), (pages, seqs, b)):
        q_out, out = torch.zeros_like(q), torch.zeros_like(q)
        assert V.varrate_paged_append(pg, sq, 0, q, k, v, None, None, 0.0, freqs(128), 128, q_out, b.status) == V.OK
        assert V.varrate_paged_attn(pg, sq, 0, 4, q_out, out, b.status, V.paged_attn_workspace(pg, sq, 4)) == V.OK
        kv = [torch.zeros((2, 1, G, 500, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        assert V.varrate_paged_gather(pg, sq, 0, 1, None, 500, *kv, b.status) == V.OK
        outs.append([out, *kv])
        q_outs.append(q_out)
    assert status(b) == V.OK
    assert torch.equal(q_outs[0], q_outs[1])
    for x, y in zip(*outs):
        assert torch.equal(x, y)
    want, tol = attn_ref(b, q_outs[0])
    close(outs[1][0], want, tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("jump", [30.0, 90.0, 400.0, 3000.0])
@pytest.mark.parametrize("at", [5, 40, 70, 100, 130, 200, 300])
def test_attn_a_score_far_above_those_before_it(dtype, jump, at):
    """One key whose score stands `jump` above all others, in each quarter of a key tile, in the first tile and later ones:
    the running reference moves by a little, by much, or past what a weight can hold."""
    for lens in ([(1, 400)], [(130, 271)]):
        b = Batch(lens, dtype, 1, 4)
        q = b.rows(b.H)
        q[..., 0] = 16.0
        b.pool[:, :, 0, :, :, 0] = 0.0
        b.pool[0, b.table_host[0, at // b.ps], 0, 0, at % b.ps, 0] = jump * D ** 0.5 / 16.0
        run_attn(b, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_of_many_sequences(dtype):
    """More sequences than a warp looks at at once, empty ones and single tokens among them, each with few keys."""
    run_attn(Batch([(s % 4, (7 * s) % 41 + 1) for s in range(500)], dtype, 2, 4, pad=3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, ctx", [(1, 120), (20, 100)])
def test_attn_of_one_tile_a_sequence(dtype, n, ctx):
    """Several units in a row for every CTA, each of one key tile: one of the two query tiles has nothing to do. Again and
    again with one workspace: the same bits."""
    b = Batch([(n, (5 * s) % ctx) for s in range(300)], dtype, 8, 1, pad=1)
    ws, q = b.workspace(), 2 * b.rows(b.H)
    out = run_attn(b, ws=ws, q=q)
    again = torch.empty_like(out)
    for _ in range(30):
        again.fill_(NAN)
        assert V.varrate_paged_attn(b.pages, b.seqs, 0, 1, q, again, b.status, ws) == V.OK
        assert torch.equal(again.view(torch.uint8), out.view(torch.uint8))
    assert status(b) == V.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[(1, 9999)], [(1, 6000), (0, 50), (1, 31)], [(40, 5000)]], ids=str)
def test_attn_one_head_long_context(dtype, lens):
    """One KV head and few rows: the keys are cut into many runs, merged at the end."""
    run_attn(Batch(lens, dtype, 1, 8, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_shared_pages(dtype):
    """Sequences that share the pages of a common prefix (read, not written)."""
    b = Batch([(1, 95), (40, 96), (1, 200)], dtype, 2, 4)
    b.table[1, :3] = b.table[0, :3]
    b.table_host[1, :3] = b.table_host[0, :3]
    b.table[2, :6] = b.table[0, :6].clone()
    b.table_host[2, :6] = b.table_host[0, :6]
    run_attn(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_workspace_found_used(dtype):
    """A counter that is not zero is reported once; the next call on the workspace is right again."""
    b = Batch([(150, 600), (1, 900)], dtype, 2, 4)
    ws = b.workspace()
    ws[0] = 3
    q = b.rows(b.H)
    out = torch.zeros_like(q)
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
    assert status(b) == V.ERR_CORRUPT
    b.status.zero_()
    run_attn(b, ws=ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count", [10 ** 6, 2 ** 30, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 7, -1, -151, -400])
def test_attn_workspace_with_any_count(dtype, count):
    """Whatever the counter holds, no unit out of range is taken; the call after is right again."""
    b = Batch([(150, 600), (1, 900), (300, 40)], dtype, 4, 2)
    ws, q = b.workspace(), b.rows(b.H)
    ws[:4].view(torch.int32)[0] = count
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, torch.zeros_like(q), b.status, ws) == V.OK
    assert status(b) == V.ERR_CORRUPT
    b.status.zero_()
    run_attn(b, ws=ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_calls_that_overlap_on_one_workspace(dtype):
    """Not allowed, and their results are not to be trusted: but nothing outside the outputs and the workspace is touched, and
    the workspace serves again once it is zeroed."""
    bs = [Batch([(1, 3000), (1, 5000)], dtype, 1, 8, seed=1), Batch([(400, 900), (300, 2000)], dtype, 2, 4, seed=2)]
    qs = [b.rows(b.H) for b in bs]
    big = [torch.full((b.T + 2, b.H, D), 7.0, dtype=b.dt, device="cuda") for b in bs]
    n = max(b.workspace().numel() for b in bs)
    ws = torch.full((n + 4096,), 90, dtype=torch.uint8, device="cuda")
    ws[:n] = 0
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for _ in range(10):
        for b, q, out, s in zip(bs, qs, big, streams):
            assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out[1:-1], b.status, ws[:n], stream=s) == V.OK
    torch.cuda.synchronize()
    assert (ws[n:] == 90).all()
    for b, out in zip(bs, big):
        assert (out[0] == 7).all() and (out[-1] == 7).all()
        ws[:n] = 0
        b.status.zero_()
        run_attn(b, ws=ws[:n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[(0, 0)], [(0, 40), (0, 0), (0, 7)]], ids=str)
def test_batch_without_new_tokens(dtype, lens):
    """A captured step of which no sequence is alive: rows and pages stay as they are."""
    b = Batch(lens, dtype, 2, 4, pad=5)
    run_append(b)
    run_attn(b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_two_streams_and_two_graphs(dtype):
    """Two batches at once on two streams, each with its workspace; then two captured graphs in turn on one workspace."""
    bs = [Batch([(120, 700), (1, 2000)], dtype, 2, 4, seed=1), Batch([(1, 1500), (9, 100)], dtype, 2, 4, seed=2)]
    qs = [b.rows(b.H) for b in bs]
    refs = [attn_ref(b, q) for b, q in zip(bs, qs)]
    outs, wss = [torch.zeros_like(q) for q in qs], [b.workspace() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, q, out, ws, s in zip(bs, qs, outs, wss, streams):
            assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws, stream=s) == V.OK
    torch.cuda.synchronize()
    for b, out, (want, tol) in zip(bs, outs, refs):
        close(out, want, tol)
        assert status(b) == V.OK
    ws = max(wss, key=lambda w: w.numel())
    graphs = []
    for b, q, out in zip(bs, qs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
        graphs.append(g)
    for _ in range(3):
        for out in outs:
            out.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for b, out, (want, tol) in zip(bs, outs, refs):
            close(out, want, tol)
            assert status(b) == V.OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_is_the_same_from_call_to_call(dtype):
    b = Batch([(150, 900), (1, 3000), (30, 30)], dtype, 2, 4)
    q, ws = b.rows(b.H), b.workspace()
    first = torch.zeros_like(q)
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, first, b.status, ws) == V.OK
    for _ in range(5):
        out = torch.zeros_like(q)
        assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, out, b.status, ws) == V.OK
        assert torch.equal(out, first)
    assert status(b) == V.OK
