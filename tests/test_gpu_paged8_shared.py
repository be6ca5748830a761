"""Paged cache in 8 bits: sequences whose first pages are the same, and batches in which every sequence is one kernel's."""
import pytest
import torch

from paged8_helpers import Batch8, attn8_ref, mass8_ref
from paper_2607_15498_gb300 import varrate as V

pytestmark = pytest.mark.gpu


def close(got, want, tol):
    bad = ~((got.double() - want).abs() <= tol) & ~torch.isnan(want)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() - tol)[bad].max()))


def run(b):
    q = b.rows(b.H).contiguous()
    out, lse = torch.empty_like(q), torch.empty((b.T, b.H), device=b.device)
    V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, out, lse, b.status, b.workspace()))
    before = b.mass.nan_to_num(0.5)
    b.mass.copy_(before)
    V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
    assert b.status.item() == 0
    want, tol, want_lse, tol_lse = attn8_ref(b, q)
    close(out, want, tol)
    close(lse, want_lse, tol_lse)
    # of each sequence by itself: its weights' error is its own
    weight, allowed, lens = before.double(), 0, b.lens
    for s in range(len(lens)):
        b.lens = [x if i == s else (0, sum(x)) for i, x in enumerate(lens)]
        w, t = mass8_ref(b, q, lse, before)
        weight, allowed = weight + (w - before.double()), allowed + t
    b.lens = lens
    # and a rounding of what stands there for each sequence that adds to it
    close(b.mass, weight, allowed + len(lens) * 2.0 ** -24 * weight.abs())


@pytest.mark.parametrize("lens, ps, pages", [([(1, 79), (1, 70), (1, 64)], 16, 4),           # steps only
                                             ([(40, 60), (3, 66), (1, 90), (200, 70)], 32, 2),   # of both kernels
                                             ([(130, 140), (300, 130)], 128, 1)])                # chunks only
def test_first_pages_of_several_sequences(lens, ps, pages):
    b = Batch8(lens, G=2, grp=4, ps=ps)
    b.table_host[1:, :pages] = b.table_host[0, :pages]
    b.table.copy_(b.table_host)
    run(b)


@pytest.mark.parametrize("lens, grp", [([(2, 100), (4, 30), (0, 50), (3, 0)], 4),              # more rows than sequences, none many
                                       ([(512, 0)], 4), ([(64, 0), (70, 900)], 7), ([(130, 3), (33, 300), (0, 40)], 1)])
def test_batches_of_one_kernel(lens, grp):
    run(Batch8(lens, G=2, grp=grp, ps=64, pad=3))


@pytest.mark.parametrize("n", [30, 64, 100, 333])
def test_many_ragged_chunks(n):
    """More units than CTAs, cut or not, and single tokens beside them."""
    lens = [(1 + (i * 7919 + n) % n, (i * 104729) % 700) for i in range(12)] + [(1, 900), (1, 5)]
    run(Batch8(lens, G=4, grp=7, ps=16))


def set_new(b, new):
    """The same sequences with other numbers of new tokens, in place."""
    b.lens = [(n, k - n) for n, k in zip(new, b.len)]
    b.start = [0]
    for n in new:
        b.start.append(b.start[-1] + n)
    b.total = b.start[-1]
    b.row_start.copy_(torch.tensor(b.start, dtype=torch.int32))


@pytest.mark.parametrize("rows", [3, 64])
def test_nothing_new(rows):
    """Rows that belong to no sequence only."""
    b = Batch8([(0, 40), (0, 3), (0, 0), (0, 700)], G=2, grp=4, pad=rows)
    b.mass.copy_(b.mass.nan_to_num(0.5))
    before = b.mass.clone()
    q = b.rows(b.H).contiguous()
    out, lse, ws = torch.full_like(q, 7.0), torch.full((b.T, b.H), 7.0, device="cuda"), b.workspace()
    for _ in range(2):
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, out, lse, b.status, ws))
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))
    assert b.status.item() == 0 and (out == 7).all() and (lse == 7).all() and torch.equal(before, b.mass)


def test_a_captured_step_takes_every_mixture():
    """One graph for 64 rows: a chunk, single tokens, nothing, both, in any order; rows of no sequence are left alone."""
    b = Batch8([(1, 99), (1, 299), (1, 63), (1, 4), (0, 0), (1, 699)], G=2, grp=4, ps=32, pad=59)
    assert b.T == 64
    q = b.rows(b.H).contiguous()
    out, lse, ws = torch.empty_like(q), torch.empty((64, b.H), device="cuda"), b.workspace()
    mass0 = b.mass.nan_to_num(0.5)

    def step():
        V.check(V.varrate_paged8_attn(b.pages, b.seqs, 0, b.grp, q, out, lse, b.status, ws))
        V.check(V.varrate_paged8_mass(b.pages, b.seqs, 0, b.grp, q, lse, b.status))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for new in ([0, 64, 0, 0, 0, 0], [1, 1, 1, 1, 0, 1], [0] * 6, [2, 30, 0, 5, 0, 1], [0, 0, 0, 0, 0, 64], [0, 0, 0, 1, 0, 0],
                [10, 10, 10, 5, 0, 10]):
        set_new(b, new)
        out.fill_(7.0)
        lse.fill_(7.0)
        b.mass.copy_(mass0)
        graph.replay()
        assert b.status.item() == 0, new
        want, tol, want_lse, tol_lse = attn8_ref(b, q)
        close(out, want, tol)
        close(lse, want_lse, tol_lse)
        assert (out[b.total:] == 7).all() and (lse[b.total:] == 7).all()
        w, allowed = mass8_ref(b, q, lse, mass0)
        close(b.mass, w, allowed)
