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
