"""Paged cache in 8 bits: calls of the kinds that its other tests do not make."""
import pytest
import torch

from paged8_helpers import Batch8, mass8_ref
from paged_helpers import close
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
