"""Edges of the paged calls on the GPU: headers of the workspace that a call may find. Tolerances are derived in
paged_helpers."""
import pytest
import torch

from paged_helpers import V, Batch
from test_gpu_paged import run_attn, status

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu(vlib):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")


# ------------------------------------------------------------------------------------ the header of the workspace

def ctas(dtype):
    return torch.cuda.get_device_properties(0).multi_processor_count * (1 if dtype == "bf16" else 2)


def found(b, ws, words):
    """A call that finds `words` at the start of the workspace raises CORRUPT; the call after it is right."""
    head = ws[:4 * len(words)].view(torch.int32)
    head.copy_(torch.tensor(words, dtype=torch.int32))
    q = b.rows(b.H)
    assert V.varrate_paged_attn(b.pages, b.seqs, 0, b.grp, q, torch.zeros_like(q), b.status, ws) == V.OK
    assert status(b) == V.ERR_CORRUPT
    b.status.zero_()
    run_attn(b, ws=ws, q=q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_counter_found_used_with_units_left_to_take(dtype):
    """More units than CTAs (one key tile a sequence, so a unit is a sequence and a head): a count that is not zero takes units
    away without the counter's end showing it."""
    units, C = 1000, ctas(dtype)
    assert C < units
    b = Batch([(1, s % 30) for s in range(units // 2)], dtype, 2, 4)
    ws = b.workspace()
    for count in (1, 3, units - C - 1, units - C, units - C + 1, units - 1, units):
        found(b, ws, [count])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attn_counter_found_used_by_a_long_prompt(dtype):
    b = Batch([(3000, 100), (1, 2000)], dtype, 4, 2)
    ws = b.workspace()
    for count in (1, 3, 100):
        found(b, ws, [count])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count", [0, 1, 3, 100, 1000])
def test_attn_header_never_zeroed(dtype, count):
    """Every word of the header holds something, as a call whose merge was never launched leaves it."""
    b = Batch([(1, s % 30) for s in range(500)], dtype, 2, 4)
    found(b, b.workspace(), [count, 0, 1, 1000, 0, 1000, 1, 1])
