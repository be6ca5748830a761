"""What the paged-cache calls refuse on the host, beside test_paged_abi.py (no GPU needed)."""
import pytest

from test_paged_abi import append, structs


@pytest.mark.parametrize("eps, want", [(1e39, -1), (1e300, -1), (3e38, 0), (1e-300, 0), (0.0, 0)])
def test_eps_is_finite_in_fp32(vlib, eps, want):
    assert append(vlib, *structs(vlib, n_rows=0), eps=eps) == want
