"""Size of the 8-bit attention's workspace (no GPU needed)."""
import ctypes

import pytest

from test_paged8_abi import structs


@pytest.mark.parametrize("group", [1, 3, 4, 5, 8])
def test_size_goes_by_rows_and_group(vlib, group):
    """Not by sequences or pages; never less for more rows."""
    def size(**kw):
        p, s = structs(vlib, **kw)
        return vlib.lib().varrate_paged8_attn_ws_bytes(ctypes.byref(p), ctypes.byref(s), group)

    rows = (0, 1, 2, 3, 4, 5, 8, 9, 16, 17, 20, 40, 64, 128, 129, 500, 512, 10 ** 6)
    for n in rows:
        assert size(n_rows=n) == size(n_rows=n, n_seqs=1) == size(n_rows=n, n_seqs=900, max_pages=70) == size(n_rows=n, n_pages=77)
    sizes = [size(n_rows=n) for n in rows]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]
