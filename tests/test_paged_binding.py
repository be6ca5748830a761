"""What the paged-cache calls refuse on the host, beside test_paged_abi.py (no GPU needed)."""
import ctypes

import pytest
import torch

from test_paged_abi import append, structs


@pytest.mark.parametrize("eps, want", [(1e39, -1), (1e300, -1), (3e38, 0), (1e-300, 0), (0.0, 0)])
def test_eps_is_finite_in_fp32(vlib, eps, want):
    assert append(vlib, *structs(vlib, n_rows=0), eps=eps) == want


class OnGpu(torch.Tensor):
    """A tensor in host memory that says it is on a GPU: for calls that are stopped before a launch or end in a stand-in."""
    index = 1

    def get_device(self):
        return self.index


def on(t, index):
    t = t.as_subclass(OnGpu)
    t.index = index
    return t


@pytest.fixture
def calls(vlib, monkeypatch):
    """The binding's calls on device 1 with a stand-in for the library: what reached it."""
    made = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(vlib, "_lib", Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)

    def call(name, at=1, seqs_at=1, status_at=1, ws_at=1, status_type=torch.int32, ws_step=1):
        V = vlib
        t = lambda *shape: on(torch.zeros(shape, dtype=torch.bfloat16), at)   # noqa: E731
        i32 = lambda *x: on(torch.tensor(x, dtype=torch.int32), seqs_at)      # noqa: E731
        pages = V.PagedCache.of(t(1, 4, 2, 2, 16, 128))
        seqs = V.SeqBatch.of(i32(0, 1, 3), i32(1, 5), on(torch.zeros((2, 2), dtype=torch.int32), seqs_at), 3)
        st = None if status_at is None else on(torch.zeros(1, dtype=status_type), status_at)
        ws = on(torch.zeros(512, dtype=torch.uint8)[::ws_step], ws_at)
        q, k = t(3, 4, 128), t(3, 2, 128)
        made.clear()
        if name == "append":
            got = V.varrate_paged_append(pages, seqs, 0, q, k, k, None, None, 1e-6, None, 0, t(3, 4, 128), st, stream=0)
        elif name == "attn":
            got = V.varrate_paged_attn(pages, seqs, 0, 2, q, t(3, 4, 128), st, ws, stream=0)
        else:
            got = V.varrate_paged_gather(pages, seqs, 0, 1, None, 5, t(2, 1, 2, 5, 128), None, st, stream=0)
        return got, len(made)

    return call


@pytest.mark.parametrize("name", ["append", "attn", "gather"])
def test_everything_on_the_cache_s_device(vlib, calls, name):
    """Tables, status word and workspace that are on the CPU or on another GPU are refused before anything is enqueued."""
    assert calls(name) == (vlib.OK, 1) and calls(name, status_at=None) == (vlib.OK, 1)
    for other in (-1, 0):
        assert calls(name, seqs_at=other) == (vlib.ERR_ARG, 0)
        assert calls(name, status_at=other) == (vlib.ERR_ARG, 0)
        if name == "attn":
            assert calls(name, ws_at=other) == (vlib.ERR_ARG, 0)
    assert calls(name, status_type=torch.int64) == (vlib.ERR_ARG, 0)
    assert calls("attn", ws_step=2) == (vlib.ERR_ARG, 0)
    assert calls(name, at=-1, seqs_at=-1, status_at=-1, ws_at=-1) == (vlib.ERR_ARG, 0)     # a cache on the CPU


def test_tables_on_one_device(vlib):
    i32 = lambda at, *x: on(torch.tensor(x, dtype=torch.int32), at)   # noqa: E731
    tables = [i32(1, 0, 1, 3), i32(1, 1, 5), i32(1, 0, 0, 0, 0).view(2, 2)]
    tables[2].index = 1
    assert vlib.SeqBatch.of(*tables, 3).device == 1
    for i in range(3):
        moved = list(tables)
        moved[i] = tables[i].clone()
        moved[i].index = 0
        with pytest.raises(vlib.VarrateError):
            vlib.SeqBatch.of(*moved, 3)


def test_a_batch_without_tables(vlib):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    table = torch.zeros((2, 2), dtype=torch.int32)
    for bad in ((i32(0, 1, 3), None, table), (i32(0, 1, 3), i32(1, 5), None), (i32(0, 1, 3), i32(1, 5), table.view(4)),
                (i32(0, 1, 3), i32(1, 5), torch.zeros((), dtype=torch.int32))):
        with pytest.raises(vlib.VarrateError):
            vlib.SeqBatch.of(*bad, 3)
    assert vlib.SeqBatch.of(None, i32(1, 5), table, 3).n_seqs == 2      # to gather


def test_workspace_size_goes_by_rows_group_and_type(vlib):
    """Not by sequences or pages; never less for more rows."""
    def size(dtype=vlib.BF16, group=4, **kw):
        p, s = structs(vlib, dtype, **kw)
        return vlib.lib().varrate_paged_attn_ws_bytes(ctypes.byref(p), ctypes.byref(s), group)

    for dtype in (vlib.BF16, vlib.F32):
        for group in (1, 3, 8):
            assert size(dtype, group) == size(dtype, group, n_seqs=900, max_pages=70) == size(dtype, group, n_pages=77)
            sizes = [size(dtype, group, n_rows=n) for n in (0, 1, 7, 40, 128, 129, 500, 10 ** 6)]
            assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]
    assert size(vlib.BF16) != size(vlib.F32) and size(group=1) != size(group=8)
