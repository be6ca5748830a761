"""What the paged-cache calls refuse on the host, before a kernel is launched (no GPU needed)."""
import ctypes

import pytest
import torch

A = 1 << 12   # a 16-byte aligned fake device pointer, never dereferenced


def structs(V, dtype=None, **kw):
    p = V.varrate_pages(A, 2, 10, 4, 64, 128, V.BF16 if dtype is None else dtype)
    s = V.varrate_seqs(A, A, A, 3, 5, 40)
    for name, value in kw.items():
        setattr(p if hasattr(p, name) else s, name, value)
    return p, s


def append(V, p, s, layer=0, group=4, q=A, qs=2048, k=A, ks=512, v=A, vs=512, wq=None, wk=None, eps=1e-6, freq=A,
           rot=128, q_out=2 * A, status=None):
    return V.lib().varrate_paged_append(ctypes.byref(p), ctypes.byref(s), layer, group, q, qs, k, ks, v, vs, wq, wk,
                                        eps, freq, rot, q_out, status, None)


def attn(V, p, s, layer=0, group=4, q=A, out=2 * A, status=None, ws=A, n=1 << 40):
    return V.lib().varrate_paged_attn(ctypes.byref(p), ctypes.byref(s), layer, group, q, out, status, ws, n, None)


def gather(V, p, s, layer=0, layers=1, first=None, n=7, k=A, v=A, status=None):
    return V.lib().varrate_paged_gather(ctypes.byref(p), ctypes.byref(s), layer, layers, first, n, k, v, status, None)


@pytest.mark.parametrize("field, value, want", [
    ("head_dim", 64, -5), ("page_size", 8, -5), ("page_size", 48, -5), ("page_size", 512, -5), ("page_size", 0, -1),
    ("n_pages", 0, -1), ("n_layers", 0, -1), ("n_kv_heads", 0, -1), ("dtype", 2, -1), ("n_seqs", -1, -1),
    ("n_rows", -1, -1), ("max_pages", 0, -1), ("pool", 0, -1), ("pool", A + 8, -1), ("kv_len", 0, -1),
    ("page_table", 0, -1), ("kv_len", A + 4, -1), ("n_pages", 2 ** 30, -5), ("n_kv_heads", 4097, -5)])
def test_bad_descriptions(vlib, field, value, want):
    for call in (append, attn, gather):
        assert call(vlib, *structs(vlib, **{field: value})) == want
    p, s = structs(vlib, **{field: value})
    if field not in ("pool", "kv_len", "page_table"):
        assert vlib.lib().varrate_paged_attn_ws_bytes(ctypes.byref(p), ctypes.byref(s), 4) == 0


def test_null_descriptions(vlib):
    L = vlib.lib()
    p, s = structs(vlib)
    assert L.varrate_paged_attn(None, ctypes.byref(s), 0, 4, A, 2 * A, None, A, 1 << 40, None) == vlib.ERR_ARG
    assert L.varrate_paged_attn(ctypes.byref(p), None, 0, 4, A, 2 * A, None, A, 1 << 40, None) == vlib.ERR_ARG
    assert L.varrate_paged_attn_ws_bytes(None, None, 4) == 0


@pytest.mark.parametrize("kw, want", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(group=0), -1), (dict(group=9, qs=1 << 20), -5), (dict(k=None), -1),
    (dict(v=None), -1), (dict(q_out=None), -1), (dict(qs=2040), -1), (dict(qs=2052), -1), (dict(ks=504), -1),
    (dict(vs=516), -1), (dict(rot=8), -1), (dict(rot=144), -1), (dict(rot=-16), -1), (dict(freq=None), -1),
    (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(k=A + 8), -1),
    (dict(freq=A + 8), -1), (dict(wq=A + 2), -1), (dict(status=A + 4), -1), (dict(q_out=A, qs=2056), -1)])
def test_append_refuses(vlib, kw, want):
    assert append(vlib, *structs(vlib), **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(layer=2), -1), (dict(group=0), -1), (dict(group=9), -5), (dict(q=None), -1), (dict(out=None), -1),
    (dict(q=A, out=A), -1), (dict(ws=None), -2), (dict(n=8), -2), (dict(out=A + 8), -1), (dict(ws=A + 8), -1)])
def test_attn_refuses(vlib, kw, want):
    for dtype in (vlib.BF16, vlib.F32):
        assert attn(vlib, *structs(vlib, dtype), **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(layer=1, layers=2), -1), (dict(layers=0), -1), (dict(layer=-1), -1), (dict(n=-1), -1), (dict(k=A + 8), -1),
    (dict(first=A + 4), -1), (dict(layer=2 ** 31 - 1), -1)])
def test_gather_refuses(vlib, kw, want):
    assert gather(vlib, *structs(vlib), **kw) == want


def test_row_start_is_not_needed_to_gather_but_to_append_and_attend(vlib):
    p, s = structs(vlib, row_start=0)
    assert append(vlib, p, s) == vlib.ERR_ARG and attn(vlib, p, s) == vlib.ERR_ARG
    assert gather(vlib, p, s, n=0) == vlib.OK


def test_nothing_to_do_is_ok(vlib):
    """No sequence, no row or no token: nothing is looked at, nothing is enqueued."""
    for kw in (dict(n_seqs=0), dict(n_rows=0)):
        p, s = structs(vlib, pool=0, kv_len=0, page_table=0, row_start=0, **kw)
        assert append(vlib, p, s, q=None, k=None, v=None, q_out=None) == vlib.OK
        assert attn(vlib, p, s, q=None, out=None, ws=None, n=0) == vlib.OK
    p, s = structs(vlib)
    assert gather(vlib, p, s, n=0) == vlib.OK and gather(vlib, p, s, k=None, v=None) == vlib.OK


def test_binding_looks_at_tensors(vlib):
    """Types, shapes and strides that the C call cannot see."""
    V = vlib
    pool = torch.zeros((1, 4, 2, 2, 16, 128), dtype=torch.bfloat16)
    pages = V.PagedCache.of(pool)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    seqs = V.SeqBatch.of(i32(0, 1, 3), i32(1, 5), torch.zeros((2, 2), dtype=torch.int32), 3)
    q, k = torch.zeros((3, 4, 128), dtype=torch.bfloat16), torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    freq = torch.zeros(64, dtype=torch.float64)
    st = torch.zeros(1, dtype=torch.int32)

    def ap(q=q, k=k, v=k, wq=None, freq=freq, q_out=q.clone()):
        return V.varrate_paged_append(pages, seqs, 0, q, k, v, wq, None, 1e-6, freq, 128, q_out, st, stream=0)

    assert ap(q=q.float()) == V.ERR_ARG
    assert ap(k=k[:2]) == V.ERR_ARG
    assert ap(v=torch.zeros((3, 128, 2), dtype=torch.bfloat16).transpose(1, 2)) == V.ERR_ARG
    assert ap(q=torch.zeros((3, 3, 128), dtype=torch.bfloat16)) == V.ERR_ARG
    assert ap(wq=torch.ones(128)) == V.ERR_ARG
    assert ap(freq=freq.float()) == V.ERR_ARG and ap(freq=freq[:8]) == V.ERR_ARG
    assert ap(q_out=torch.zeros((3, 8, 128), dtype=torch.bfloat16)[:, ::2]) == V.ERR_ARG
    assert V.varrate_paged_attn(pages, seqs, 0, 2, q[:, ::2], q, st, q, stream=0) == V.ERR_ARG
    out = torch.zeros((2, 1, 2, 5, 128), dtype=torch.bfloat16)
    assert V.varrate_paged_gather(pages, seqs, 0, 1, None, 4, out, out, st, stream=0) == V.ERR_ARG
    assert V.varrate_paged_gather(pages, seqs, 0, 1, torch.zeros(2), 5, out, out, st, stream=0) == V.ERR_ARG
    with pytest.raises(V.VarrateError):
        V.SeqBatch.of(i32(0, 1, 3), i32(1, 5), torch.zeros((2, 2), dtype=torch.int64), 3)
    with pytest.raises(V.VarrateError):
        V.SeqBatch.of(i32(0, 3), i32(1, 5), torch.zeros((2, 2), dtype=torch.int32), 3)
    with pytest.raises(V.VarrateError):
        V.PagedCache.of(pool.transpose(3, 4))


def test_binding_refuses_what_is_missing(vlib):
    V = vlib
    pages = V.PagedCache.of(torch.zeros((1, 4, 2, 2, 16, 128), dtype=torch.bfloat16))
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)   # noqa: E731
    seqs = V.SeqBatch.of(i32(0, 1, 3), i32(1, 5), torch.zeros((2, 2), dtype=torch.int32), 3)
    q, k = torch.zeros((3, 4, 128), dtype=torch.bfloat16), torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    freq, st = torch.zeros(64, dtype=torch.float64), torch.zeros(1, dtype=torch.int32)
    for a in ((q, None, k, freq, q), (q, k, None, freq, q), (q, k, k, None, q), (q, k, k, freq, None), (q[0], k, k, freq, q)):
        assert V.varrate_paged_append(pages, seqs, 0, *a[:3], None, None, 1e-6, a[3], 128, a[4], st, stream=0) == V.ERR_ARG
    assert V.varrate_paged_attn(pages, seqs, 0, 2, None, q, st, q, stream=0) == V.ERR_ARG
    assert V.varrate_paged_attn(pages, seqs, 0, 2, q, None, st, q, stream=0) == V.ERR_ARG
    assert V.varrate_paged_attn(pages, seqs, 0, 2, q, q.clone(), st, None, stream=0) == V.ERR_WORKSPACE


def test_rows_apart_in_every_form(vlib):
    """Distance of the rows of a tensor: parts of wider rows, one head, and one row, of which it can be any number."""
    pages = vlib.PagedCache.of(torch.zeros((1, 1, 2, 1, 16, 128), dtype=torch.bfloat16))
    x = torch.zeros((5, 8, 128), dtype=torch.bfloat16)
    assert pages.row_stride(x, 5, 8) == 1024 and pages.row_stride(x[:, 2:4], 5, 2) == 1024
    assert pages.row_stride(x[:, 3:4], 5, 1) == 1024 and pages.row_stride(x[:, 3:4].transpose(0, 1), 1, 5) == -1
    assert pages.row_stride(x.view(5, 1, 1024)[:, :, 128:256], 5, 1) == 1024
    assert pages.row_stride(x[::2], 3, 8) == 2048 and pages.row_stride(x[:, ::2], 5, 4) == -1
    one = torch.zeros((8, 1, 128), dtype=torch.bfloat16).transpose(0, 1)      # [1][8][d] with 128 from row to row
    assert one.stride(0) == 128 and pages.row_stride(one, 1, 8) == 1024


def test_calls_run_with_the_cache_s_device_as_the_current_one(vlib, monkeypatch):
    V = vlib
    entered, current = [], [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *a):
            entered.append(None)

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    pages = V.PagedCache.of(torch.zeros((1, 4, 2, 2, 16, 128), dtype=torch.bfloat16))
    call = lambda *a: entered.append(a) or 5   # noqa: E731
    assert V._on_device(pages, call, 1, 2) == 5 and entered == [(1, 2)]          # on the CPU: as it is
    pages.device = 1
    entered.clear()
    assert V._on_device(pages, call, 7) == 5 and entered == [1, (7,), None]
    current[0] = 1
    entered.clear()
    assert V._on_device(pages, call, 7) == 5 and entered == [(7,)]
