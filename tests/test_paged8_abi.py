"""What the calls of the 8-bit paged cache refuse on the host, before a kernel is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from test_paged_binding import on

A = 1 << 12   # a 16-byte aligned fake device pointer, never dereferenced


def structs(V, **kw):
    p = V.varrate_pages8(A, A, A, 2, 10, 4, 64, 128)
    s = V.varrate_seqs(A, A, A, 3, 5, 40)
    for name, value in kw.items():
        setattr(p if hasattr(p, name) else s, name, value)
    return p, s


def append(V, p, s, layer=0, group=4, q=A, qs=2048, k=A, ks=512, v=A, vs=512, wq=None, wk=None, eps=1e-6, freq=A,
           rot=128, gone=None, q_out=2 * A, status=None):
    return V.lib().varrate_paged8_append(ctypes.byref(p), ctypes.byref(s), layer, group, q, qs, k, ks, v, vs, wq, wk,
                                         eps, freq, rot, gone, q_out, status, None)


def attn(V, p, s, layer=0, group=4, q=A, out=2 * A, lse=A, status=None, ws=A, n=1 << 40):
    return V.lib().varrate_paged8_attn(ctypes.byref(p), ctypes.byref(s), layer, group, q, out, lse, status, ws, n, None)


def mass(V, p, s, layer=0, group=4, q=A, lse=A, status=None):
    return V.lib().varrate_paged8_mass(ctypes.byref(p), ctypes.byref(s), layer, group, q, lse, status, None)


def evict(V, p, s, layer=0, layers=1, budget=8, first=2, last=3, kept=A, new=2 * A, gone=None, status=None):
    return V.lib().varrate_paged8_evict(ctypes.byref(p), ctypes.byref(s), layer, layers, budget, first, last, kept, new, gone,
                                        status, None)


@pytest.mark.parametrize("field, value, want", [
    ("head_dim", 64, -5), ("page_size", 8, -5), ("page_size", 48, -5), ("page_size", 512, -5), ("page_size", 0, -1),
    ("n_pages", 0, -1), ("n_layers", 0, -1), ("n_kv_heads", 0, -1), ("n_seqs", -1, -1), ("n_rows", -1, -1),
    ("max_pages", 0, -1), ("codes", 0, -1), ("codes", A + 8, -1), ("scale", 0, -1), ("scale", A + 1, -1), ("mass", A + 4, -1),
    ("kv_len", 0, -1), ("page_table", 0, -1), ("kv_len", A + 4, -1), ("n_pages", 2 ** 30, -5), ("n_kv_heads", 4097, -5)])
def test_bad_descriptions(vlib, field, value, want):
    for call in (append, attn, mass, evict):
        assert call(vlib, *structs(vlib, **{field: value})) == want, call.__name__
    if field not in ("codes", "scale", "mass", "kv_len", "page_table"):
        p, s = structs(vlib, **{field: value})
        assert vlib.lib().varrate_paged8_attn_ws_bytes(ctypes.byref(p), ctypes.byref(s), 4) == 0


def test_null_descriptions(vlib):
    L = vlib.lib()
    p, s = structs(vlib)
    assert L.varrate_paged8_attn(None, ctypes.byref(s), 0, 4, A, 2 * A, None, None, A, 1 << 40, None) == vlib.ERR_ARG
    assert L.varrate_paged8_mass(ctypes.byref(p), None, 0, 4, A, A, None, None) == vlib.ERR_ARG
    assert L.varrate_paged8_attn_ws_bytes(None, None, 4) == 0


@pytest.mark.parametrize("kw, want", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(group=0), -1), (dict(group=9, qs=1 << 20), -5), (dict(k=None), -1),
    (dict(v=None), -1), (dict(q_out=None), -1), (dict(qs=2040), -1), (dict(qs=2052), -1), (dict(ks=504), -1),
    (dict(vs=516), -1), (dict(rot=8), -1), (dict(rot=144), -1), (dict(rot=-16), -1), (dict(freq=None), -1),
    (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1), (dict(eps=1e39), -1), (dict(k=A + 8), -1),
    (dict(freq=A + 8), -1), (dict(wq=A + 2), -1), (dict(status=A + 4), -1), (dict(q_out=A, qs=2056), -1), (dict(gone=A + 4), -1)])
def test_append_refuses(vlib, kw, want):
    assert append(vlib, *structs(vlib), **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(layer=2), -1), (dict(group=0), -1), (dict(group=9), -5), (dict(q=None), -1), (dict(out=None), -1),
    (dict(q=A, out=A), -1), (dict(ws=None), -2), (dict(n=8), -2), (dict(out=A + 8), -1), (dict(ws=A + 8), -1),
    (dict(lse=A + 4), -1)])
def test_attn_refuses(vlib, kw, want):
    assert attn(vlib, *structs(vlib), **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(layer=2), -1), (dict(layer=-1), -1), (dict(group=0), -1), (dict(group=9), -5), (dict(q=None), -1),
    (dict(lse=None), -1), (dict(q=A + 8), -1), (dict(lse=A + 4), -1), (dict(status=A + 4), -1)])
def test_mass_refuses(vlib, kw, want):
    assert mass(vlib, *structs(vlib), **kw) == want


@pytest.mark.parametrize("kw, want", [
    (dict(layer=1, layers=2), -1), (dict(layers=0), -1), (dict(layer=-1), -1), (dict(layer=2 ** 31 - 1), -1), (dict(budget=0), -1),
    (dict(first=-1), -1), (dict(last=-1), -1), (dict(first=6), -1), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1, budget=2 ** 31 - 1), -1),
    (dict(kept=None), -1), (dict(new=None), -1), (dict(new=A), -1), (dict(gone=2 * A), -1), (dict(kept=A + 4), -1),
    (dict(status=A + 4), -1)])
def test_evict_refuses(vlib, kw, want):
    assert evict(vlib, *structs(vlib), **kw) == want


def test_weights_have_to_be_there(vlib):
    p, s = structs(vlib, mass=None)
    assert mass(vlib, p, s) == vlib.ERR_ARG and evict(vlib, p, s) == vlib.ERR_ARG


def test_row_start_is_not_needed_to_evict(vlib):
    p, s = structs(vlib, row_start=0)
    assert append(vlib, p, s) == attn(vlib, p, s) == mass(vlib, p, s) == vlib.ERR_ARG
    p, s = structs(vlib, row_start=0, n_seqs=0)
    assert evict(vlib, p, s) == vlib.OK


def test_nothing_to_do_is_ok(vlib):
    for kw in (dict(n_seqs=0), dict(n_rows=0)):
        p, s = structs(vlib, codes=0, scale=0, mass=0, kv_len=0, page_table=0, row_start=0, **kw)
        assert append(vlib, p, s, q=None, k=None, v=None, q_out=None) == vlib.OK
        assert attn(vlib, p, s, q=None, out=None, ws=None, n=0) == vlib.OK
        assert mass(vlib, p, s, q=None, lse=None) == vlib.OK
    assert evict(vlib, *structs(vlib, codes=0, scale=0, mass=0, kv_len=0, page_table=0, n_seqs=0), kept=None, new=None) == vlib.OK


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


@pytest.mark.parametrize("codes, scale, mass", [
    (u8(1, 4, 2, 2, 16, 128), u8(1, 4, 2, 2, 2), None), (u8(1, 4, 3, 2, 16, 128), u8(1, 4, 3, 2, 1), None),
    (u8(4, 2, 2, 16, 128), u8(4, 2, 2, 1), None), (u8(1, 4, 2, 2, 24, 128), u8(1, 4, 2, 2, 1), None),
    (u8(1, 4, 2, 2, 16, 128).bfloat16(), u8(1, 4, 2, 2, 1), None), (u8(1, 4, 2, 2, 16, 128), u8(1, 4, 2, 2, 1).float(), None),
    (u8(1, 4, 2, 2, 16, 128), u8(1, 4, 2, 2, 1), u8(1, 4, 2, 16)), (u8(1, 4, 2, 2, 16, 128), u8(1, 4, 2, 2, 1), u8(1, 4, 16).float()),
    (u8(1, 4, 2, 2, 16, 256)[..., ::2], u8(1, 4, 2, 2, 1), None)])
def test_cache_is_refused(vlib, codes, scale, mass):
    with pytest.raises(vlib.VarrateError):
        vlib.Paged8Cache.of(codes, scale, mass)


def test_cache_takes_both_kinds_of_bytes(vlib):
    V = vlib
    c = V.Paged8Cache.allocate(2, 4, 3, 32, device="cpu")
    assert (c.codes.dtype, c.scale.dtype) == (torch.float8_e4m3fn, torch.float8_e8m0fnu) and c.mass.shape == (2, 4, 3, 32)
    assert V.Paged8Cache.of(c.codes.view(torch.uint8), c.scale.view(torch.uint8)).c.mass is None
    assert V.Paged8Cache.allocate(2, 4, 3, 32, mass=False, device="cpu").mass is None


@pytest.fixture
def calls(vlib, monkeypatch):
    """The binding's calls on device 1 with a stand-in for the library: what came back, and how many reached it."""
    made = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(vlib, "_lib", Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    V = vlib
    t = lambda *shape, dt=torch.bfloat16, at=1: on(torch.zeros(shape, dtype=dt), at)   # noqa: E731
    i32, f32 = dict(dt=torch.int32), dict(dt=torch.float32)
    pages = V.Paged8Cache.of(t(1, 4, 2, 2, 16, 128, dt=torch.uint8), t(1, 4, 2, 2, 1, dt=torch.uint8), t(1, 4, 2, 16, **f32))
    seqs = V.SeqBatch.of(t(3, **i32), t(2, **i32), t(2, 2, **i32), 3)
    base = {
        "append": (V.varrate_paged8_append, dict(q=t(3, 4, 128), k=t(3, 2, 128), v=t(3, 2, 128), q_norm=None, k_norm=t(128), eps=0.0,
                                                 freq=t(64, dt=torch.float64), rot_dim=128, gone=t(2, **i32), q_out=t(3, 4, 128))),
        "attn": (V.varrate_paged8_attn, dict(group=2, q=t(3, 4, 128), out=t(3, 4, 128), lse=t(3, 4, **f32), ws=t(512, dt=torch.uint8))),
        "mass": (V.varrate_paged8_mass, dict(group=2, q=t(3, 4, 128), lse=t(3, 4, **f32))),
        "evict": (V.varrate_paged8_evict, dict(n_layers=1, budget=5, n_first=0, n_last=0, kept=t(2, 1, 2, 5, **i32), new_len=t(2, **i32),
                                               gone=t(2, **i32)))}

    def call(name, status=t(1, **i32), **kw):
        made.clear()
        f, args = base[name]
        got = f(pages, seqs, 0, dev_status=status, stream=0, **{**args, **kw})
        return got, len(made)

    call.t, call.i32, call.f32 = t, i32, f32
    return call


def test_binding_takes_what_is_right(calls):
    for name, kw in (("append", {}), ("append", dict(q=None, q_out=None, gone=None)), ("attn", {}), ("attn", dict(lse=None)),
                     ("mass", {}), ("evict", {}), ("evict", dict(gone=None)), ("mass", dict(status=None))):
        assert calls(name, **kw) == (0, 1), (name, kw)


def test_binding_refuses(calls):
    t, i32, f32 = calls.t, calls.i32, calls.f32
    for name, kw in [
            ("append", dict(q=t(3, 4, 128, **f32))), ("append", dict(k=t(2, 2, 128))), ("append", dict(gone=t(3, **i32))),
            ("append", dict(gone=t(2, **f32))), ("append", dict(gone=t(2, at=0, **i32))), ("append", dict(q_out=t(3, 2, 128))),
            ("append", dict(freq=t(10, dt=torch.float64))), ("append", dict(status=t(1, at=0, **i32))),
            ("attn", dict(lse=t(3, 4))), ("attn", dict(lse=t(4, 3, **f32))), ("attn", dict(lse=t(3, 4, at=0, **f32))),
            ("attn", dict(q=t(3, 4, 128, at=0))), ("attn", dict(group=3)), ("attn", dict(ws=t(512, dt=torch.uint8, at=0))),
            ("attn", dict(out=None)), ("mass", dict(lse=None)), ("mass", dict(q=t(3, 2, 128))), ("mass", dict(status=t(1, **f32))),
            ("evict", dict(kept=t(2, 1, 2, 4, **i32))), ("evict", dict(kept=None)), ("evict", dict(new_len=None)),
            ("evict", dict(new_len=t(3, **i32))), ("evict", dict(gone=t(1, **i32))), ("evict", dict(kept=t(2, 1, 2, 5, at=0, **i32)))]:
        assert calls(name, **kw) == (-1, 0), (name, list(kw))
