"""Thin Python binding of the VarRate C ABI (include/varrate.h).

Argument marshalling only: every step of the hot path runs in the CUDA library ``libvarrate.so``.
Functions keep the C names and argument order; tensor arguments are torch tensors (device memory
owned by the caller) or ``None`` for NULL, and ``stream`` defaults to torch's current stream.
Importing this module does not load the library; the first call does, and it raises if the
library has not been built (there is no CPU fallback).

Typical use (one encode of a prompt's cache, then one decode call per layer and step)::

    cfg = make_config(n_layers, n_kv_heads, group, n_ctx, batch=B, budget_frac=0.2, r_min=16,
                      window=32, dtype=BF16)
    packed = PackedCache.allocate(cfg, "cuda")            # static upper bound: no host sync later
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    check(varrate_encode(cfg, q_win, k, v, basis_k, basis_v, None, packed, None, status,
                         workspace(cfg, CALL_ENCODE)), "varrate_encode")
    ws = workspace(cfg, CALL_DECODE)                      # zero-filled; reusable by every decode call
    check(varrate_decode_attn(cfg, packed, basis_k, basis_v, q, layer, None, None, 0, out, status,
                              ws), "varrate_decode_attn")
    # after a synchronise: status.item() is OK (0), FLOOR_BINDS (1) or a negative error

While a prompt is prefilled its keys and values stand in the pages of a PagedCache::

    pages, seqs = PagedCache.allocate(n_layers, n_pages, n_kv_heads, 64), SeqBatch.of(row_start, kv_len, table, n_rows)
    ws = paged_attn_workspace(pages, seqs, group)         # zero-filled; reusable by every call on the stream
    check(varrate_paged_append(pages, seqs, layer, q, k, v, q_norm, k_norm, eps, freq, rot_dim, q_out, status))
    check(varrate_paged_attn(pages, seqs, layer, group, q_out, out, status, ws))
    check(varrate_paged_gather(pages, seqs, 0, n_layers, None, n, k, v, status))   # for varrate_encode

Shapes: q_win [B][L][w][H][d], k and v [B][L][G][N][d], bases [L][G][d][d] (row j = basis vector
j), q and out [B][H][d]; every tensor contiguous on the GPU and 16-byte aligned.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvarrate.so")

OK, FLOOR_BINDS = 0, 1
ERR_ARG, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED, ERR_CORRUPT = -1, -2, -3, -4, -5, -6
F32, BF16 = 0, 1
SALIENCE, UNIFORM = 0, 1
CALL_SALIENCE, CALL_PACK, CALL_ENCODE, CALL_DECODE, CALL_DECODE_WINDOW, CALL_DECODE_Q = 0, 1, 2, 3, 4, 5

_c_void_p = ctypes.c_void_p


class varrate_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("group", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_ctx", ctypes.c_int64), ("batch", ctypes.c_int32), ("r_min", ctypes.c_int32),
                ("budget_frac", ctypes.c_double), ("window", ctypes.c_int32),
                ("pool_len", ctypes.c_int32), ("dtype", ctypes.c_int32), ("mode", ctypes.c_int32)]


class varrate_packed(ctypes.Structure):
    _fields_ = [("coef", _c_void_p), ("bucket_count", _c_void_p), ("bucket_base", _c_void_p),
                ("perm", _c_void_p), ("pos", _c_void_p), ("ranks", _c_void_p),
                ("cap_elems", ctypes.c_int64)]


class varrate_qpacked(ctypes.Structure):
    _fields_ = [("data", _c_void_p), ("qbase", _c_void_p), ("bucket_count", _c_void_p),
                ("bits", ctypes.c_int32), ("qcap_bytes", ctypes.c_int64)]


class varrate_pages(ctypes.Structure):
    _fields_ = [("pool", _c_void_p), ("n_layers", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class varrate_seqs(ctypes.Structure):
    _fields_ = [("row_start", _c_void_p), ("kv_len", _c_void_p), ("page_table", _c_void_p),
                ("n_seqs", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_rows", ctypes.c_int32)]


_lib = None

_SIGS = {
    "varrate_version": (ctypes.c_int32, []),
    "varrate_status_string": (ctypes.c_char_p, [ctypes.c_int32]),
    "varrate_check_config": (ctypes.c_int32, [ctypes.POINTER(varrate_config)]),
    "varrate_coded_budget": (ctypes.c_int64, [ctypes.POINTER(varrate_config)]),
    "varrate_packed_cap_elems": (ctypes.c_int64, [ctypes.POINTER(varrate_config)]),
    "varrate_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(varrate_config), ctypes.c_int32]),
    "varrate_salience": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                          _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_allocate": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                          _c_void_p, _c_void_p, _c_void_p]),
    "varrate_pack": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                      _c_void_p, _c_void_p, ctypes.POINTER(varrate_packed),
                                      _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_encode": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                        _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                        ctypes.POINTER(varrate_packed), _c_void_p, _c_void_p,
                                        _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_decode_attn": (ctypes.c_int32, [ctypes.POINTER(varrate_config),
                                             ctypes.POINTER(varrate_packed), _c_void_p, _c_void_p,
                                             _c_void_p, ctypes.c_int32, _c_void_p, _c_void_p,
                                             ctypes.c_int32, _c_void_p, _c_void_p, _c_void_p,
                                             ctypes.c_size_t, _c_void_p]),
    "varrate_decode_window": (ctypes.c_int32, [ctypes.POINTER(varrate_config),
                                               ctypes.POINTER(varrate_packed), _c_void_p, _c_void_p,
                                               _c_void_p, ctypes.c_int32, ctypes.c_int32, _c_void_p,
                                               _c_void_p, ctypes.c_int32, _c_void_p, _c_void_p,
                                               _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_qpacked_cap_bytes": (ctypes.c_int64, [ctypes.POINTER(varrate_config), ctypes.c_int32]),
    "varrate_quantize": (ctypes.c_int32, [ctypes.POINTER(varrate_config), ctypes.POINTER(varrate_packed),
                                          ctypes.POINTER(varrate_qpacked), _c_void_p, _c_void_p]),
    "varrate_decode_attn_q": (ctypes.c_int32, [ctypes.POINTER(varrate_config),
                                               ctypes.POINTER(varrate_qpacked), _c_void_p, _c_void_p,
                                               _c_void_p, ctypes.c_int32, _c_void_p, _c_void_p,
                                               ctypes.c_int32, _c_void_p, _c_void_p, _c_void_p,
                                               ctypes.c_size_t, _c_void_p]),
    "varrate_decode_attn_noalloc": (ctypes.c_int32, [ctypes.POINTER(varrate_config),
                                                     ctypes.POINTER(varrate_packed), _c_void_p,
                                                     _c_void_p, _c_void_p, ctypes.c_int32,
                                                     _c_void_p, _c_void_p, ctypes.c_int32,
                                                     _c_void_p, _c_void_p, _c_void_p]),
    "varrate_selftest_wait_timeout": (ctypes.c_int32, [_c_void_p, ctypes.c_uint32, _c_void_p]),
    "varrate_anchor_search_ws_bytes": (ctypes.c_size_t, [ctypes.POINTER(varrate_config), ctypes.c_int32]),
    "varrate_anchor_search": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                               ctypes.c_int32, ctypes.c_int32, _c_void_p, _c_void_p,
                                               _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_anchor_residual": (ctypes.c_int32, [ctypes.POINTER(varrate_config), _c_void_p, _c_void_p,
                                                 ctypes.c_int32, ctypes.c_int32, _c_void_p, _c_void_p,
                                                 _c_void_p, _c_void_p]),
    "varrate_paged_append": (ctypes.c_int32, [ctypes.POINTER(varrate_pages), ctypes.POINTER(varrate_seqs),
                                              ctypes.c_int32, ctypes.c_int32, _c_void_p, ctypes.c_int64,
                                              _c_void_p, ctypes.c_int64, _c_void_p, ctypes.c_int64,
                                              _c_void_p, _c_void_p, ctypes.c_double, _c_void_p,
                                              ctypes.c_int32, _c_void_p, _c_void_p, _c_void_p]),
    "varrate_paged_attn_ws_bytes": (ctypes.c_size_t, [ctypes.POINTER(varrate_pages),
                                                      ctypes.POINTER(varrate_seqs), ctypes.c_int32]),
    "varrate_paged_attn": (ctypes.c_int32, [ctypes.POINTER(varrate_pages), ctypes.POINTER(varrate_seqs),
                                            ctypes.c_int32, ctypes.c_int32, _c_void_p, _c_void_p,
                                            _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
    "varrate_paged_gather": (ctypes.c_int32, [ctypes.POINTER(varrate_pages), ctypes.POINTER(varrate_seqs),
                                              ctypes.c_int32, ctypes.c_int32, _c_void_p, ctypes.c_int32,
                                              _c_void_p, _c_void_p, _c_void_p, _c_void_p]),
}

EXPORTED = tuple(_SIGS)


def lib() -> ctypes.CDLL:
    """The loaded CUDA library (loaded on first use; raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_15498_gb300.build` (no CPU fallback exists)")
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


class VarrateError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def check(status: int, what: str = "varrate") -> int:
    """Raise VarrateError on a negative status; return it otherwise (OK or a warning)."""
    if status < 0:
        raise VarrateError(status, what)
    return status


# ------------------------------------------------------------------ plain C functions

def varrate_version() -> int:
    return lib().varrate_version()


def status_string(status: int) -> str:
    return lib().varrate_status_string(status).decode()


varrate_status_string = status_string


def varrate_check_config(cfg: varrate_config) -> int:
    return lib().varrate_check_config(ctypes.byref(cfg))


def varrate_coded_budget(cfg: varrate_config) -> int:
    return lib().varrate_coded_budget(ctypes.byref(cfg))


def varrate_packed_cap_elems(cfg: varrate_config) -> int:
    return lib().varrate_packed_cap_elems(ctypes.byref(cfg))


def varrate_workspace_bytes(cfg: varrate_config, which_call: int) -> int:
    return lib().varrate_workspace_bytes(ctypes.byref(cfg), which_call)


def varrate_salience(cfg, q_win, k, sal_out, ws, stream=None) -> int:
    return lib().varrate_salience(ctypes.byref(cfg), _ptr(q_win), _ptr(k), _ptr(sal_out), _ptr(ws),
                                  _nbytes(ws), _stream(stream))


def varrate_allocate(cfg, sal, ranks, realized_sum, dev_status, stream=None) -> int:
    return lib().varrate_allocate(ctypes.byref(cfg), _ptr(sal), _ptr(ranks), _ptr(realized_sum),
                                  _ptr(dev_status), _stream(stream))


def varrate_pack(cfg, k, v, basis_k, basis_v, packed, dev_status, ws=None, stream=None) -> int:
    return lib().varrate_pack(ctypes.byref(cfg), _ptr(k), _ptr(v), _ptr(basis_k), _ptr(basis_v),
                              ctypes.byref(packed.c), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                              _stream(stream))


def varrate_encode(cfg, q_win, k, v, basis_k, basis_v, sal_out, packed, realized_sum, dev_status,
                   ws, stream=None) -> int:
    return lib().varrate_encode(ctypes.byref(cfg), _ptr(q_win), _ptr(k), _ptr(v), _ptr(basis_k),
                                _ptr(basis_v), _ptr(sal_out), ctypes.byref(packed.c),
                                _ptr(realized_sum), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                _stream(stream))


def varrate_decode_attn(cfg, packed, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail, out,
                        dev_status, ws, stream=None) -> int:
    return lib().varrate_decode_attn(ctypes.byref(cfg), ctypes.byref(packed.c), _ptr(basis_k),
                                     _ptr(basis_v), _ptr(q), layer, _ptr(tail_k), _ptr(tail_v),
                                     n_tail, _ptr(out), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                     _stream(stream))


def varrate_decode_attn_noalloc(cfg, packed, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail,
                                out, dev_status, stream=None) -> int:
    return lib().varrate_decode_attn_noalloc(ctypes.byref(cfg), ctypes.byref(packed.c),
                                             _ptr(basis_k), _ptr(basis_v), _ptr(q), layer,
                                             _ptr(tail_k), _ptr(tail_v), n_tail, _ptr(out),
                                             _ptr(dev_status), _stream(stream))


def varrate_selftest_wait_timeout(dev_status, polls, stream=None) -> int:
    return lib().varrate_selftest_wait_timeout(_ptr(dev_status), polls, _stream(stream))


def varrate_anchor_search_ws_bytes(cfg: varrate_config, stride: int) -> int:
    return lib().varrate_anchor_search_ws_bytes(ctypes.byref(cfg), stride)


def varrate_anchor_search(cfg, k, v, stride, c, idx_out, dist_out, dev_status, ws, stream=None) -> int:
    return lib().varrate_anchor_search(ctypes.byref(cfg), _ptr(k), _ptr(v), stride, c, _ptr(idx_out),
                                       _ptr(dist_out), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                       _stream(stream))


def varrate_anchor_residual(cfg, k, v, stride, c, idx, e_out, dev_status, stream=None) -> int:
    return lib().varrate_anchor_residual(ctypes.byref(cfg), _ptr(k), _ptr(v), stride, c, _ptr(idx),
                                         _ptr(e_out), _ptr(dev_status), _stream(stream))


def varrate_decode_window(cfg, packed, basis_k, basis_v, q, n_q, layer, tail_k, tail_v, n_tail, out,
                          dev_status, ws, stream=None) -> int:
    return lib().varrate_decode_window(ctypes.byref(cfg), ctypes.byref(packed.c), _ptr(basis_k),
                                       _ptr(basis_v), _ptr(q), n_q, layer, _ptr(tail_k), _ptr(tail_v),
                                       n_tail, _ptr(out), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                       _stream(stream))


def varrate_qpacked_cap_bytes(cfg: varrate_config, bits: int) -> int:
    return lib().varrate_qpacked_cap_bytes(ctypes.byref(cfg), bits)


def varrate_quantize(cfg, packed, qpacked, dev_status, stream=None) -> int:
    return lib().varrate_quantize(ctypes.byref(cfg), ctypes.byref(packed.c), ctypes.byref(qpacked.c),
                                  _ptr(dev_status), _stream(stream))


def varrate_decode_attn_q(cfg, qpacked, basis_k, basis_v, q, layer, tail_k, tail_v, n_tail, out,
                          dev_status, ws, stream=None) -> int:
    return lib().varrate_decode_attn_q(ctypes.byref(cfg), ctypes.byref(qpacked.c), _ptr(basis_k),
                                       _ptr(basis_v), _ptr(q), layer, _ptr(tail_k), _ptr(tail_v),
                                       n_tail, _ptr(out), _ptr(dev_status), _ptr(ws), _nbytes(ws),
                                       _stream(stream))


def _on_device(pages, call, *args) -> int:
    """The call with the cache's device as the current one."""
    if pages.device < 0 or pages.device == torch._C._cuda_getDevice():
        return call(*args)
    with torch.cuda.device(pages.device):
        return call(*args)


def varrate_paged_append(pages, seqs, layer, q, k, v, q_norm, k_norm, eps, freq, rot_dim, q_out,
                         dev_status, stream=None) -> int:
    """q [T][H][d] or None, k, v [T][G][d]: rows may be apart (parts of one joint projection), heads not.
    ERR_ARG where a tensor is not of the cache's type, shape or device."""
    if not pages.works_with(seqs, dev_status):
        return ERR_ARG
    G, T = pages.heads, seqs.n_rows
    k_row, v_row = pages.row_stride(k, T, G), pages.row_stride(v, T, G)
    if q is None:
        H, q_row, q_ptr, out_ptr = G, 0, None, None
    else:
        H = q.shape[1] if q.dim() == 3 else 0
        q_row = pages.row_stride(q, T, H)
        if q_row < 0 or H % G or not pages.takes(q_out, (T, H, 128)):
            return ERR_ARG
        q_ptr, out_ptr = q.data_ptr(), q_out.data_ptr()
    if k_row < 0 or v_row < 0:
        return ERR_ARG
    if (q_norm is not None and not pages.takes(q_norm, (128,))) or (k_norm is not None and not pages.takes(k_norm, (128,))):
        return ERR_ARG
    freq_ptr = None
    if rot_dim and freq is not None:
        freq_ptr = freq.data_ptr()
        if not (freq.dtype is torch.float64 and freq.is_contiguous() and 2 * freq.numel() >= rot_dim
                and freq.get_device() == pages.device):
            return ERR_ARG
    return _on_device(
        pages, (_lib or lib()).varrate_paged_append, pages.ref, seqs.ref, layer, H // G, q_ptr, q_row, k.data_ptr(), k_row,
        v.data_ptr(), v_row, _ptr(q_norm), _ptr(k_norm), eps, freq_ptr, rot_dim, out_ptr, _ptr(dev_status),
        pages.stream(stream))


def varrate_paged_attn_ws_bytes(pages, seqs, group) -> int:
    return _on_device(pages, lib().varrate_paged_attn_ws_bytes, pages.ref, seqs.ref, group)


def varrate_paged_attn(pages, seqs, layer, group, q, out, dev_status, ws, stream=None) -> int:
    """q and out [T][H][d], dense. ERR_ARG where a tensor is not of the cache's type, shape or device."""
    shape = (seqs.n_rows, pages.heads * group, 128)
    if not (pages.takes(q, shape) and pages.takes(out, shape)):
        return ERR_ARG
    if ws is not None and not (pages.works_with(seqs, dev_status) and ws.get_device() == pages.device and ws.is_contiguous()):
        return ERR_ARG                                # (without one the C call launches nothing)
    return _on_device(pages, (_lib or lib()).varrate_paged_attn, pages.ref, seqs.ref, layer, group, q.data_ptr(),
                      out.data_ptr(), _ptr(dev_status), _ptr(ws), _nbytes(ws), pages.stream(stream))


def varrate_paged_gather(pages, seqs, layer, n_layers, first, n, k_out, v_out, dev_status, stream=None) -> int:
    """k_out, v_out [S][n_layers][G][n][d], dense, or None. ERR_ARG where a tensor is not of the cache's
    type, shape or device."""
    shape = (seqs.n_seqs, n_layers, pages.heads, n, 128)
    if (k_out is not None and not pages.takes(k_out, shape)) or (v_out is not None and not pages.takes(v_out, shape)):
        return ERR_ARG
    if not pages.works_with(seqs, dev_status):
        return ERR_ARG
    if first is not None and not (first.dtype is torch.int32 and first.is_contiguous()
                                  and first.shape == (seqs.n_seqs,) and first.get_device() == pages.device):
        return ERR_ARG
    return _on_device(pages, (_lib or lib()).varrate_paged_gather, pages.ref, seqs.ref, layer, n_layers, _ptr(first), n,
                      _ptr(k_out), _ptr(v_out), _ptr(dev_status), pages.stream(stream))


# ------------------------------------------------------------- device-memory plumbing

def make_config(n_layers, n_kv_heads, group, n_ctx, batch=1, budget_frac=0.2, r_min=16, window=32,
                pool_len=5, dtype=BF16, mode=SALIENCE, head_dim=128) -> varrate_config:
    return varrate_config(n_layers=n_layers, n_kv_heads=n_kv_heads, group=group, head_dim=head_dim,
                          n_ctx=n_ctx, batch=batch, r_min=r_min, budget_frac=budget_frac,
                          window=window, pool_len=pool_len, dtype=dtype, mode=mode)


def torch_dtype(cfg: varrate_config) -> torch.dtype:
    return torch.bfloat16 if cfg.dtype == BF16 else torch.float32


@dataclass
class PackedCache:
    """Torch-allocated device buffers of a packed cache plus the C struct pointing at them."""
    coef: torch.Tensor
    bucket_count: torch.Tensor
    bucket_base: torch.Tensor
    perm: torch.Tensor
    pos: torch.Tensor
    ranks: torch.Tensor
    cap_elems: int
    c: varrate_packed

    @staticmethod
    def allocate(cfg: varrate_config, device="cuda") -> "PackedCache":
        cap = varrate_packed_cap_elems(cfg)
        if cap < 0:
            raise VarrateError(ERR_ARG, "varrate_packed_cap_elems")
        B, L, G, N, d = cfg.batch, cfg.n_layers, cfg.n_kv_heads, cfg.n_ctx, cfg.head_dim
        coef = torch.empty((B, L, G, 2, cap), dtype=torch_dtype(cfg), device=device)
        cnt = torch.zeros((B, L, d + 1), dtype=torch.int32, device=device)
        base = torch.zeros((B, L, d + 2), dtype=torch.int64, device=device)
        perm = torch.empty((B, L, N), dtype=torch.int32, device=device)
        pos = torch.empty((B, L, N), dtype=torch.int32, device=device)
        ranks = torch.empty((B, L, N), dtype=torch.uint8, device=device)
        c = varrate_packed(coef.data_ptr(), cnt.data_ptr(), base.data_ptr(), perm.data_ptr(),
                           pos.data_ptr(), ranks.data_ptr(), cap)
        return PackedCache(coef, cnt, base, perm, pos, ranks, cap, c)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in
                   (self.coef, self.bucket_count, self.bucket_base, self.perm, self.pos, self.ranks))


@dataclass
class QPackedCache:
    """Torch-allocated buffers of a quantized cache (codes and group parameters, bucket byte
    offsets) plus the C struct; the bucket counts are those of the source PackedCache."""
    data: torch.Tensor
    qbase: torch.Tensor
    source: PackedCache
    bits: int
    qcap_bytes: int
    c: varrate_qpacked

    @staticmethod
    def allocate(cfg: varrate_config, source: PackedCache, bits: int, device="cuda") -> "QPackedCache":
        cap = varrate_qpacked_cap_bytes(cfg, bits)
        if cap < 0:
            raise VarrateError(ERR_ARG, "varrate_qpacked_cap_bytes")
        B, L, G, d = cfg.batch, cfg.n_layers, cfg.n_kv_heads, cfg.head_dim
        data = torch.zeros((B, L, G, 2, cap), dtype=torch.uint8, device=device)
        qbase = torch.zeros((B, L, d + 2), dtype=torch.int64, device=device)
        c = varrate_qpacked(data.data_ptr(), qbase.data_ptr(), source.bucket_count.data_ptr(), bits, cap)
        return QPackedCache(data, qbase, source, bits, cap, c)


@dataclass
class PagedCache:
    """The pages of a paged cache: pool [n_layers][n_pages][2][G][page_size][d] (0 is K, 1 is V) plus the
    C struct pointing at it. Which page belongs to which sequence is the caller's."""
    pool: torch.Tensor
    c: varrate_pages

    @staticmethod
    def of(pool: torch.Tensor) -> "PagedCache":
        if pool.dim() != 6 or pool.shape[2] != 2 or not pool.is_contiguous() or pool.dtype not in (
                torch.bfloat16, torch.float32):
            raise VarrateError(ERR_ARG, "PagedCache.of")
        L, P, _, G, ps, d = pool.shape
        c = varrate_pages(pool.data_ptr(), L, P, G, ps, d, BF16 if pool.dtype == torch.bfloat16 else F32)
        return PagedCache(pool, c)

    @staticmethod
    def allocate(n_layers, n_pages, n_kv_heads, page_size, dtype=BF16, device="cuda") -> "PagedCache":
        return PagedCache.of(torch.empty((n_layers, n_pages, 2, n_kv_heads, page_size, 128), device=device,
                                         dtype=torch.bfloat16 if dtype == BF16 else torch.float32))

    def __post_init__(self):
        self.ref = ctypes.byref(self.c)
        self.heads, self.dtype, self.device = self.c.n_kv_heads, self.pool.dtype, self.pool.get_device()

    def takes(self, t: torch.Tensor, shape) -> bool:
        """Whether t has this shape and the cache's type and device and is dense."""
        return (t is not None and t.shape == shape and t.dtype is self.dtype and t.is_contiguous()
                and t.get_device() == self.device)

    def row_stride(self, t: torch.Tensor, rows: int, heads: int) -> int:
        """Elements from row to row of t [rows][heads][d], whose rows may be apart, or -1 where it has not this shape, the
        cache's type and device and dense rows."""
        if t is None or t.shape != (rows, heads, 128) or t.dtype is not self.dtype or t.get_device() != self.device:
            return -1
        row, head, elem = t.stride()
        if elem != 1 or (head != 128 and heads > 1):
            return -1 if rows else 0
        return row if rows > 1 else heads * 128      # of one row: any number

    def works_with(self, seqs, dev_status) -> bool:
        """Whether the cache, a batch's tables and a status word (int32; None or a raw pointer pass) are on one GPU."""
        return seqs.device == self.device >= 0 and (dev_status is None or type(dev_status) is int or (
            dev_status.dtype is torch.int32 and dev_status.get_device() == self.device))

    def stream(self, stream) -> int | None:
        """`stream` as _stream takes it; None is torch's current stream on the cache's device."""
        if stream is None and self.device >= 0:
            return torch._C._cuda_getCurrentRawStream(self.device)
        return _stream(stream)


@dataclass
class SeqBatch:
    """A batch of sequences with new tokens: row_start [S + 1], kv_len [S] and page_table [S][max_pages],
    int32 on the cache's GPU, n_rows rows of queries, keys and values; plus the C struct. The tensors may be
    refilled in place from step to step (the calls read them on the stream)."""
    row_start: torch.Tensor
    kv_len: torch.Tensor
    page_table: torch.Tensor
    c: varrate_seqs

    @staticmethod
    def of(row_start: torch.Tensor, kv_len: torch.Tensor, page_table: torch.Tensor, n_rows: int) -> "SeqBatch":
        if kv_len is None or page_table is None or page_table.dim() != 2:   # row_start may be missing, to gather
            raise VarrateError(ERR_ARG, "SeqBatch.of")
        S = kv_len.numel()
        for t, shape in ((row_start, (S + 1,)), (kv_len, (S,)), (page_table, (S, page_table.shape[-1]))):
            if t is not None and (t.shape != shape or t.dtype != torch.int32 or not t.is_contiguous()
                                  or t.get_device() != kv_len.get_device()):
                raise VarrateError(ERR_ARG, "SeqBatch.of")
        c = varrate_seqs(_ptr(row_start), _ptr(kv_len), _ptr(page_table), S, page_table.shape[-1], n_rows)
        return SeqBatch(row_start, kv_len, page_table, c)

    def __post_init__(self):
        self.ref = ctypes.byref(self.c)
        self.n_seqs, self.n_rows, self.device = self.c.n_seqs, self.c.n_rows, self.kv_len.get_device()


def paged_attn_workspace(pages: PagedCache, seqs: SeqBatch, group: int) -> torch.Tensor:
    """Device scratch of varrate_paged_attn for batches of this size, zero-filled as its first call wants it."""
    n = varrate_paged_attn_ws_bytes(pages, seqs, group)
    return torch.zeros(max(n, 256), dtype=torch.uint8, device=pages.pool.device)


def workspace(cfg: varrate_config, which_call: int, device="cuda") -> torch.Tensor:
    """Device scratch for one kind of call, zero-filled (the decode workspace's header must be zero
    before the first decode call that uses it; later calls keep it consistent themselves)."""
    n = varrate_workspace_bytes(cfg, which_call)
    return torch.zeros(max(n, 256), dtype=torch.uint8, device=device)
