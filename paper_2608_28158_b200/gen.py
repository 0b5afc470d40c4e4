"""ctypes binding of the harts_gen_* entry points (same names as the C ABI): sampling on rollout trees.

Argument checks here are those that need the tensors' shapes, types, strides and devices; a bad argument raises :class:`HartsError`
with HARTS_EINVAL (HARTS_EUNSUPPORTED for a type or size without a kernel) and launches nothing."""
from __future__ import annotations

import contextlib
import ctypes as C

import numpy as np
import torch

from .binding import lib, HartsError, HARTS_BF16, _check, _DTYPE_CODE, _I32P

HARTS_E4M3 = 2
HARTS_EINVAL, HARTS_EUNSUPPORTED = -1, -3
_vp, _i32, _i64, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
lib.harts_gen_la_workspace_bytes.argtypes = [_i32, _i32, _i64] + [_i32] * 4 + [C.POINTER(_sz)]
lib.harts_gen_la.argtypes = [_i32, _vp, _vp, _vp, _vp, _i32, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp] + [_i32] * 5 + [
    _vp, _sz, _vp, _vp]
lib.harts_gen_cache_write.argtypes = [_i64, _vp, _vp, _i64, _vp, _i64] + [_vp] * 4 + [_i32] * 5 + [_vp, _vp]
lib.harts_gen_cache_read.argtypes = [_i64] + [_vp] * 7 + [_i32] * 5 + [_vp, _vp]
lib.harts_gen_attn_index.argtypes = [_i32] + [_I32P] * 6 + [_i32, _i32, _I32P, _I32P] + [_i32] * 3 + [_i64, _I32P, C.POINTER(_i64)]
lib.harts_gen_attn_workspace_bytes.argtypes = [_I32P, C.POINTER(_sz)]
lib.harts_gen_attn.argtypes = [_I32P, _vp, _vp, _i64] + [_vp] * 4 + [_i32, _i32, _vp, _vp, _vp, C.c_float, _vp, _sz, _vp, _vp]
for _n in ("harts_gen_la_workspace_bytes", "harts_gen_la", "harts_gen_cache_write", "harts_gen_cache_read", "harts_gen_attn_index",
           "harts_gen_attn_workspace_bytes", "harts_gen_attn"):
    getattr(lib, _n).restype = _i32


def _bad(where, what, code=HARTS_EINVAL):
    raise HartsError(code, f"{where} ({what})")


def _p(t):
    return None if t is None else t.data_ptr()


def _code(where, dtype):
    if dtype not in _DTYPE_CODE:
        _bad(where, f"no kernel for {dtype}", HARTS_EUNSUPPORTED)
    return _DTYPE_CODE[dtype]


def _rows(where, name, t, heads, d, dtype, n=None):
    """Elements between the rows of a [rows, heads, d] tensor whose heads are contiguous."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != d or t.dtype != dtype or (n is not None and t.shape[0] != n):
        _bad(where, f"{name}: {tuple(t.shape)} {t.dtype}")
    if (d > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != d):
        _bad(where, f"{name}: strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else heads * d


def _plain(where, name, t, dtype, shape):
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        _bad(where, f"{name}: {t.dtype} {tuple(t.shape)}, strides {t.stride()}")


def _one_device(where, **tensors):
    dev = None
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            _bad(where, f"{name} is not on a CUDA device")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            _bad(where, f"{name} is on {t.device}, others on {dev}")
    return dev


def _on(dev, stream):
    """The device made current for the launch, and the stream: the given one or the current one of that device."""
    guard = contextlib.nullcontext() if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)
    return guard, (torch.cuda.current_stream(dev) if stream is None else stream).cuda_stream


def harts_gen_la_workspace_bytes(n_seq, max_len, n_rows, H, dk, dv, dtype) -> int:
    n = _sz(0)
    _check(lib.harts_gen_la_workspace_bytes(n_seq, max_len, n_rows, H, dk, dv, _code("harts_gen_la_workspace_bytes", dtype), C.byref(n)),
           "harts_gen_la_workspace_bytes")
    return n.value


def harts_gen_la(q, k, v, g, o, states, seq_begin, seq_len, in_state, out_state, max_len, workspace=None, dev_status=None, stream=None):
    """Linear attention from and into kept states (harts_gen.h).  q may be None where o is."""
    w = "harts_gen_la"
    dev = _one_device(w, k=k, q=q, v=v, g=g, o=o, states=states, seq_begin=seq_begin, seq_len=seq_len, in_state=in_state,
                      out_state=out_state, workspace=workspace, dev_status=dev_status)
    if k.dim() != 3:
        _bad(w, f"k: {tuple(k.shape)}")
    (rows, H, d), dt, n_seq = k.shape, k.dtype, seq_begin.shape[0] if seq_begin.dim() == 1 else -1
    code = _code(w, dt)
    ld_k, ld_v = _rows(w, "k", k, H, d, dt), _rows(w, "v", v, H, d, dt, rows)
    ld_q = 0
    if o is not None:
        if q is None:
            _bad(w, "o without q")
        ld_q = _rows(w, "q", q, H, d, dt, rows)
        _plain(w, "o", o, dt, (rows, H, d))
    _plain(w, "g", g, torch.float32, (rows, H))
    if states.dim() != 4:
        _bad(w, f"states: {tuple(states.shape)}")
    _plain(w, "states", states, torch.float32, (states.shape[0], H, d, d))
    for name, t in (("seq_begin", seq_begin), ("seq_len", seq_len), ("in_state", in_state), ("out_state", out_state)):
        _plain(w, name, t, torch.int32, (n_seq,))
    if workspace is not None and not workspace.is_contiguous():
        _bad(w, "workspace is not contiguous")
    guard, st = _on(dev, stream)
    with guard:
        _check(lib.harts_gen_la(n_seq, _p(seq_begin), _p(seq_len), _p(in_state), _p(out_state), max_len, rows, _p(q), ld_q, _p(k), ld_k,
                                _p(v), ld_v, _p(g), _p(o), _p(states), states.shape[0], H, d, d, code, _p(workspace),
                                0 if workspace is None else workspace.numel() * workspace.element_size(), _p(dev_status), st), w)


def _cache(where, k_cache, v_cache, k_exp, v_exp):
    """(n_pages, Hkv, page, type) of a cache, checked."""
    if k_cache.dim() != 4:
        _bad(where, f"k_cache: {tuple(k_cache.shape)}")
    n_pages, hkv, page, d = k_cache.shape
    kind = {torch.bfloat16: HARTS_BF16, torch.float8_e4m3fn: HARTS_E4M3}.get(k_cache.dtype)
    if kind is None:
        _bad(where, f"no cache of {k_cache.dtype}", HARTS_EUNSUPPORTED)
    _plain(where, "k_cache", k_cache, k_cache.dtype, k_cache.shape)
    _plain(where, "v_cache", v_cache, k_cache.dtype, k_cache.shape)
    if d != 128:
        _bad(where, f"rows of {d}", HARTS_EUNSUPPORTED)
    for name, e in (("k_exp", k_exp), ("v_exp", v_exp)):
        if (e is None) != (kind == HARTS_BF16):
            _bad(where, f"{name} goes with an 8-bit cache")
        if e is not None:
            _plain(where, name, e, torch.uint8, (n_pages, hkv, page))
    return n_pages, hkv, page, kind


def harts_gen_cache_write(k, v, slot, k_cache, v_cache, k_exp=None, v_exp=None, dev_status=None, stream=None):
    """Rows of k, v into slots of a paged cache (harts_gen.h); torch.float8_e4m3fn caches have k_exp, v_exp."""
    w = "harts_gen_cache_write"
    dev = _one_device(w, k=k, v=v, slot=slot, k_cache=k_cache, v_cache=v_cache, k_exp=k_exp, v_exp=v_exp, dev_status=dev_status)
    n_pages, hkv, page, kind = _cache(w, k_cache, v_cache, k_exp, v_exp)
    n = k.shape[0] if k.dim() else 0
    _plain(w, "slot", slot, torch.int32, (n,))
    ld_k, ld_v = _rows(w, "k", k, hkv, 128, torch.bfloat16), _rows(w, "v", v, hkv, 128, torch.bfloat16, n)
    guard, st = _on(dev, stream)
    with guard:
        _check(lib.harts_gen_cache_write(n, _p(slot), _p(k), ld_k, _p(v), ld_v, _p(k_cache), _p(v_cache), _p(k_exp), _p(v_exp), n_pages, page, hkv,
                                         128, kind, _p(dev_status), st), w)


def harts_gen_cache_read(k_cache, v_cache, slot, k, v, k_exp=None, v_exp=None, dev_status=None, stream=None):
    """Rows of a paged cache into k, v (bf16, contiguous; either may be None)."""
    w = "harts_gen_cache_read"
    dev = _one_device(w, slot=slot, k_cache=k_cache, v_cache=v_cache, k=k, v=v, k_exp=k_exp, v_exp=v_exp, dev_status=dev_status)
    n_pages, hkv, page, kind = _cache(w, k_cache, v_cache, k_exp, v_exp)
    n = slot.shape[0] if slot.dim() else -1
    _plain(w, "slot", slot, torch.int32, (n,))
    for name, t in (("k", k), ("v", v)):
        if t is not None:
            _plain(w, name, t, torch.bfloat16, (n, hkv, 128))
    guard, st = _on(dev, stream)
    with guard:
        _check(lib.harts_gen_cache_read(n, _p(slot), _p(k_cache), _p(v_cache), _p(k_exp), _p(v_exp), _p(k), _p(v), n_pages, page, hkv, 128, kind,
                                        _p(dev_status), st), w)


class GenAttnIndex:
    """The index blob on the host (numpy int32) and, after ``upload``, on the device."""

    def __init__(self, blob):
        self.host = blob
        self.n_q, self.Hq, self.Hkv, self.page, self.n_narrow, self.n_wide, self.n_parts = map(int, blob[:7])
        n = _sz(0)
        _check(lib.harts_gen_attn_workspace_bytes(blob.ctypes.data_as(_I32P), C.byref(n)), "harts_gen_attn_workspace_bytes")
        self.workspace_bytes = n.value
        self.dev = None

    def upload(self, device="cuda"):
        self.dev = torch.as_tensor(self.host).to(device)
        return self


def harts_gen_attn_index(tree_node_ptr, node_parent, node_fork_off, node_len, node_page_ptr, node_page, page, q_node, q_pos, Hq, Hkv,
                         grow=0) -> GenAttnIndex:
    """Work lists for the queries (q_node, q_pos) on a cached forest (harts_gen.h)."""
    w = "harts_gen_attn_index"
    arrs = [np.ascontiguousarray(np.asarray(a), dtype=np.int32) for a in
            (tree_node_ptr, node_parent, node_fork_off, node_len, node_page_ptr, node_page, q_node, q_pos)]
    if any(a.ndim != 1 for a in arrs) or len(arrs[0]) < 1:
        _bad(w, "arrays have one dimension")
    n_nodes = int(arrs[0][-1])
    if [len(a) for a in arrs[1:5]] != [n_nodes] * 3 + [n_nodes + 1] or len(arrs[5]) != arrs[4][-1] or len(arrs[6]) != len(arrs[7]):
        _bad(w, "lengths of the arrays do not agree")
    ip = lambda a: a.ctypes.data_as(_I32P)  # noqa: E731
    n = _i64(0)
    # room for what indices usually need, so that they are built once; the call says how much it wants otherwise
    blob = np.empty(1 << 14, np.int32)
    build = lambda: lib.harts_gen_attn_index(len(arrs[0]) - 1, *map(ip, arrs[:6]), page, len(arrs[6]), ip(arrs[6]), ip(arrs[7]), Hq, Hkv, grow,  # noqa: E731
                                             len(blob), ip(blob), C.byref(n))
    code = build()
    if n.value > len(blob):
        blob = np.empty(n.value, np.int32)
        code = build()
    _check(code, w)
    return GenAttnIndex(blob[:n.value].copy())


def harts_gen_attn(index: GenAttnIndex, q, k_cache, v_cache, q_pos, o, lse, scale, workspace=None, k_exp=None, v_exp=None, dev_status=None,
                   stream=None):
    """Attention of sampled tokens on the cached tree (harts_gen.h)."""
    w = "harts_gen_attn"
    if index.dev is None:
        _bad(w, "the index has not been uploaded")
    dev = _one_device(w, q=q, index=index.dev, k_cache=k_cache, v_cache=v_cache, k_exp=k_exp, v_exp=v_exp, q_pos=q_pos, o=o, lse=lse,
                      workspace=workspace, dev_status=dev_status)
    n_pages, hkv, page, kind = _cache(w, k_cache, v_cache, k_exp, v_exp)
    if hkv != index.Hkv or page != index.page:
        _bad(w, f"a cache of {hkv} heads and pages of {page} with an index for {index.Hkv} and {index.page}")
    ld_q = _rows(w, "q", q, index.Hq, 128, torch.bfloat16, index.n_q)
    _plain(w, "q_pos", q_pos, torch.int32, (index.n_q,))
    _plain(w, "o", o, torch.bfloat16, (index.n_q, index.Hq, 128))
    _plain(w, "lse", lse, torch.float32, (index.n_q, index.Hq))
    if workspace is not None and not workspace.is_contiguous():
        _bad(w, "workspace is not contiguous")
    guard, st = _on(dev, stream)
    with guard:
        _check(lib.harts_gen_attn(index.host.ctypes.data_as(_I32P), _p(index.dev), _p(q), ld_q, _p(k_cache), _p(v_cache), _p(k_exp), _p(v_exp),
                                  n_pages, kind, _p(q_pos), _p(o), _p(lse), scale, _p(workspace),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _p(dev_status), st), w)
