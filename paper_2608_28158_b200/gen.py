"""ctypes binding of the harts_gen_* entry points (same names as the C ABI): sampling on rollout trees.

Argument checks here are those that need the tensors' shapes, types, strides and devices; a bad argument raises :class:`HartsError`
with HARTS_EINVAL (HARTS_EUNSUPPORTED for a type or size without a kernel) and launches nothing."""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from .binding import lib, HartsError, HARTS_FP32, _check, _DTYPE_CODE

HARTS_EINVAL, HARTS_EUNSUPPORTED = -1, -3
_vp, _i32, _i64, _sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
lib.harts_gen_la_workspace_bytes.argtypes = [_i32, _i32, _i64] + [_i32] * 4 + [C.POINTER(_sz)]
lib.harts_gen_la.argtypes = [_i32, _vp, _vp, _vp, _vp, _i32, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp] + [_i32] * 5 + [
    _vp, _sz, _vp, _vp]
for _n in ("harts_gen_la_workspace_bytes", "harts_gen_la"):
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
