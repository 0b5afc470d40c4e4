"""ctypes binding of the harts_gen_* entry points (same names as the C ABI): sampling on rollout trees.

Argument checks here are those that need the tensors' shapes, types, strides and devices; a bad argument raises :class:`HartsError`
with HARTS_EINVAL (HARTS_EUNSUPPORTED for a type or size without a kernel) and launches nothing."""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from .binding import lib, HartsError, HARTS_BF16, HARTS_OK, _check, _DTYPE_CODE, _I32P

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


# the current stream's handle without the Stream object around it, which costs more than a call's other checks together
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _bad(where, what, code=HARTS_EINVAL):
    raise HartsError(code, f"{where} ({what})")


def _bad_tensor(where, name, t, dev):
    if t.get_device() != dev:
        _bad(where, f"{name} is on {t.device}" + (f", others on cuda:{dev}" if t.is_cuda else ""))
    _bad(where, f"{name}: {t.dtype} {tuple(t.shape)}, strides {t.stride()}")


def _p(t):
    return None if t is None else t.data_ptr()


def _code(where, dtype):
    if dtype not in _DTYPE_CODE:
        _bad(where, f"no kernel for {dtype}", HARTS_EUNSUPPORTED)
    return _DTYPE_CODE[dtype]


def _int32(where, **sizes):
    """Sizes that the C ABI takes in 32 bits (ctypes would cut them off without a word)."""
    for name, x in sizes.items():
        if not -2 ** 31 <= x < 2 ** 31:
            _bad(where, f"{name}: {x} is not a number of 32 bits")


def _int32_array(where, name, a):
    """One-dimensional whole numbers of any type as int32, none of them changed."""
    a = np.asarray(a)
    if a.ndim != 1:
        _bad(where, f"{name}: {a.ndim} dimensions, wants one")
    if a.dtype != np.int32 and a.size and not (-2 ** 31 <= a.min() <= a.max() < 2 ** 31 and (a.dtype.kind in "iub" or (a == np.rint(a)).all())):
        _bad(where, f"{name}: numbers from {a.min()} to {a.max()}, wants whole ones of 32 bits")
    return np.ascontiguousarray(a, dtype=np.int32)


def _device(where, name, t):
    dev = t.get_device()
    if dev < 0:
        _bad(where, f"{name} is not on a CUDA device")
    return dev


def _rows(where, name, t, shape, dtype, dev):
    """Elements between the rows of a [rows, heads, d] tensor whose heads are contiguous."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _bad_tensor(where, name, t, dev)
    rows, heads, d = shape
    ld, sh, sd = t.stride()
    if (sd != 1 and d > 1) or (sh != d and heads > 1):
        _bad_tensor(where, name, t, dev)
    return ld if rows > 1 else heads * d


def _plain(where, name, t, dtype, shape, dev):
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != dev:
        _bad_tensor(where, name, t, dev)
    return t.data_ptr()


def _bytes(where, name, t, dev):
    """Pointer and size of a work buffer of any type, or of none."""
    if t is None:
        return None, 0
    if not t.is_contiguous() or t.get_device() != dev:
        _bad_tensor(where, name, t, dev)
    return t.data_ptr(), t.numel() * t.element_size()


def _status(where, t, dev):
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() < 2 or not t.is_contiguous() or t.get_device() != dev:
        _bad_tensor(where, "dev_status", t, dev)
    return t.data_ptr()


def _call(where, f, dev, stream, *args):
    """The call on the given stream, or the current one of the tensors' device, with that device current."""
    st = _raw_stream(dev) if stream is None else stream.cuda_stream
    if dev == torch.cuda.current_device():
        code = f(*args, st)
    else:
        with torch.cuda.device(dev):
            code = f(*args, st)
    if code != HARTS_OK:
        raise HartsError(code, where)


def harts_gen_la_workspace_bytes(n_seq, max_len, n_rows, H, dk, dv, dtype) -> int:
    _int32("harts_gen_la_workspace_bytes", n_seq=n_seq, max_len=max_len, H=H, dk=dk, dv=dv)
    n = _sz(0)
    _check(lib.harts_gen_la_workspace_bytes(n_seq, max_len, n_rows, H, dk, dv, _code("harts_gen_la_workspace_bytes", dtype), C.byref(n)),
           "harts_gen_la_workspace_bytes")
    return n.value


def harts_gen_la(q, k, v, g, o, states, seq_begin, seq_len, in_state, out_state, max_len, workspace=None, dev_status=None, stream=None):
    """Linear attention from and into kept states (harts_gen.h).  q may be None where o is."""
    w = "harts_gen_la"
    dev = _device(w, "k", k)
    if k.dim() != 3 or states.dim() != 4 or seq_begin.dim() != 1:
        _bad(w, f"k: {tuple(k.shape)}, states: {tuple(states.shape)}, seq_begin: {tuple(seq_begin.shape)}")
    shape, dt, n_seq, n_states = k.shape, k.dtype, seq_begin.shape[0], states.shape[0]
    rows, H, d = shape
    code = _code(w, dt)
    ld_k, ld_v = _rows(w, "k", k, shape, dt, dev), _rows(w, "v", v, shape, dt, dev)
    ld_q = o_ptr = 0
    if o is not None:
        if q is None:
            _bad(w, "o without q")
        ld_q = _rows(w, "q", q, shape, dt, dev)
        o_ptr = _plain(w, "o", o, dt, shape, dev)
    if not -2 ** 31 <= max_len < 2 ** 31:
        _int32(w, max_len=max_len)
    i32, one = torch.int32, (n_seq,)
    ws, ws_bytes = _bytes(w, "workspace", workspace, dev)
    _call(w, lib.harts_gen_la, dev, stream, n_seq, _plain(w, "seq_begin", seq_begin, i32, one, dev), _plain(w, "seq_len", seq_len, i32, one, dev),
          _plain(w, "in_state", in_state, i32, one, dev), _plain(w, "out_state", out_state, i32, one, dev), max_len, rows,
          _p(q) if o_ptr else None, ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, _plain(w, "g", g, torch.float32, (rows, H), dev), o_ptr or None,
          _plain(w, "states", states, torch.float32, (n_states, H, d, d), dev), n_states, H, d, d, code, ws, ws_bytes,
          _status(w, dev_status, dev))


_CACHE_TYPES = {torch.bfloat16: HARTS_BF16, torch.float8_e4m3fn: HARTS_E4M3}


def _cache(where, k_cache, v_cache, k_exp, v_exp, dev):
    """Shape, type and pointers of a cache, checked."""
    shape = k_cache.shape
    kind = _CACHE_TYPES.get(k_cache.dtype)
    if kind is None or len(shape) != 4 or shape[3] != 128:
        _bad(where, f"no cache of {k_cache.dtype} {tuple(shape)}", HARTS_EUNSUPPORTED)
    k, v, ke, ve = _plain(where, "k_cache", k_cache, k_cache.dtype, shape, dev), _plain(where, "v_cache", v_cache, k_cache.dtype, shape, dev), None, None
    if (k_exp is None) != (kind == HARTS_BF16) or (v_exp is None) != (kind == HARTS_BF16):
        _bad(where, "k_exp and v_exp go with an 8-bit cache, and only with one")
    if k_exp is not None:
        ke, ve = _plain(where, "k_exp", k_exp, torch.uint8, shape[:3], dev), _plain(where, "v_exp", v_exp, torch.uint8, shape[:3], dev)
    return shape, kind, (k, v, ke, ve)


def harts_gen_cache_write(k, v, slot, k_cache, v_cache, k_exp=None, v_exp=None, dev_status=None, stream=None):
    """Rows of k, v into slots of a paged cache (harts_gen.h); torch.float8_e4m3fn caches have k_exp, v_exp."""
    w = "harts_gen_cache_write"
    dev = _device(w, "k_cache", k_cache)
    (n_pages, hkv, page, _), kind, ptrs = _cache(w, k_cache, v_cache, k_exp, v_exp, dev)
    n = k.shape[0] if k.dim() else 0
    shape = (n, hkv, 128)
    slots = _plain(w, "slot", slot, torch.int32, (n,), dev)
    ld_k, ld_v = _rows(w, "k", k, shape, torch.bfloat16, dev), _rows(w, "v", v, shape, torch.bfloat16, dev)
    _call(w, lib.harts_gen_cache_write, dev, stream, n, slots, k.data_ptr(), ld_k, v.data_ptr(), ld_v, *ptrs, n_pages, page, hkv, 128, kind,
          _status(w, dev_status, dev))


def harts_gen_cache_read(k_cache, v_cache, slot, k, v, k_exp=None, v_exp=None, dev_status=None, stream=None):
    """Rows of a paged cache into k, v (bf16, contiguous; either may be None)."""
    w = "harts_gen_cache_read"
    dev = _device(w, "k_cache", k_cache)
    (n_pages, hkv, page, _), kind, ptrs = _cache(w, k_cache, v_cache, k_exp, v_exp, dev)
    n = slot.shape[0] if slot.dim() else -1
    slots = _plain(w, "slot", slot, torch.int32, (n,), dev)
    out = [None if t is None else _plain(w, name, t, torch.bfloat16, (n, hkv, 128), dev) for name, t in (("k", k), ("v", v))]
    _call(w, lib.harts_gen_cache_read, dev, stream, n, slots, *ptrs, *out, n_pages, page, hkv, 128, kind, _status(w, dev_status, dev))


class GenAttnIndex:
    """The index blob on the host (numpy int32) and, after ``upload``, on the device."""

    def __init__(self, blob):
        self.host = blob
        self.host_ptr = blob.ctypes.data_as(_I32P)
        self.n_q, self.Hq, self.Hkv, self.page, self.n_narrow, self.n_wide, self.n_parts = map(int, blob[:7])
        n = _sz(0)
        _check(lib.harts_gen_attn_workspace_bytes(self.host_ptr, C.byref(n)), "harts_gen_attn_workspace_bytes")
        self.workspace_bytes = n.value
        self.dev = None

    def upload(self, device="cuda"):
        self.dev = torch.as_tensor(self.host).to(device)
        return self


def harts_gen_attn_index(tree_node_ptr, node_parent, node_fork_off, node_len, node_page_ptr, node_page, page, q_node, q_pos, Hq, Hkv,
                         grow=0) -> GenAttnIndex:
    """Work lists for the queries (q_node, q_pos) on a cached forest (harts_gen.h)."""
    w = "harts_gen_attn_index"
    _int32(w, page=page, Hq=Hq, Hkv=Hkv, grow=grow)
    arrs = [_int32_array(w, *x) for x in (("tree_node_ptr", tree_node_ptr), ("node_parent", node_parent), ("node_fork_off", node_fork_off),
                                          ("node_len", node_len), ("node_page_ptr", node_page_ptr), ("node_page", node_page), ("q_node", q_node),
                                          ("q_pos", q_pos))]
    if len(arrs[0]) < 1:
        _bad(w, "tree_node_ptr is empty")
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
    dev = _device(w, "k_cache", k_cache)
    (n_pages, hkv, page, _), kind, ptrs = _cache(w, k_cache, v_cache, k_exp, v_exp, dev)
    if hkv != index.Hkv or page != index.page:
        _bad(w, f"a cache of {hkv} heads and pages of {page} with an index for {index.Hkv} and {index.page}")
    shape = (index.n_q, index.Hq, 128)
    ws, ws_bytes = _bytes(w, "workspace", workspace, dev)
    _call(w, lib.harts_gen_attn, dev, stream, index.host_ptr, _plain(w, "index", index.dev, torch.int32, index.host.shape, dev), q.data_ptr(),
          _rows(w, "q", q, shape, torch.bfloat16, dev), *ptrs, n_pages, kind, _plain(w, "q_pos", q_pos, torch.int32, shape[:1], dev),
          _plain(w, "o", o, torch.bfloat16, shape, dev), _plain(w, "lse", lse, torch.float32, shape[:2], dev), scale, ws, ws_bytes,
          _status(w, dev_status, dev))
