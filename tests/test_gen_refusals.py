"""What the harts_gen_* calls refuse, on the host: nothing is launched, so the pointers need not be any device's."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2608_28158_b200 as H
from paper_2608_28158_b200 import gen

EINVAL, EUNSUPPORTED, OK = -1, -3, 0
P = 1 << 20                 # a 16-byte-aligned address that nothing reads
FP32, BF16, E4M3 = 0, 1, 2


LA = dict(n_seq=3, seq_begin=P, seq_len=P, in_state=P, out_state=P, max_len=4, n_rows=12, q=P, ld_q=512, k=P, ld_k=512, v=P, ld_v=512, g=P, o=P, states=P,
          n_states=6, H=4, dk=128, dv=128, dtype=BF16, ws=None, ws_bytes=0, status=None, stream=None)


def la(**kw):
    return gen.lib.harts_gen_la(*{**LA, **kw}.values())


@pytest.mark.parametrize("bad,code", [
    (dict(n_seq=-1), EINVAL), (dict(max_len=-1), EINVAL), (dict(n_rows=-1), EINVAL), (dict(n_rows=2 ** 31), EINVAL), (dict(n_seq=65536), EINVAL),
    (dict(H=0), EINVAL), (dict(H=65536), EINVAL), (dict(n_states=-1), EINVAL), (dict(dtype=2), EUNSUPPORTED), (dict(dv=64), EUNSUPPORTED),
    (dict(dk=96, dv=96), EUNSUPPORTED), (dict(seq_begin=None), EINVAL), (dict(seq_len=None), EINVAL), (dict(in_state=None), EINVAL),
    (dict(out_state=None), EINVAL), (dict(states=None), EINVAL), (dict(states=P + 8), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(g=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(k=P + 2), EINVAL), (dict(o=P + 8), EINVAL), (dict(ld_q=511), EINVAL),
    (dict(ld_k=508), EINVAL), (dict(ld_v=516), EINVAL), (dict(dtype=FP32, ld_k=514), EINVAL), (dict(max_len=100), EINVAL),
    (dict(max_len=100, ws=P, ws_bytes=16), EINVAL), (dict(max_len=100, ws=P + 8, ws_bytes=1 << 40), EINVAL)])
def test_la_refuses(bad, code):
    assert la(**bad) == code


def test_la_without_sequences_does_nothing():
    assert la(n_seq=0) == OK
    assert la(n_seq=0, seq_begin=None, k=None, states=None) == OK


def test_la_workspace():
    f = H.harts_gen_la_workspace_bytes
    assert f(200, 1, 200, 32, 128, 128, torch.bfloat16) == 0 and f(2, 5000, 9000, 4, 64, 64, torch.bfloat16) == 0
    assert f(2, 5000, 9000, 4, 128, 128, torch.float32) == 0 and f(0, 5000, 9000, 4, 128, 128, torch.bfloat16) == 0
    small, large = f(300, 40, 12000, 32, 128, 128, torch.bfloat16), f(1, 31000, 31000, 4, 128, 128, torch.bfloat16)
    assert 0 < small < 1 << 16                                       # tables only
    assert large > 4 * 20 * 65536                                    # start states of segments
    for bad in ((-1, 1, 1, 1, 64, 64, torch.float32), (1, 1, 1, 0, 64, 64, torch.float32), (1, 1, 1, 1, 64, 128, torch.float32),
                (1, 1, 1, 1, 64, 64, torch.float16)):
        with pytest.raises(H.HartsError):
            f(*bad)


CACHE = dict(n=5, slot=P, k=P, ld_k=512, v=P, ld_v=512, k_cache=P, v_cache=P, k_exp=P, v_exp=P, n_pages=7, page=16, Hkv=4, d=128, kind=E4M3, status=None,
             stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(n=-1), EINVAL), (dict(n=2 ** 31), EINVAL), (dict(n_pages=-1), EINVAL), (dict(page=8), EINVAL), (dict(page=256), EINVAL), (dict(page=48), EINVAL),
    (dict(Hkv=0), EINVAL), (dict(d=64), EUNSUPPORTED), (dict(kind=0), EUNSUPPORTED), (dict(kind=3), EUNSUPPORTED), (dict(slot=None), EINVAL),
    (dict(k=None), EINVAL), (dict(v=P + 8), EINVAL), (dict(ld_k=504), EINVAL), (dict(ld_v=516), EINVAL), (dict(k_cache=None), EINVAL),
    (dict(v_cache=P + 8), EINVAL), (dict(k_exp=None), EINVAL), (dict(v_exp=P + 1), EINVAL), (dict(n_pages=2 ** 31 - 1, page=16), EINVAL),
    (dict(n_pages=2 ** 30, Hkv=4, page=16), EINVAL)])
def test_cache_write_refuses(bad, code):
    assert gen.lib.harts_gen_cache_write(*{**CACHE, **bad}.values()) == code


READ = dict(n=5, slot=P, k_cache=P, v_cache=P, k_exp=P, v_exp=P, k=P, v=P, n_pages=7, page=16, Hkv=4, d=128, kind=E4M3, status=None, stream=None)


@pytest.mark.parametrize("bad,code", [(dict(n=-1), EINVAL), (dict(page=17), EINVAL), (dict(d=96), EUNSUPPORTED), (dict(slot=None), EINVAL), (dict(k=P + 8), EINVAL),
                                      (dict(k_cache=P + 4), EINVAL), (dict(v_exp=None), EINVAL)])
def test_cache_read_refuses(bad, code):
    assert gen.lib.harts_gen_cache_read(*{**READ, **bad}.values()) == code


def test_cache_calls_without_rows_do_nothing():
    assert gen.lib.harts_gen_cache_write(*{**CACHE, "n": 0, "slot": None, "k": None}.values()) == OK
    assert gen.lib.harts_gen_cache_read(*{**READ, "n": 0, "slot": None}.values()) == OK
    assert gen.lib.harts_gen_cache_read(*{**READ, "k": None, "v": None}.values()) == OK


def index(**kw):
    return H.harts_gen_attn_index(**{**dict(tree_node_ptr=[0, 3], node_parent=[-1, 0, 0], node_fork_off=[0, 700, 700], node_len=[700, 5, 9],
                                             node_page_ptr=[0, 11, 12, 13], node_page=list(range(13)), page=64, q_node=[1, 2], q_pos=[4, 8], Hq=8, Hkv=2), **kw})


ATTN = dict(q=P, ld_q=1024, k_cache=P, v_cache=P, k_exp=None, v_exp=None, n_pages=13, kind=BF16, q_pos=P, o=P, lse=P, scale=0.1, ws=P, ws_bytes=1 << 30,
            status=None, stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), EINVAL), (dict(q=P + 8), EINVAL), (dict(ld_q=1016), EINVAL), (dict(ld_q=1028), EINVAL), (dict(k_cache=None), EINVAL),
    (dict(v_cache=P + 8), EINVAL), (dict(kind=E4M3), EINVAL), (dict(kind=0), EUNSUPPORTED), (dict(n_pages=12), EINVAL), (dict(q_pos=None), EINVAL),
    (dict(o=None), EINVAL), (dict(o=P + 8), EINVAL), (dict(lse=None), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(ws=None), EINVAL), (dict(ws=P + 8), EINVAL), (dict(ws_bytes=15), EINVAL), (dict(dev=None), EINVAL),
    (dict(dev=P + 4), EINVAL)])
def test_attn_refuses(bad, code):
    ix = index()
    args = {**dict(host=ix.host_ptr, dev=P), **ATTN, **bad}
    assert gen.lib.harts_gen_attn(*args.values()) == code


def test_attn_refuses_what_is_no_index():
    ix = index()
    n = C.c_size_t(0)
    for blob in (None, np.zeros(32, np.int32), np.full(32, -1, np.int32)):
        p = None if blob is None else blob.ctypes.data_as(C.POINTER(C.c_int32))
        assert gen.lib.harts_gen_attn(p, P, *ATTN.values()) == EINVAL
        assert gen.lib.harts_gen_attn_workspace_bytes(p, C.byref(n)) == EINVAL
    assert gen.lib.harts_gen_attn_workspace_bytes(ix.host_ptr, None) == EINVAL
    assert gen.lib.harts_gen_attn(index(q_node=[], q_pos=[]).host_ptr, P, *ATTN.values()) == OK        # no queries


def test_index_blob_that_is_too_small():
    arrays = [np.array(x, np.int32) for x in ([0, 1], [-1], [0], [5], [0, 1], [0], [0], [4])]
    p = [a.ctypes.data_as(C.POINTER(C.c_int32)) for a in arrays]
    n = C.c_int64(0)
    call = lambda cap, blob: gen.lib.harts_gen_attn_index(1, *p[:6], 16, 1, p[6], p[7], 4, 2, 0, cap, blob, C.byref(n))  # noqa: E731
    assert call(0, None) == OK and n.value >= 32
    blob = np.zeros(n.value, np.int32)
    assert call(n.value - 1, blob.ctypes.data_as(C.POINTER(C.c_int32))) == EINVAL and not blob.any()
    assert call(n.value, blob.ctypes.data_as(C.POINTER(C.c_int32))) == OK


def test_tensors_of_the_host_are_refused():
    x = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(H.HartsError) as e:
        H.harts_gen_la(x, x, x, torch.zeros(3, 4), torch.zeros_like(x), torch.zeros(3, 4, 128, 128), i, i, i, i, 1)
    assert e.value.code == EINVAL
    c = torch.zeros(2, 4, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(H.HartsError):
        H.harts_gen_cache_write(x, x, i, c, c)
    with pytest.raises(H.HartsError):
        H.harts_gen_cache_read(c, c, i, x, x)
    with pytest.raises(H.HartsError):
        H.harts_gen_attn(index(), x, c, c, i, x, torch.zeros(3, 4), 0.1)


def test_attn_refuses_an_infinite_scale():
    args = {**dict(host=index().host_ptr, dev=P), **ATTN, "scale": float("inf")}
    assert gen.lib.harts_gen_attn(*args.values()) == EINVAL


@pytest.mark.parametrize("scale,code", [(np.finfo(np.float32).max, EINVAL), (2.36e38, EINVAL), (2.3586e38, OK)])
def test_attn_refuses_a_scale_that_base_2_exponents_cannot_hold(scale, code):
    """scale / ln 2 in fp32; the one below it is taken (of a call without queries, which launches nothing)."""
    ix = index() if code else index(q_node=[], q_pos=[])
    assert gen.lib.harts_gen_attn(*{**dict(host=ix.host_ptr, dev=P), **ATTN, "scale": float(scale)}.values()) == code


@pytest.mark.parametrize("at", [0, 1, 3, 4])
def test_sizes_that_32_bits_do_not_hold_are_refused(at):
    sizes = [3, 40, 120, 4, 128, 128]
    assert H.harts_gen_la_workspace_bytes(*sizes, torch.bfloat16) > 0
    sizes[at] += 1 << 32
    with pytest.raises(H.HartsError) as e:
        H.harts_gen_la_workspace_bytes(*sizes, torch.bfloat16)
    assert e.value.code == EINVAL
