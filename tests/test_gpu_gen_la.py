"""harts_gen_la on the GPU: the recurrence from and into kept states against its definition token by token in 64 bits."""
import pytest
import torch

import paper_2608_28158_b200 as H

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def oracle(q, k, v, g, states, begin, lens, ins, outs):
    """fp64, on the device: o of the sequences' rows (others NaN) and the pool afterwards."""
    o = torch.full(v.shape, float("nan"), dtype=torch.float64, device=v.device)
    pool = states.double().clone()
    new = {}
    for b, n, i, to in zip(begin, lens, ins, outs):
        S = states[i].double() if i >= 0 else torch.zeros(states.shape[1:], dtype=torch.float64, device=v.device)
        for t in range(b, b + n):
            S = S * g[t].double().exp()[:, None, None] + k[t].double()[:, :, None] * v[t].double()[:, None, :]
            if q is not None:
                o[t] = (q[t].double()[:, None, :] @ S)[:, 0]
        if to >= 0:
            new[to] = S
    for to, S in new.items():
        pool[to] = S
    return o, pool


def problem(lens, heads, d, dtype, seed, gaps=0, strong=False, ld=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    begin, at = [], gaps
    for n in lens:
        begin.append(at)
        at += n + gaps
    rows, n = at, len(lens)

    def tensor(scale):
        x = (normal(rows, heads, d) * scale).to(DT[dtype])
        if ld:                                     # rows of a wider tensor
            wide = torch.full((rows, ld), float("nan"), dtype=DT[dtype], device="cuda")
            y = wide[:, 8:8 + heads * d].view(rows, heads, d)
            y.copy_(x)
            return y
        return x

    q, k, v = tensor(1 / 8), tensor(1 / 8), tensor(1)
    x = normal(rows, heads) + 3
    if strong:
        x[::7] -= 40
    g = torch.nn.functional.logsigmoid(x)
    states = normal(2 * n + 1, heads, d, d) * 0.3
    ins = [2 * i if i % 4 != 3 else -1 for i in range(n)]
    outs = [2 * i + 1 if i % 5 != 4 else -1 for i in range(n)]
    return q, k, v, g, states, begin, ins, outs


def call(q, k, v, g, states, begin, lens, ins, outs, o="new", max_len=None, stream=None):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rows, heads, d = k.shape
    if isinstance(o, str):
        o = torch.full((rows, heads, d), float("nan"), dtype=k.dtype, device="cuda")
    top = max(lens, default=0) if max_len is None else max_len
    ws = torch.empty(max(1, H.harts_gen_la_workspace_bytes(len(lens), top, rows, heads, d, d, k.dtype)), dtype=torch.uint8, device="cuda")
    ws.fill_(255)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    H.harts_gen_la(q, k, v, g, o, states, dev(begin), dev(lens), dev(ins), dev(outs), top, workspace=ws, dev_status=status, stream=stream)
    return o, status


def rel(x, y):
    y = y.double()
    return float((x.double() - y).norm() / y.norm().clamp(min=1e-300))


# fp32 sums of n terms are off by less than n 2^-24 of their terms' sizes, in practice by some 2^-24 sqrt(n); tests' chains of 64 rows
# and up to some hundred effective tokens stay under 1e-5.  Outputs of bf16 calls are rounded once (2^-9 on average 2^-9 / sqrt 3 of a
# value) by the walk; chunks round scores and states too, three roundings of that size: sqrt(3) 2^-9 / sqrt 3 = 2e-3, held to 2^-8.
def tol(dtype, chunked):
    return 1e-5, (1e-5 if dtype == "fp32" else 2.0 ** -8 if chunked else 2.0 ** -9)


def check(lens, heads, d, dtype, seed=0, **kw):
    max_len = kw.pop("max_len", None)
    q, k, v, g, states, begin, ins, outs = problem(lens, heads, d, dtype, seed, **kw)
    ref_o, ref_s = oracle(q, k, v, g, states, begin, lens, ins, outs)
    before = states.clone()
    o, status = call(q, k, v, g, states, begin, lens, ins, outs, max_len=max_len)
    H.harts_la_check(status)
    own = ~torch.isnan(ref_o)
    assert torch.equal(torch.isnan(o), ~own)                     # rows of no sequence are as they were
    ts, to = tol(dtype, dtype == "bf16" and d == 128)
    if own.any():
        assert rel(o[own], ref_o[own]) <= to
    for i in range(states.shape[0]):
        if i in outs:
            assert rel(states[i], ref_s[i]) <= ts, i
        else:
            assert torch.equal(states[i], before[i])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("n,heads", [(1, 1), (5, 4), (70, 5)])
def test_single_tokens(dtype, d, n, heads):
    check([1] * n, heads, d, dtype)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 64), ("fp32", 128)])
def test_short_runs_empty_ones_and_gaps(dtype, d):
    check([0, 1, 2, 3, 7, 8, 9, 16, 5, 0, 11], 3, d, dtype, gaps=2)
    check([3, 0, 8, 1], 130, d, dtype, gaps=1)
    check([3, 0, 14, 1], 130, d, dtype, gaps=1)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("fp32", 64), ("fp32", 128)])
def test_long_runs_token_by_token(dtype, d):
    check([130, 1, 0, 65], 2, d, dtype, gaps=3, strong=True)


@pytest.mark.parametrize("lens,heads", [([21], 1), ([63, 64, 65, 1, 0, 128, 129], 2), ([40] * 30, 8), ([190, 1, 777], 16)])
def test_chunks(lens, heads):
    check(lens, heads, 128, "bf16", gaps=5)


@pytest.mark.parametrize("lens,heads", [([1025], 1), ([1500, 0, 3, 800, 2049], 4), ([700] * 5 + [9], 2), ([4000], 3), ([900, 901, 902], 16)])
def test_segments_of_long_sequences(lens, heads):
    check(lens, heads, 128, "bf16", gaps=1)


def test_strong_decays_in_chunks():
    check([300, 77, 1200], 2, 128, "bf16", strong=True)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("lens", [[1, 3, 2], [100, 900, 1, 1300]])
def test_rows_of_a_wider_tensor(dtype, d, lens):
    check(lens, 2, d, dtype, ld=1024, gaps=1)


@pytest.mark.parametrize("max_len", [17, 21, 5000])
def test_a_bound_far_above_the_lengths(max_len):
    check([1, 2, 0, 17], 2, 128, "bf16", max_len=max_len)


@pytest.mark.parametrize("lens", [[1, 4, 2], [70, 1, 200], [1700, 30]])
def test_in_place_and_a_second_call_continues(lens):
    """Two calls over the halves of the sequences, states in place, give what one call over all gives."""
    q, k, v, g, states, begin, _, _ = problem([2 * n for n in lens], 2, 128, "bf16", 3)
    ins = [2 * i for i in range(len(lens))]
    ref_o, ref_s = oracle(q, k, v, g, states, begin, [2 * n for n in lens], ins, ins)
    o = torch.full_like(v, float("nan"))
    call(q, k, v, g, states, begin, lens, ins, ins, o=o)
    _, status = call(q, k, v, g, states, [b + n for b, n in zip(begin, lens)], lens, ins, ins, o=o)
    H.harts_la_check(status)
    assert rel(o, ref_o) <= 2.0 ** -8
    assert rel(states, ref_s) <= 1e-5


@pytest.mark.parametrize("lens", [[3, 1], [100, 65, 1500]])
def test_states_without_outputs(lens):
    q, k, v, g, states, begin, _, _ = problem(lens, 2, 128, "bf16", 4)
    ins, outs = [0] * len(lens), [1 + i for i in range(len(lens))]            # branches of one state
    _, ref = oracle(None, k, v, g, states, begin, lens, ins, outs)
    _, status = call(None, k, v, g, states, begin, lens, ins, outs, o=None)
    H.harts_la_check(status)
    assert rel(states, ref) <= 1e-5


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_foreign_rows_may_hold_anything(dtype, d):
    """NaN and infinities in rows of no sequence, right behind every sequence and chunk, reach nothing."""
    lens = [1, 5, 66, 130, 20, 1100]
    q, k, v, g, states, begin, ins, outs = problem(lens, 2, d, dtype, 5, gaps=70)
    own = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, n in zip(begin, lens):
        own[b:b + n] = True
    clean = [x.clone() for x in (q, k, v, g)]
    s1, s2 = states.clone(), states.clone()
    o1, _ = call(*clean, s1, begin, lens, ins, outs)
    for x, bad in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (g, float("inf"))):
        x[~own] = bad
    o2, status = call(q, k, v, g, s2, begin, lens, ins, outs)
    H.harts_la_check(status)
    assert torch.equal(s1, s2) and torch.equal(o1[own], o2[own])


@pytest.mark.parametrize("lens", [[1, 2, 3, 1, 2], [100, 30, 700, 64, 50]])
def test_a_bad_sequence_is_left_out_and_reported(lens):
    for what, value in (("in", 99), ("in", -2), ("out", 99), ("out", -2), ("len", max(lens) + 1), ("len", -1), ("begin", -1), ("begin", 100000)):
        q, k, v, g, states, begin, ins, outs = problem(lens, 2, 128, "bf16", 6)
        lens2 = list(lens)
        {"in": ins, "out": outs, "len": lens2, "begin": begin}[what][2] = value
        good = [i for i in range(5) if i != 2]
        pick = lambda x: [x[i] for i in good]  # noqa: E731
        ref_o, ref_s = oracle(q, k, v, g, states, pick(begin), pick(lens), pick(ins), pick(outs))
        o, status = call(q, k, v, g, states, begin, lens2, ins, outs, max_len=max(lens))
        with pytest.raises(H.HartsError) as e:
            H.harts_la_check(status)
        assert e.value.code == -1 and int(status[1]) == 2
        own = ~torch.isnan(ref_o)
        assert torch.equal(torch.isnan(o), ~own)
        assert rel(o[own], ref_o[own]) <= 2.0 ** -8 and rel(states, ref_s) <= 1e-5


@pytest.mark.parametrize("lens", [[1] * 9, [90, 1200, 3]])
def test_captured_replayed_and_the_same_bits_every_time(lens):
    q, k, v, g, states, begin, ins, outs = problem(lens, 4, 128, "bf16", 7)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    o = torch.empty_like(v)
    ws = torch.empty(max(1, H.harts_gen_la_workspace_bytes(len(lens), max(lens), q.shape[0], 4, 128, 128, q.dtype)), dtype=torch.uint8, device="cuda")
    args = (q, k, v, g, o, states, dev(begin), dev(lens), dev(ins), dev(outs), max(lens))
    H.harts_gen_la(*args, workspace=ws)
    torch.cuda.synchronize()
    first = o.clone(), states.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.harts_gen_la(*args, workspace=ws)
    for _ in range(3):
        o.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, first[0]) and torch.equal(states, first[1])
    q.mul_(2)                                       # new values in the same tensors
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, 2 * first[0])


def test_another_stream():
    q, k, v, g, states, begin, ins, outs = problem([5, 300], 2, 128, "bf16", 8)
    s1, s2 = states.clone(), states.clone()
    o1, _ = call(q, k, v, g, s1, begin, [5, 300], ins, outs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    o2 = torch.full_like(o1, float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(q, k, v, g, s2, begin, [5, 300], ins, outs, o=o2)
    side.synchronize()
    assert torch.equal(o1, o2) and torch.equal(s1, s2)


def test_the_framework_s_own_forward_gives_the_same_outputs():
    """A training forward over single-node trees and a sampling call over the same rows."""
    lens = [200, 64, 333]
    fo = ([0, 1, 2, 3], [-1] * 3, [0] * 3, lens)
    plan = H.harts_la_plan(*fo, 64).upload()
    rows = torch.as_tensor(plan.row_of_token.astype("int64"), device="cuda")
    q, k, v, g, states, begin, _, _ = problem(lens, 4, 128, "bf16", 9)
    ws = H.Workspace(plan, 4, 128, 128, torch.bfloat16)
    phys = [torch.empty_like(x) for x in (q, k, v, g)]
    for y, x in zip(phys, (q, k, v, g)):
        y[rows] = x
    ref = torch.empty_like(v)
    H.harts_la_fwd(plan, 0, *phys, ref, ws.slots, ws.chunk_states, dev_status=ws.dev_status)
    o, status = call(q, k, v, g, states, begin, lens, [-1] * 3, [-1] * 3)
    H.harts_la_check(status)
    assert rel(o, ref[rows]) <= 2.0 ** -8


def test_sequences_that_share_rows_beyond_the_workspace_are_refused_on_the_device():
    """Twelve sequences of the same 4,000 rows: more segments than 4,000 rows can have.  None is done, and the call says so."""
    q, k, v, g, states, _, _, _ = problem([4000], 8, 128, "bf16", 11)
    pool = torch.zeros(13, 8, 128, 128, device="cuda")
    o, status = call(q, k, v, g, pool, [0] * 12, [4000] * 12, [-1] * 12, list(range(12)))
    with pytest.raises(H.HartsError) as e:
        H.harts_la_check(status)
    assert e.value.code == -1
    assert bool(torch.isnan(o).all()) and not pool.any()


@pytest.mark.parametrize("dtype,d,lens", [("bf16", 128, [5, 1]), ("fp32", 128, [9, 100]), ("bf16", 128, [300, 77, 1200])])
@pytest.mark.parametrize("value,every", [(float("-inf"), 7), (-1e30, 5), (-3000.0, 1), (-100.0, 2)])
def test_decays_that_leave_nothing(dtype, d, lens, value, every):
    """A gate of any size, minus infinity too, forgets the state and disturbs no row behind it."""
    q, k, v, g, states, begin, ins, outs = problem(lens, 2, d, dtype, 3)
    g[::every] = value
    ref_o, ref_s = oracle(q, k, v, g, states, begin, lens, ins, outs)
    o, status = call(q, k, v, g, states, begin, lens, ins, outs)
    H.harts_la_check(status)
    ts, to = tol(dtype, dtype == "bf16")
    assert rel(o, ref_o) <= to
    for i in outs:
        if i >= 0:
            assert rel(states[i], ref_s[i]) <= ts


@pytest.mark.parametrize("lens,heads", [([1, 0, 3] * 230 + [6000, 2, 2500], 1), ([3840], 2), ([7680, 3840, 1920], 4)])
def test_segments_beside_many_short_sequences_and_without_a_rest(lens, heads):
    check(lens, heads, 128, "bf16")


@pytest.mark.parametrize("lens,heads", [([0] * 300 + [100] + [0] * 300 + [70, 0], 8), ([0] * 90, 64)])
def test_copies_of_states_in_a_call_of_chunks(lens, heads):
    """Forks as sequences without tokens, many in a row: their states come out as they went in."""
    q, k, v, g, states, begin, ins, outs = problem(lens, heads, 128, "bf16", 12, gaps=1)
    before = states.clone()
    o, status = call(q, k, v, g, states, begin, lens, ins, outs, max_len=128)
    H.harts_la_check(status)
    for n, i, to in zip(lens, ins, outs):
        if n == 0 and to >= 0:
            assert torch.equal(states[to], before[i] if i >= 0 else torch.zeros_like(states[to]))
    own = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, n in zip(begin, lens):
        own[b:b + n] = True
    assert not torch.isnan(o[own]).any() and bool(torch.isnan(o[~own]).all())


@pytest.mark.parametrize("lens,heads", [([4000], 2), ([1500, 0, 2049, 70], 4), ([40, 3, 129], 3)])
@pytest.mark.parametrize("pool_off,ws_off", [(0, 16), (16, 0), (16, 16), (0, 48)])
def test_bases_of_16_bytes_alignment_only(lens, heads, pool_off, ws_off):
    """Pool and workspace as slices of larger buffers, each 16 bytes past a multiple of 32 or not: the same bits as in buffers of their own."""
    q, k, v, g, states, begin, ins, outs = problem(lens, heads, 128, "bf16", 13)
    first, dev = states.clone(), lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    o1, _ = call(q, k, v, g, first, begin, lens, ins, outs)

    def placed(n_bytes, off):
        buf = torch.full((n_bytes + 512,), 255, dtype=torch.uint8, device="cuda")
        at = -buf.data_ptr() % 256 + off
        assert (buf.data_ptr() + at) % 32 == off % 32
        return buf[at:at + n_bytes]

    pool = placed(states.numel() * 4, pool_off).view(torch.float32).view(states.shape)
    pool.copy_(states)
    ws = placed(H.harts_gen_la_workspace_bytes(len(lens), max(lens), q.shape[0], heads, 128, 128, q.dtype), ws_off)
    o2, status = torch.full_like(o1, float("nan")), torch.zeros(4, dtype=torch.int32, device="cuda")
    H.harts_gen_la(q, k, v, g, o2, pool, dev(begin), dev(lens), dev(ins), dev(outs), max(lens), workspace=ws, dev_status=status)
    H.harts_la_check(status)
    assert torch.equal(o1, o2) and torch.equal(first, pool)


@pytest.mark.parametrize("lens,heads", [([1] * 60 + [2000], 32), ([5000, 1, 1, 40, 1, 3000] + [1] * 30, 16), ([1, 1, 2500, 0, 13, 1], 48)])
def test_single_tokens_and_prompts_in_one_call(lens, heads):
    check(lens, heads, 128, "bf16", seed=14)


def at_16(x):
    """x in a buffer of its own, 16 bytes past a multiple of 256."""
    n = x.numel() * x.element_size()
    buf = torch.full((n + 512,), 255, dtype=torch.uint8, device="cuda")
    off = -buf.data_ptr() % 256 + 16
    y = buf[off:off + n].view(x.dtype).view(x.shape)
    return y.copy_(x)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 64), ("fp32", 128)])
@pytest.mark.parametrize("lens", [[1, 3, 1], [30, 0, 130, 700]])
def test_tensors_of_16_bytes_alignment_only(dtype, d, lens):
    q, k, v, g, states, begin, ins, outs = problem(lens, 3, d, dtype, 15, gaps=1)
    pool = at_16(states)
    o1, _ = call(q, k, v, g, states, begin, lens, ins, outs)
    o2 = at_16(torch.full_like(v, float("nan")))
    _, status = call(at_16(q), at_16(k), at_16(v), at_16(g), pool, begin, lens, ins, outs, o=o2)
    H.harts_la_check(status)
    assert torch.equal(torch.nan_to_num(o1), torch.nan_to_num(o2)) and torch.equal(torch.isnan(o1), torch.isnan(o2)) and torch.equal(states, pool)
