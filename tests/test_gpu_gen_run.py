"""The sampling calls together, as a decoding loop makes them, against the training passes over the finished tree."""
import math

import numpy as np
import pytest
import torch

import paper_2608_28158_b200 as H

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def finished_tree(seed):
    """Two prompts, branches that fork at the prompt's end, inside it, and off another branch."""
    ptr = [0, 5, 7]
    par = [-1, 0, 0, 0, 1, -1, 0]
    off = [0, 150, 150, 101, 9, 0, 70]
    ln = [150, 20, 33, 7, 12, 70, 25]
    return ptr, par, off, ln


def draw(n, hq, hkv, H_la, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    bf = lambda x: x.to(torch.bfloat16)  # noqa: E731
    return {"q": bf(normal(n, hq, 128)), "k": bf(normal(n, hkv, 128)), "v": bf(normal(n, hkv, 128)), "lq": bf(normal(n, H_la, 128) / 8),
            "lk": bf(normal(n, H_la, 128) / 8), "lv": bf(normal(n, H_la, 128)), "g": torch.nn.functional.logsigmoid(normal(n, H_la) + 3)}


def training(forest, x, hq, scale):
    """The framework's training forwards over all compact tokens, canonical order."""
    n = sum(forest[3])
    plan = H.harts_la_plan(*forest, 64).upload()
    rows = torch.as_tensor(plan.row_of_token.astype(np.int64), device="cuda")
    phys = {name: torch.empty_like(t) for name, t in x.items()}
    for name, t in x.items():
        phys[name][rows] = t
    H_la = x["lq"].shape[1]
    ws = H.Workspace(plan, H_la, 128, 128, torch.bfloat16)
    lo = torch.empty_like(phys["lv"])
    H.harts_la_fwd(plan, 0, phys["lq"], phys["lk"], phys["lv"], phys["g"], lo, ws.slots, ws.chunk_states, dev_status=ws.dev_status)
    index = H.harts_attn_index(*forest, plan.row_of_token).upload()
    o, lse = torch.empty_like(phys["q"]), torch.empty(n, hq, device="cuda")
    H.harts_attn_fwd(index, phys["q"], phys["k"], phys["v"], o, lse, scale, dev_status=ws.dev_status)
    H.harts_la_check(ws.dev_status)
    return lo[rows], o[rows], lse[rows]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("graph", [False, True])
def test_a_tree_is_sampled_as_it_is_trained_on(kind, graph):
    hq, hkv, H_la, page, scale = 8, 2, 4, 16, 1 / math.sqrt(128)
    forest = finished_tree(0)
    ptr, par, off, ln = forest
    base = np.concatenate([[0], np.cumsum(ln)])
    x = draw(int(base[-1]), hq, hkv, H_la, 1)
    if kind == "e4m3":        # what the cache holds is what the training pass is given
        c = [torch.zeros(64, hkv, page, 128, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
        e = [torch.zeros(64, hkv, page, dtype=torch.uint8, device="cuda") for _ in range(2)]
        slot = torch.arange(int(base[-1]), **I32)
        H.harts_gen_cache_write(x["k"], x["v"], slot, *c, *e)
        H.harts_gen_cache_read(*c, slot, x["k"], x["v"], *e)
    want = training(forest, x, hq, scale)

    # pages of every node, in any order; a pool of states: one for each node's end and one at the fork inside the first prompt
    counts = [-(-n // page) for n in ln]
    order = np.random.default_rng(0).permutation(sum(counts) + 2)
    page_ptr = np.concatenate([[0], np.cumsum(counts)])
    pages = order[:page_ptr[-1]]
    slot_of = lambda v, j: int(pages[page_ptr[v] + j // page]) * page + j % page  # noqa: E731
    f8 = kind == "e4m3"
    cache = [torch.full((len(order), hkv, page, 128), 0 if f8 else float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    if f8:
        cache = [t.to(torch.float8_e4m3fn) for t in cache]
        cache[0].view(torch.uint8).fill_(0x7f)
    exps = [torch.full((len(order), hkv, page), 255, dtype=torch.uint8, device="cuda") if f8 else None for _ in range(2)]
    states = torch.full((9, H_la, 128, 128), float("nan"), device="cuda")
    o_la, o_at = torch.zeros_like(x["lv"]), torch.zeros_like(x["q"])
    lse = torch.zeros(x["q"].shape[:2], device="cuda")
    status = torch.zeros(4, **I32)

    # prompts: the first in two parts, as a branch forks at its token 101 (state 7); keys and values into the cache
    def la(begin, lens, ins, outs):
        ws = torch.empty(max(1, H.harts_gen_la_workspace_bytes(len(lens), max(lens), x["lq"].shape[0], H_la, 128, 128, torch.bfloat16)), dtype=torch.uint8,
                         device="cuda")
        H.harts_gen_la(x["lq"], x["lk"], x["lv"], x["g"], o_la, states, *(torch.tensor(t, **I32) for t in (begin, lens, ins, outs)), max(lens), workspace=ws,
                       dev_status=status)

    la([0, int(base[5])], [101, 70], [-1, -1], [7, 5])
    la([101], [49], [7], [0])
    for v in (0, 5):
        r = slice(int(base[v]), int(base[v]) + ln[v])
        H.harts_gen_cache_write(x["k"][r], x["v"][r], torch.tensor([slot_of(v, j) for j in range(ln[v])], **I32), *cache, *exps, dev_status=status)

    def decode(nodes, starts):
        """All tokens of `nodes`, a token of each a step; a node that is done stays as padding."""
        n = len(nodes)
        have = [0 if v in nodes else ln[v] for v in range(7)]           # nothing of the new ones yet
        index = H.harts_gen_attn_index(ptr, par, [min(f, have[p + (0 if i < 5 else 5)]) if p >= 0 else 0 for i, (f, p) in enumerate(zip(off, par))], have,
                                       page_ptr, pages, page, nodes, [-1] * n, hq, hkv, grow=64).upload()
        ws = torch.empty(max(1, index.workspace_bytes), dtype=torch.uint8, device="cuda")
        b = {k: torch.zeros(n, *t.shape[1:], dtype=t.dtype, device="cuda") for k, t in x.items()}
        pos, slots, lens, ins, outs = (torch.zeros(n, **I32) for _ in range(5))
        begin = torch.arange(n, **I32)
        lo, o, l = torch.zeros_like(b["lv"]), torch.zeros_like(b["q"]), torch.zeros(n, hq, device="cuda")

        def step():
            H.harts_gen_cache_write(b["k"], b["v"], slots, *cache, *exps, dev_status=status)
            H.harts_gen_attn(index, b["q"], *cache, pos, o, l, scale, workspace=ws, k_exp=exps[0], v_exp=exps[1], dev_status=status)
            H.harts_gen_la(b["lq"], b["lk"], b["lv"], b["g"], lo, states, begin, lens, ins, outs, 1, dev_status=status)

        recorded = None
        for t in range(max(ln[v] for v in nodes)):
            live = [t < ln[v] for v in nodes]
            rows = [int(base[v]) + min(t, ln[v] - 1) for v in nodes]
            for name in b:
                b[name].copy_(x[name][rows])
            pos.copy_(torch.tensor([min(t, ln[v] - 1) for v in nodes], **I32))
            slots.copy_(torch.tensor([slot_of(v, t) if a else -1 for v, a in zip(nodes, live)], **I32))
            lens.copy_(torch.tensor([int(a) for a in live], **I32))
            ins.copy_(torch.tensor([s if t == 0 else v for v, s in zip(nodes, starts)], **I32))
            outs.copy_(torch.tensor([v if a else -1 for v, a in zip(nodes, live)], **I32))
            if graph and t == 1:                                        # (the first step has made everything that is made once)
                torch.cuda.synchronize()
                recorded = torch.cuda.CUDAGraph()
                with torch.cuda.graph(recorded):
                    step()
            if recorded is not None:
                recorded.replay()
            else:
                step()
            for i, a in enumerate(live):
                if a:
                    o_la[rows[i]], o_at[rows[i]], lse[rows[i]] = lo[i], o[i], l[i]

    # four branches at once; the one that forks off node 1 follows when its parent is there, from the parent's state at token 9
    keep = [x[n][int(base[1]):int(base[1]) + 9] for n in ("lq", "lk", "lv", "g")]
    ws9 = [torch.tensor(t, **I32) for t in ([0], [9], [0], [8])]
    H.harts_gen_la(*keep, None, states, *ws9, 9, dev_status=status)       # (only the state of that fork is wanted)
    decode([1, 2, 3, 6], [0, 0, 7, 5])
    decode([4], [8])
    H.harts_la_check(status)

    def rel(a, b):
        return float((a.double() - b.double()).norm() / b.double().norm())

    sampled = torch.zeros(int(base[-1]), dtype=torch.bool, device="cuda")
    for v in (1, 2, 3, 4, 6):
        sampled[int(base[v]):int(base[v]) + ln[v]] = True
    # both passes round scores and states to bf16 (2e-3 each of the output), independently
    assert rel(o_la, want[0]) <= 2.0 ** -8
    assert rel(o_at[sampled], want[1][sampled]) <= 2.0 ** -8
    assert float((lse[sampled] - want[2][sampled]).abs().max()) <= 1e-4


def test_what_python_refuses():
    q = torch.zeros(6, 4, 128, dtype=torch.bfloat16, device="cuda")
    g, states, i = torch.zeros(6, 4, device="cuda"), torch.zeros(3, 4, 128, 128, device="cuda"), torch.zeros(2, **I32)
    ok = dict(q=q, k=q.clone(), v=q.clone(), g=g, o=torch.zeros_like(q), states=states, seq_begin=i, seq_len=i, in_state=i, out_state=i - 1, max_len=1)
    H.harts_gen_la(**ok)
    wrong = [dict(q=q.float()), dict(k=q[:5]), dict(v=q[:, :3]), dict(v=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(g=g.double()), dict(g=g[:5]),
             dict(o=torch.zeros(6, 8, 128, dtype=torch.bfloat16, device="cuda")[:, ::2]), dict(states=states.bfloat16()), dict(states=states[:, :, :64]),
             dict(seq_len=i.long()), dict(in_state=i[:1]), dict(seq_begin=i[None]), dict(q=None), dict(max_len=-1), dict(max_len=40),
             dict(k=q.half()), dict(dev_status=torch.zeros(1, **I32)), dict(g=g.cpu())]
    for kw in wrong:
        with pytest.raises(H.HartsError):
            H.harts_gen_la(**{**ok, **kw})
    c = torch.zeros(4, 4, 16, 128, dtype=torch.bfloat16, device="cuda")
    s6 = torch.zeros(6, **I32)
    for args in ((q, q, s6[:5], c, c), (q.float(), q, s6, c, c), (q, q, s6, c, c[:3]), (q, q, s6, c.half(), c.half()), (q, q, s6, c, c, s6, s6),
                 (q, q[:, :, :64], s6, c, c), (q, q, s6, c.to(torch.float8_e4m3fn), c.to(torch.float8_e4m3fn))):
        with pytest.raises(H.HartsError):
            H.harts_gen_cache_write(*args)
    ix = H.harts_gen_attn_index([0, 1], [-1], [0], [5], [0, 1], [0], 16, [0] * 6, [4] * 6, 4, 4)
    o, lse = torch.zeros_like(q), torch.zeros(6, 4, device="cuda")
    with pytest.raises(H.HartsError):
        H.harts_gen_attn(ix, q, c, c, s6, o, lse, 0.1)                    # not uploaded
    ix.upload()
    H.harts_gen_attn(ix, q, c, c, s6 + 4, o, lse, 0.1, torch.zeros(max(16, ix.workspace_bytes), dtype=torch.uint8, device="cuda"))
    for kw in (dict(q=q[:5]), dict(k_cache=c[:, :2]), dict(q_pos=s6.long()), dict(o=o.float()), dict(lse=lse.double()), dict(scale=0.0)):
        with pytest.raises(H.HartsError):
            H.harts_gen_attn(**{**dict(index=ix, q=q, k_cache=c, v_cache=c, q_pos=s6, o=o, lse=lse, scale=0.1), **kw})
    torch.cuda.synchronize()
