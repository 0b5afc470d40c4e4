"""harts_gen_attn on the GPU: attention of sampled tokens on a cached tree against its definition, query by query in 64 bits."""
import ctypes
import math
import random

import numpy as np
import pytest
import torch

import paper_2608_28158_b200 as H

pytestmark = pytest.mark.gpu


class Tree:
    """A cached forest in random pages; all other places of the pages hold NaN (bf16) or any bytes (8 bits)."""

    def __init__(self, ptr, par, off, ln, page, hkv, kind, seed, grow=0, spare=3, scale=1.0):
        rng = random.Random(seed)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.ptr, self.par, self.off, self.len, self.page, self.hkv, self.kind, self.grow = ptr, par, off, ln, page, hkv, kind, grow
        counts = [-(-(n + grow) // page) for n in ln]
        order = list(range(sum(counts) + spare))
        rng.shuffle(order)
        self.page_ptr, self.pages, n_pages = np.concatenate([[0], np.cumsum(counts)]), order[:sum(counts)], len(order)
        slots = []
        for v, n in enumerate(ln):
            at = np.asarray(self.pages[self.page_ptr[v]:self.page_ptr[v + 1]], dtype=np.int64)
            j = np.arange(n + grow)
            slots.append(torch.as_tensor(at[j // page] * page + j % page if n + grow else np.zeros(0, np.int64)).cuda())
        self.slots = slots
        self.exp = [None, None]
        self.cache, self.values = [], []
        for i in range(2):
            x = torch.randn(n_pages, hkv, page, 128, generator=gen, device="cuda") * scale
            if kind == "bf16":
                c = x.to(torch.bfloat16)
                c.view(-1)[torch.randint(0, 3, (c.numel(),), generator=gen, device="cuda") == 0] += 0
                used = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
                for v, n in enumerate(ln):
                    s = slots[v][:n + grow]
                    used[s // page, s % page] = True
                c.transpose(1, 2)[~used] = float("nan") if i == 0 else float("inf")
                self.cache.append(c)
                self.values.append(c.double())
            else:
                c = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
                e = torch.randint(117, 124, (n_pages, hkv, page), generator=gen, device="cuda").to(torch.uint8)
                self.cache.append(c)
                self.exp[i] = e
                self.values.append(c.float().double() * (e.cpu().double() - 127).exp2().cuda()[..., None])

    def index(self, q_node, q_pos, G):
        return H.harts_gen_attn_index(self.ptr, self.par, self.off, self.len, self.page_ptr, self.pages, self.page, q_node, q_pos, G * self.hkv, self.hkv,
                                      self.grow).upload()

    def visible(self, v, p):
        base = max(x for x in self.ptr if x <= v)
        parts = [self.slots[v][:p + 1]]
        while self.par[v] >= 0:
            u = base + self.par[v]
            parts.append(self.slots[u][:self.off[v]])
            v = u
        return torch.cat(parts)

    def oracle(self, q, q_node, q_pos, scale):
        n, hq, _ = q.shape
        o = torch.zeros(n, hq, 128, dtype=torch.float64, device="cuda")
        lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
        K, V = (x.transpose(1, 2).reshape(-1, self.hkv, 128) for x in self.values)
        for r in range(n):
            if q_node[r] < 0:
                continue
            at = self.visible(q_node[r], q_pos[r])
            if len(at) == 0:
                continue
            s = torch.einsum("hgd,thd->hgt", q[r].double().view(self.hkv, -1, 128), K[at]) * scale
            lse[r] = torch.logsumexp(s, -1).reshape(hq)
            o[r] = torch.einsum("hgt,thd->hgd", torch.softmax(s, -1), V[at]).reshape(hq, 128)
        return o, lse


def run(tree, index, q, q_pos, scale, ws=None, stream=None):
    n, hq, _ = q.shape
    o = torch.full((n, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, hq), float("nan"), device="cuda")
    if ws is None:
        ws = torch.full((max(16, index.workspace_bytes),), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    pos = torch.tensor(q_pos, dtype=torch.int32, device="cuda")
    H.harts_gen_attn(index, q, *tree.cache, pos, o, lse, scale, workspace=ws, k_exp=tree.exp[0], v_exp=tree.exp[1], dev_status=status, stream=stream)
    return o, lse, status


def queries(n, hq, seed, scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1000)
    return (torch.randn(n, hq, 128, generator=gen, device="cuda") * scale).to(torch.bfloat16)


# A p is rounded to bf16 (off by 2^-9 of it at most) and so is the output, once (2^-9): 2 x 2^-9 = 2^-8 of the output's size where the p's
# errors add up, which over rows of many values they do not.  lse: fp32 sums of bf16 products, 2^-24 a step over log terms: 2e-5 absolute.
def compare(o, lse, ref_o, ref_lse):
    none = torch.isneginf(ref_lse)
    assert torch.equal(torch.isneginf(lse), none)
    assert not o[none].any()
    if (~none).any():
        d = o.double()[~none] - ref_o[~none]
        assert float(d.norm() / ref_o[~none].norm()) <= 2.0 ** -8
        rows = d.norm(dim=-1) / ref_o[~none].norm(dim=-1)
        assert float(rows.max()) <= 2.0 ** -6            # a row of few tokens: sums of a few rounded p's
        assert float((lse.double() - ref_lse)[~none].abs().max()) <= 2e-5 * max(1.0, float(ref_lse[~none].abs().max()))


def check(tree, q_node, q_pos, G, seed=0, later=None, scale=1 / math.sqrt(128), q_scale=1.0):
    index = tree.index(q_node, q_pos, G)
    q = queries(len(q_node), G * tree.hkv, seed, q_scale)
    pos = list(q_pos) if later is None else later
    o, lse, status = run(tree, index, q, pos, scale)
    H.harts_la_check(status)
    compare(o, lse, *tree.oracle(q, q_node, pos, scale))
    return index


KINDS = ["bf16", "e4m3"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 15, 16, 63, 64, 65, 129, 1000])
def test_one_sequence(kind, page, n):
    tree = Tree([0, 1], [-1], [0], [n], page, 2, kind, n)
    check(tree, [0], [n - 1], 4, n)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G,hkv", [(1, 1), (1, 5), (3, 2), (5, 1), (8, 4), (16, 1), (17, 2), (40, 1)])
def test_head_layouts(kind, G, hkv):
    tree = Tree([0, 4], [-1, 0, 0, 0], [0, 200, 200, 137], [200, 30, 71, 5], 32, hkv, kind, G)
    check(tree, [1, 2, 3], [29, 70, 4], G, G)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches,prefix", [(2, 64), (7, 700), (33, 1025), (64, 333), (150, 4000)])
def test_branches_of_a_prompt(kind, branches, prefix):
    rng = random.Random(branches)
    ln = [prefix] + [rng.randint(1, 300) for _ in range(branches)]
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [prefix] * branches, ln, 64, 2, kind, branches)
    check(tree, list(range(1, branches + 1)), [n - 1 for n in ln[1:]], 4, branches)


def any_forest(rng, trees, nodes, long=900):
    ptr, par, off, ln = [0], [], [], []
    for _ in range(trees):
        t = [(-1, 0, rng.choice([0, 1, 63, 64, 500, long]))]
        for i in range(1, nodes):
            p = rng.randrange(i)
            t.append((p, rng.randint(0, t[p][2]), rng.choice([0, 1, 2, 40, 64, 130, 300])))
        par += [x[0] for x in t]
        off += [x[1] for x in t]
        ln += [x[2] for x in t]
        ptr.append(len(par))
    return ptr, par, off, ln


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("seed", range(8))
def test_any_tree_with_drafts_and_padding(kind, seed):
    rng = random.Random(seed)
    ptr, par, off, ln = any_forest(rng, rng.randint(1, 3), rng.choice([3, 12, 30]))
    tree = Tree(ptr, par, off, ln, rng.choice([16, 32, 64, 128]), rng.choice([1, 2]), kind, seed)
    q_node, q_pos = [], []
    for v in range(len(ln)):
        c = min(rng.choice([0, 1, 1, 2, 4, 9]), ln[v] + 1)
        q_node += [v] * c
        q_pos += [ln[v] - c + i for i in range(c)]
        if rng.random() < 0.2:
            q_node.append(-1)
            q_pos.append(rng.randint(-5, 5))
    check(tree, q_node + [-1], q_pos + [0], rng.choice([1, 4, 8]), seed)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G", [2, 8])
def test_the_index_serves_growing_branches(kind, G):
    ln = [777, 0, 10, 63, 100, 200]
    tree = Tree([0, 6], [-1, 0, 0, 0, 0, 4], [0, 777, 777, 300, 777, 50], ln, 32, 2, kind, 5, grow=70)
    q_node = [1, 2, 3, 4, 5, 5, 5]
    q_pos = [-1, 9, 62, 99, 197, 198, 199]
    for step in (0, 1, 2, 35, 70):
        check(tree, q_node, q_pos, G, step, later=[p + step for p in q_pos])


@pytest.mark.parametrize("kind", KINDS)
def test_large_scores_and_far_apart_maxima(kind):
    """Scores of some hundreds, growing along the sequence, so that the running maximum is raised again and again."""
    tree = Tree([0, 1], [-1], [0], [2000], 64, 1, kind, 3)
    grow = torch.linspace(0.01, 4, 2000, device="cuda").double()
    at = tree.slots[0]
    if kind == "bf16":
        c = tree.cache[0]
        c[at // 64, 0, at % 64] = (c[at // 64, 0, at % 64].double() * grow[:, None]).to(torch.bfloat16)
        tree.values[0] = c.double()
    check(tree, [0] * 3, [10, 1500, 1999], 8, 3, q_scale=8.0)


@pytest.mark.parametrize("G", [1, 4, 8])
def test_tokens_that_a_query_does_not_see_may_hold_anything_8_bits(G):
    """The same with NaN bytes, in places that no query sees and in later drafts, which see them."""
    tree = Tree([0, 3], [-1, 0, 0], [0, 100, 70], [131, 40, 9], 16, 1, "e4m3", 4)
    q_node, q_pos = [1, 1, 1, 2], [36, 37, 39, 8]
    index = tree.index(q_node, q_pos, G)
    q = queries(4, G, 4)
    clean, clean_lse, _ = run(tree, index, q, q_pos, 0.1)
    compare(clean, clean_lse, *tree.oracle(q, q_node, q_pos, 0.1))
    used = torch.zeros(tree.cache[0].shape[0], 16, dtype=torch.bool, device="cuda")
    for s in (tree.slots[0][:100], tree.slots[1][:38], tree.slots[2]):
        used[s // 16, s % 16] = True
    for i in range(2):
        tree.cache[i].view(torch.uint8).transpose(1, 2)[~used] = 0x7f if i else 0xff
        tree.exp[i].transpose(1, 2)[~used] = 254
    o, lse, status = run(tree, index, q, q_pos, 0.1)
    H.harts_la_check(status)
    assert bool(torch.isnan(o[2]).all())
    for r in (0, 1, 3):
        assert float((o[r].double() - clean[r].double()).norm()) <= 2.0 ** -8 * float(clean[r].double().norm()) and torch.equal(lse[r], clean_lse[r])


@pytest.mark.parametrize("G", [1, 8, 16])
def test_tokens_that_a_query_does_not_see_may_hold_anything(G):
    """Drafts: later drafts' keys and values infinite or NaN; a fork: the parent's tokens behind it.  (All places of no node hold NaN already.)"""
    tree = Tree([0, 3], [-1, 0, 0], [0, 100, 70], [131, 40, 9], 16, 1, "bf16", 4)
    q_node, q_pos = [1, 1, 1, 2], [36, 37, 39, 8]
    index = tree.index(q_node, q_pos, G)
    q = queries(4, G, 4)
    clean, clean_lse, _ = run(tree, index, q, q_pos, 0.1)
    compare(clean, clean_lse, *tree.oracle(q, q_node, q_pos, 0.1))
    for value in (float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min):
        for i in range(2):
            at = torch.cat([tree.slots[1][38:40], tree.slots[0][100:]])
            tree.cache[i][at // 16, 0, at % 16] = value
        o, lse, status = run(tree, index, q, q_pos, 0.1)
        H.harts_la_check(status)
        for r in (0, 1, 3):
            assert float((o[r].double() - clean[r].double()).norm()) <= 2.0 ** -8 * float(clean[r].double().norm()) and torch.equal(lse[r], clean_lse[r])


def test_a_nan_that_is_seen_comes_out_as_one():
    tree = Tree([0, 3], [-1, 0, 0], [0, 300, 300], [300, 40, 9], 16, 2, "bf16", 4)
    s = tree.slots[0][5]
    tree.cache[1][s // 16, 0, s % 16, 3] = float("nan")
    s = tree.slots[1][7]
    tree.cache[0][s // 16, 1, s % 16, 3] = float("nan")
    index = tree.index([1, 2], [39, 8], 4)
    o, lse, _ = run(tree, index, queries(2, 8, 4), [39, 8], 0.1)
    want = torch.zeros(2, 8, 128, dtype=torch.bool, device="cuda")
    want[:, :4, 3] = True                       # the value, seen by both
    want[0, 4:] = True                          # the key, seen by the first
    assert torch.equal(torch.isnan(o), want)
    assert torch.equal(torch.isnan(lse), want.all(-1))


def test_rows_of_nan_in_an_8_bit_cache():
    tree = Tree([0, 3], [-1, 0, 0], [0, 300, 300], [300, 40, 9], 16, 2, "e4m3", 4)
    s = tree.slots[1][7]
    tree.exp[1][s // 16, 1, s % 16] = 255
    index = tree.index([1, 2], [39, 8], 4)
    o, lse, _ = run(tree, index, queries(2, 8, 4), [39, 8], 0.1)
    want = torch.zeros(2, 8, 128, dtype=torch.bool, device="cuda")
    want[0, 4:] = True
    assert torch.equal(torch.isnan(o), want) and not torch.isnan(lse).any()


@pytest.mark.parametrize("kind", KINDS)
def test_a_long_sequence_is_split(kind):
    tree = Tree([0, 2], [-1, -1][:1] + [0], [0, 30000], [30000, 77], 64, 2, kind, 6)
    index = check(tree, [1, 1], [75, 76], 4, 6)
    assert index.n_narrow + index.n_wide > 20


@pytest.mark.parametrize("kind", KINDS)
def test_captured_replayed_and_the_same_bits(kind):
    ln = [900] + [50] * 40
    tree = Tree([0, 41], [-1] + [0] * 40, [0] + [900] * 40, ln, 64, 2, kind, 7, grow=20)
    q_node, q_pos = list(range(1, 41)), [49] * 40
    index = tree.index(q_node, q_pos, 4)
    q = queries(40, 8, 7)
    ws = torch.full((index.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
    o, lse, _ = run(tree, index, q, q_pos, 0.1, ws)
    o2, lse2, pos = torch.empty_like(o), torch.empty_like(lse), torch.tensor(q_pos, dtype=torch.int32, device="cuda")
    call = lambda: H.harts_gen_attn(index, q, *tree.cache, pos, o2, lse2, 0.1, workspace=ws, k_exp=tree.exp[0], v_exp=tree.exp[1])  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        o2.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    pos += 13                                             # the branches have grown
    graph.replay()
    torch.cuda.synchronize()
    compare(o2, lse2, *tree.oracle(q, q_node, [62] * 40, 0.1))


def test_positions_out_of_range_are_brought_in_and_reported():
    ln = [500, 70, 130]
    tree = Tree([0, 3], [-1, 0, 0], [0, 500, 500], ln, 32, 1, "bf16", 8, grow=10)
    q_node, q_pos = [1, 2], [69, 129]
    index = tree.index(q_node, q_pos, 4)
    q = queries(2, 4, 8)
    for r, bad, used in ((1, 140, 139), (0, 80, 79), (0, 2 ** 31 - 1, 79), (0, 68, 69), (1, -1, 129), (1, -2 ** 31, 129)):
        pos = list(q_pos)
        pos[r] = bad
        o, lse, status = run(tree, index, q, pos, 0.1)
        with pytest.raises(H.HartsError):
            H.harts_la_check(status)
        assert int(status[1]) == r
        pos[r] = used
        compare(o, lse, *tree.oracle(q, q_node, pos, 0.1))


@pytest.mark.parametrize("kind", KINDS)
def test_queries_of_a_wider_tensor_and_another_stream(kind):
    tree = Tree([0, 3], [-1, 0, 0], [0, 300, 300], [300, 40, 9], 16, 2, kind, 9)
    index = tree.index([1, 2], [39, 8], 4)
    wide = torch.randn(2, 1024 + 256, device="cuda").to(torch.bfloat16)
    q = wide[:, 128:128 + 1024].view(2, 8, 128)
    a, la, _ = run(tree, index, q.contiguous(), [39, 8], 0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b, lb, _ = run(tree, index, q, [39, 8], 0.1)
    side.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_nothing_to_see():
    tree = Tree([0, 2], [-1, 0], [0, 0], [50, 0], 16, 1, "bf16", 10)
    check(tree, [1, -1, 0], [-1, 7, 49], 4)
    check(tree, [1], [-1], 4)
    check(tree, [-1, -1], [3, 0], 4)


@pytest.mark.parametrize("n", [1, 5, 40])
def test_values_whose_powers_differ_much(n):
    """8 bits: the value that a row attends to most may be 2^40 below its neighbours', and all of a sequence's may be tiny or NaN."""
    tree = Tree([0, 1], [-1], [0], [n], 16, 1, "e4m3", 20 + n)
    e = torch.randint(60, 190, tree.exp[1].shape, device="cuda").to(torch.uint8)
    tree.exp[1].copy_(e)
    tree.values[1] = tree.cache[1].float().double() * (e.cpu().double() - 127).exp2().cuda()[..., None]
    check(tree, [0], [n - 1], 8, n, q_scale=30.0, scale=0.5)
    tree.exp[1].fill_(255)
    index = tree.index([0], [n - 1], 8)
    o, lse, _ = run(tree, index, queries(1, 8, n), [n - 1], 0.1)
    assert bool(torch.isnan(o).all()) and not bool(torch.isnan(lse).any())


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1e4, 1e20])
def test_queries_of_any_size(scale):
    for kind in KINDS:
        tree = Tree([0, 1], [-1], [0], [200], 32, 2, kind, 30)
        check(tree, [0, 0], [150, 199], 4, 30, q_scale=scale, scale=0.1 / scale)


@pytest.mark.parametrize("drafts,n", [(8, 640), (8, 641), (3, 64)])
def test_positions_below_the_index_s_are_reported_by_shared_runs_too(drafts, n):
    tree = Tree([0, 1], [-1], [0], [n], 64, 1, "bf16", 12)
    q_pos = [n - 1] * drafts
    index = tree.index([0] * drafts, q_pos, 8)
    q = queries(drafts, 8, 12)
    o, lse, status = run(tree, index, q, [n - 1] * (drafts - 1) + [n - 2], 0.1)
    with pytest.raises(H.HartsError):
        H.harts_la_check(status)
    assert int(status[1]) == drafts - 1
    compare(o, lse, *tree.oracle(q, [0] * drafts, q_pos, 0.1))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [1, 5])
def test_pages_far_into_a_large_cache(kind, rows):
    """Places beyond 2^32 bytes and elements."""
    n_pages, hkv, page, n = 70000, 4, 128, 300
    dt = torch.float8_e4m3fn if kind == "e4m3" else torch.bfloat16
    cache = [torch.zeros(n_pages, hkv, page, 128, dtype=dt, device="cuda") for _ in range(2)]
    exps = [torch.full((n_pages, hkv, page), 120, dtype=torch.uint8, device="cuda") if kind == "e4m3" else None for _ in range(2)]
    pages = [n_pages - 1, n_pages // 2 + 1, n_pages - 7]
    kv = [torch.randn(n, hkv, 128, device="cuda").to(torch.bfloat16) for _ in range(2)]
    slot = torch.tensor([pages[j // page] * page + j % page for j in range(n)], dtype=torch.int32, device="cuda")
    H.harts_gen_cache_write(*kv, slot, *cache, *exps)
    H.harts_gen_cache_read(*cache, slot, *kv, *exps)
    q_node, q_pos = [0] * rows, [n - 1 - i for i in range(rows)]
    index = H.harts_gen_attn_index([0, 1], [-1], [0], [n], [0, 3], pages, page, q_node, q_pos, 16 * hkv, hkv).upload()
    q = queries(rows, 16 * hkv, 1)
    o, lse = torch.empty_like(q), torch.empty(rows, 16 * hkv, device="cuda")
    ws = torch.empty(max(16, index.workspace_bytes), dtype=torch.uint8, device="cuda")
    H.harts_gen_attn(index, q, *cache, torch.tensor(q_pos, dtype=torch.int32, device="cuda"), o, lse, 0.1, ws, *exps)
    for r, p in enumerate(q_pos):
        s = torch.einsum("hgd,thd->hgt", q[r].double().view(hkv, 16, 128), kv[0][:p + 1].double()) * 0.1
        ref = torch.einsum("hgt,thd->hgd", torch.softmax(s, -1), kv[1][:p + 1].double()).reshape(-1, 128)
        assert float((o[r].double() - ref).norm() / ref.norm()) <= 2.0 ** -8


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,G", [(1, 4), (3, 4), (16, 8), (40, 4)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_of_nan_or_infinity_reaches_no_other(kind, n, G, bad):
    tree = Tree([0, n + 1], [-1] + [0] * n, [0] + [700] * n, [700] + [70] * n, 32, 2, kind, 5)
    node, pos = list(range(1, n + 1)), [69] * n
    index, q = tree.index(node, pos, G), queries(n, 2 * G, 1)
    o, lse, _ = run(tree, index, q, pos, 0.09)
    q[n // 2, 1, 5] = bad
    o2, lse2, _ = run(tree, index, q, pos, 0.09)
    assert bool(torch.isnan(o2[n // 2, 1]).all()) and not math.isfinite(float(lse2[n // 2, 1]))
    o2[n // 2, 1], lse2[n // 2, 1] = o[n // 2, 1], lse[n // 2, 1]
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("prefix", [3000, 4000])
def test_both_kernels_at_once_give_the_same_bits_every_time(kind, prefix):
    """Runs of many rows and of few in one call, a thousand times: stages are not overwritten under the reads of the one by the copies of the next."""
    rng = random.Random(150)
    ln = [prefix] + [rng.randint(1, 300) for _ in range(150)]
    tree = Tree([0, 151], [-1] + [0] * 150, [0] + [prefix] * 150, ln, 64, 2, kind, 150)
    node, pos = list(range(1, 151)), [n - 1 for n in ln[1:]]
    index, q = tree.index(node, pos, 4), queries(150, 8, 150)
    assert index.n_wide and index.n_narrow
    first, bad = None, torch.zeros((), dtype=torch.int64, device="cuda")
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(150, 8, device="cuda")
    ws = torch.empty(index.workspace_bytes, dtype=torch.uint8, device="cuda")
    for _ in range(1000):
        ws.fill_(255)
        H.harts_gen_attn(index, q, *tree.cache, p, o, lse, 0.09, workspace=ws, k_exp=tree.exp[0], v_exp=tree.exp[1])
        now = torch.cat([o.float().flatten(), lse.flatten()]).view(torch.int32)
        first = now if first is None else first
        bad += (now != first).any()
    assert int(bad) == 0


@pytest.mark.parametrize("branches", [2, 40])
@pytest.mark.parametrize("place", ["value", "value row", "key", "key row"])
def test_nan_in_an_8_bit_cache_comes_out_whichever_kernel_reads_it(branches, place):
    """A byte that is NaN, or a row whose power is, in the prompt that all branches see: read by few rows, and by many (the wide kernel)."""
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, "e4m3", 21)
    node, pos = list(range(1, branches + 1)), [69] * branches
    index, q = tree.index(node, pos, 4), queries(branches, 8, 21)
    assert (index.n_wide > 0) == (branches > 16)
    want = torch.zeros(branches, 8, 128, dtype=torch.bool, device="cuda")
    seen = tree.oracle(q, node, pos, 0.1)
    for token, byte, d in ((5, 0x7f, 3), (333, 0xff, 124), (699, 0x7f, 17)):
        s = tree.slots[0][token]
        if place == "value":
            tree.cache[1].view(torch.uint8)[s // 32, 0, s % 32, d] = byte
            want[:, :4, d] = True                     # the heads of key head 0
        elif place == "key":
            tree.cache[0].view(torch.uint8)[s // 32, 0, s % 32, d] = byte
        else:
            tree.exp[place == "value row"][s // 32, 0, s % 32] = 255
        if place != "value":
            want[:, :4] = True
    o, lse, status = run(tree, index, q, pos, 0.1)
    H.harts_la_check(status)
    assert torch.equal(torch.isnan(o), want)
    assert torch.equal(torch.isnan(lse), want.all(-1) & place.startswith("key"))
    rest = ~want
    d = (o.double() - seen[0])[rest]
    assert float(d.norm() / seen[0][rest].norm()) <= 2.0 ** -8


@pytest.mark.parametrize("node,q_pos", [([1, 1], [-1, -1]), ([0, 1], [299, 9])])
def test_a_call_s_first_kernel_waits_for_what_ran_before(node, q_pos):
    """What fills the index on the device may be the kernel right before the call: no kernel of the call is launched ahead of it, also where
    there is nothing to see and the merge is the only one.  (Of a captured call: edges of type 1 let a kernel start before the one ahead is complete.)"""
    tree = Tree([0, 2], [-1, 0], [0, 0 if q_pos[0] < 0 else 300], [300, q_pos[1] + 1], 32, 2, "bf16", 22)
    index, q = tree.index(node, q_pos, 4), queries(2, 8, 22)
    assert (index.n_narrow + index.n_wide > 0) == (q_pos[0] >= 0)
    o, lse, pos = torch.empty_like(q), torch.empty(2, 8, device="cuda"), torch.tensor(q_pos, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, index.workspace_bytes), dtype=torch.uint8, device="cuda")
    blob = index.dev.clone()

    def work():
        index.dev.copy_(blob + 0)                     # a kernel, then a copy
        index.dev.add_(0)                             # and a kernel right before the call
        H.harts_gen_attn(index, q, *tree.cache, pos, o, lse, 0.1, workspace=ws)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        work()
    driver, n = ctypes.CDLL("libcuda.so.1"), ctypes.c_size_t(0)
    raw = ctypes.c_void_p(graph.raw_cuda_graph())
    assert driver.cuGraphGetEdges_v2(raw, None, None, None, ctypes.byref(n)) == 0
    start, end, kind = (ctypes.c_void_p * n.value)(), (ctypes.c_void_p * n.value)(), (ctypes.c_uint8 * (8 * n.value))()
    assert driver.cuGraphGetEdges_v2(raw, start, end, kind, ctypes.byref(n)) == 0
    after = {a: (b, kind[8 * i + 2]) for i, (a, b) in enumerate(zip(start, end))}       # a chain; an edge's bytes are from, to, type
    at, ahead = next(a for a in start if a not in set(end)), []
    while at in after:
        at, k = after[at]
        ahead.append(k)
    assert len(ahead) == n.value
    # sum, copy, sum, the call's first kernel; a merge behind it is launched ahead of its end
    assert ahead == [0, 0, 0] + [1] * (q_pos[0] >= 0)
    graph.instantiate()
    o.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    compare(o, lse, *tree.oracle(q, node, q_pos, 0.1))


@pytest.mark.parametrize("branches", [2, 40])
def test_large_queries_and_large_keys_that_are_orthogonal(branches):
    """All scores are 0, whatever the factors: the values' mean."""
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, "e4m3", 24)
    tree.cache[0].view(torch.uint8)[..., 5] = 0
    tree.exp[0].fill_(247)
    tree.values[0] = tree.cache[0].float().double() * 2.0 ** 120
    node, pos = list(range(1, branches + 1)), [69] * branches
    index, q = tree.index(node, pos, 4), torch.zeros(branches, 8, 128, dtype=torch.bfloat16, device="cuda")
    q[..., 5] = 2.0 ** 40
    assert (index.n_wide > 0) == (branches > 16)
    o, lse, status = run(tree, index, q, pos, 0.1)
    H.harts_la_check(status)
    compare(o, lse, *tree.oracle(q, node, pos, 0.1))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches", [2, 40])
@pytest.mark.parametrize("q_scale", [2.0 ** 16, 2.0 ** 24, 2.0 ** 40, 2.0 ** 90])
def test_scores_of_any_size(kind, branches, q_scale):
    """Finite scores of 2^17 to 2^100, of which the largest takes all: its value, to its own rounding."""
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, kind, 25)
    index = check(tree, list(range(1, branches + 1)), [69] * branches, 4, 25, q_scale=q_scale)
    assert (index.n_wide > 0) == (branches > 16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches", [2, 40])
@pytest.mark.parametrize("q_scale,scale", [(2.0 ** 110, 2.0 ** -112), (2.0 ** 120, 2.0 ** -127 * 1.5), (2.0 ** -100, 2.0 ** 100), (1.0, 2.0 ** -140)])
def test_scales_of_any_size(kind, branches, q_scale, scale):
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, kind, 26)
    check(tree, list(range(1, branches + 1)), [69] * branches, 4, 26, q_scale=q_scale, scale=scale)


# Finite keys of any size against queries that make finite scores of them: both kernels, to the tolerances of every other size.
@pytest.mark.parametrize("branches", [2, 40])
@pytest.mark.parametrize("q_scale,lo,hi", [(2.0 ** -113, 228, 237), (2.0 ** -60, 120, 248), (2.0 ** -20, 244, 248), (2.0 ** 60, 1, 60), (2.0 ** 100, 1, 20)])
def test_keys_of_any_size_in_an_8_bit_cache(branches, q_scale, lo, hi):
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, "e4m3", 23)
    e = torch.randint(lo, hi, tree.exp[0].shape, device="cuda").to(torch.uint8)
    tree.exp[0].copy_(e)
    tree.values[0] = tree.cache[0].float().double() * (e.cpu().double() - 127).exp2().cuda()[..., None]
    index = check(tree, list(range(1, branches + 1)), [69] * branches, 4, 23, q_scale=q_scale)
    assert (index.n_wide > 0) == (branches > 16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches", [2, 40])
def test_subnormal_queries(kind, branches):
    """Rows whose largest is below 2^-126, and a scale that makes scores of some units of them."""
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, kind, 27)
    index = check(tree, list(range(1, branches + 1)), [69] * branches, 4, 27, q_scale=2.0 ** -129, scale=2.0 ** 126)
    assert (index.n_wide > 0) == (branches > 16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches,prefix", [(1, 500), (24, 2500)])
def test_an_index_of_mostly_growth(kind, branches, prefix):
    """Branches of a few tokens with room for thousands, at the first step, in between and at the last one."""
    rng = random.Random(branches)
    ln, grow = [prefix] + [rng.randint(0, 40) for _ in range(branches)], 3000
    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [prefix] * branches, ln, 64, 2, kind, 28, grow=grow)
    node, pos = list(range(1, branches + 1)), [n - 1 for n in ln[1:]]
    for step in (0, 1, 777, grow):
        check(tree, node, pos, 4, step, later=[p + step for p in pos])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("branches", [2, 40])
def test_tensors_of_16_bytes_alignment_only(kind, branches):
    """Cache, powers, queries, outputs, index and workspace 16 bytes past a multiple of 256: written, read and attended to as elsewhere."""
    def at_16(x):
        n = x.numel() * x.element_size()
        buf = torch.full((n + 512,), 255, dtype=torch.uint8, device="cuda")
        off = -buf.data_ptr() % 256 + 16
        return buf[off:off + n].view(x.dtype).view(x.shape).copy_(x)

    tree = Tree([0, branches + 1], [-1] + [0] * branches, [0] + [700] * branches, [700] + [70] * branches, 32, 2, kind, 29)
    node, pos = list(range(1, branches + 1)), [69] * branches
    index, q = tree.index(node, pos, 4), queries(branches, 8, 29)
    rows = [torch.randn(700, 2, 128, device="cuda").to(torch.bfloat16) for _ in range(2)]
    slot = tree.slots[0].int()
    got = []
    for place in (torch.clone, at_16):
        cache, exps = [place(x) for x in tree.cache], [None if x is None else place(x) for x in tree.exp]
        H.harts_gen_cache_write(*(place(x) for x in rows), place(slot), *cache, *exps)
        back = [place(x) for x in rows]
        H.harts_gen_cache_read(*cache, place(slot), *back, *exps)
        index.dev = place(index.dev)
        o, lse, ws = place(q), place(torch.empty(q.shape[:2], device="cuda")), place(torch.zeros(max(16, index.workspace_bytes), dtype=torch.uint8, device="cuda"))
        H.harts_gen_attn(index, place(q), *cache, place(torch.tensor(pos, dtype=torch.int32, device="cuda")), o, lse, 0.1, ws, *exps)
        got.append(back + [o, lse])
    assert all(torch.equal(a, b) for a, b in zip(*got))
