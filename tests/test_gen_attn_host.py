"""harts_gen_attn_index on the host: every token that a query sees is in exactly one of its units, and what is refused."""
import random

import numpy as np
import pytest

import paper_2608_28158_b200 as H

NARROW, WIDE = 16, 128


def arrays(ix):
    b = ix.host
    at = b[10:16]
    units = [b[at[i]:at[i] + 8 * b[4 + i]].reshape(-1, 8) for i in range(2)]
    entries = b[at[2]:at[3]].reshape(-1, 4)
    lists = b[b[18]:b[18] + b[17] + 1] if b[17] else np.zeros(1, np.int32)
    assert lists[0] == 0 and lists[-1] == len(units[0]) and (np.diff(lists) > 0).all()          # every narrow unit is in one list
    return units, entries, b[at[3]:], b[at[4]:at[4] + ix.n_q + 1], b[at[5]:]


def forest(rng, shape):
    par, off, ln, ptr = [], [], [], [0]
    for _ in range(rng.randint(1, 3)):
        n = rng.choice([1, 2, 5, 12, 40])
        nodes = [(-1, 0, rng.choice([0, 1, 63, 64, 65, 700, 5000]))]
        for i in range(1, n):
            p = rng.randrange(i) if shape != "fan" else 0
            m = nodes[p][2]
            f = m if shape == "turns" else rng.randint(0, m)
            nodes.append((p, f, rng.choice([0, 1, 7, 64, 100, 130, 900])))
        par += [x[0] for x in nodes]
        off += [x[1] for x in nodes]
        ln += [x[2] for x in nodes]
        ptr.append(len(par))
    return ptr, par, off, ln


def sees(ptr, par, off, v, p):
    """node -> tokens of it that a query at position p of node v sees."""
    base = max(x for x in ptr if x <= v)
    out = {v: p + 1}
    while par[v] >= 0:
        out[base + par[v]] = off[v]
        v = base + par[v]
    return {v: m for v, m in out.items() if m > 0}


@pytest.mark.parametrize("seed", range(40))
def test_every_visible_token_is_in_one_unit(seed):
    rng = random.Random(seed)
    ptr, par, off, ln = forest(rng, rng.choice(["fan", "turns", "any"]))
    page, grow = rng.choice([16, 32, 64, 128]), rng.choice([0, 0, 5, 300])
    G, hkv = rng.choice([1, 3, 4, 8, 17]), rng.choice([1, 2])
    q_node, q_pos = [], []
    for v in range(len(ln)):
        if rng.random() < 0.6:
            for i in range(rng.choice([1, 1, 2, 5, 40])):
                q_node.append(v)
                q_pos.append(rng.randint(-1, ln[v] - 1))
    q_node += [-1]
    q_pos += [0]
    counts = [-(-(n + grow) // page) for n in ln]
    page_ptr = np.concatenate([[0], np.cumsum(counts)])
    pages = rng.sample(range(10 * sum(counts) + 5), sum(counts))
    ix = H.harts_gen_attn_index(ptr, par, off, ln, page_ptr, pages, page, q_node, q_pos, G * hkv, hkv, grow)
    units, entries, listed, part_ptr, part = arrays(ix)
    assert list(listed[:len(pages)]) == pages
    now = [p + rng.randint(0, ln[v] - 1 + grow - p) if v >= 0 else 0 for v, p in zip(q_node, q_pos)]      # after some growth
    got = {}                               # (query, head of the group) -> [(node, from, to, part)]
    for wide in range(2):
        for entry, flat0, n, k0, k1, page0, part0, _ in units[wide]:
            assert 1 <= n <= (WIDE if wide else NARROW) and 0 <= k0 < k1
            node = int(np.searchsorted(page_ptr, page0, side="right")) - 1
            while page_ptr[node] != page0 or counts[node] == 0:
                node -= 1
            assert k1 <= counts[node] * page
            for i in range(flat0, flat0 + n):
                row, limit, least, most = entries[entry + i // G]
                alone, most = most < 0, (-most - 1 if most < 0 else most)
                if limit < 0:
                    assert least <= q_pos[row] + 1 and now[row] + 1 <= most
                    limit = now[row] + 1
                elif wide:
                    assert limit >= k1                 # no row of a wide unit has a limit inside
                got.setdefault((row, i % G), []).append((node, k0, min(k1, limit), part0 + i, alone))
    for r, v in enumerate(q_node):
        want = sees(ptr, par, off, v, now[r]) if v >= 0 else {}
        ids = list(part[part_ptr[r]:part_ptr[r + 1]])
        for g in range(G):
            runs = got.get((r, g), [])
            if len(runs) == 1:
                assert ids == [-1] and runs[0][4]
            else:
                assert sorted(i + g for i in ids) == sorted(x[3] for x in runs) and not any(x[4] for x in runs)
            seen = {}
            for node, a, b, p, _ in runs:
                if b > a:
                    seen.setdefault(node, []).append((a, b))
                assert p < ix.n_parts
            for node, spans in seen.items():
                spans.sort()
                assert spans[0][0] == 0 and all(x[1] == y[0] for x, y in zip(spans, spans[1:])), (r, node, spans)
            assert {node: spans[-1][1] for node, spans in seen.items()} == want, (r, g)
    assert len({x[3] for runs in got.values() for x in runs}) == sum(map(len, got.values()))      # no part is written twice


def test_shared_prefix_is_read_once():
    """64 branches of one prompt, 8 query heads to a key head: the prompt's tokens are in units of 128 rows, four times over (512 rows)."""
    n = 64
    ptr, par, off, ln = [0, n + 1], [-1] + [0] * n, [0] + [4096] * n, [4096] + [100] * n
    pages = [64] + [2] * n
    page_ptr = np.concatenate([[0], np.cumsum(pages)])
    ix = H.harts_gen_attn_index(ptr, par, off, ln, page_ptr, np.arange(sum(pages)), 64, np.arange(1, n + 1), [99] * n, 8, 1)
    units, *_ = arrays(ix)
    read = sum(int(u[4] - u[3]) for k in range(2) for u in units[k] if u[5] == 0)
    assert read == 4096 * 512 // (WIDE if ix.n_wide else NARROW)


GOOD = dict(tree_node_ptr=[0, 2], node_parent=[-1, 0], node_fork_off=[0, 10], node_len=[10, 5], node_page_ptr=[0, 1, 2], node_page=[3, 4], page=16,
            q_node=[1], q_pos=[4], Hq=4, Hkv=2)


def test_the_good_one_is_taken():
    H.harts_gen_attn_index(**GOOD)
    for grow in (11, 12, 2 ** 31 - 1):              # as far as the pages go
        entries = arrays(H.harts_gen_attn_index(**GOOD, grow=grow))[1]
        assert {abs(x[3]) for x in entries if x[1] < 0} == {16}
    H.harts_gen_attn_index([0], [], [], [], [0], [], 16, [], [], 4, 2)
    H.harts_gen_attn_index([0], [], [], [], [0], [], 16, [-1], [0], 4, 2)


@pytest.mark.parametrize("bad", [
    dict(page=17), dict(page=8), dict(page=256), dict(Hq=3), dict(Hkv=0), dict(Hq=0), dict(grow=-1), dict(q_pos=[5]), dict(q_pos=[-2]),
    dict(q_node=[2]), dict(node_len=[10, -1]), dict(node_len=[17, 5]), dict(node_fork_off=[0, 11]), dict(node_fork_off=[0, -1]),
    dict(node_fork_off=[1, 10]), dict(node_parent=[0, 0]), dict(node_parent=[-1, 1]), dict(node_parent=[-1, -1]), dict(node_page=[3, -1]),
    dict(node_page_ptr=[0, 2, 2]), dict(node_page_ptr=[0, 3, 2]), dict(node_page_ptr=[1, 1, 2]), dict(tree_node_ptr=[0, 0, 2]), dict(q_pos=[4, 4]),
    dict(node_page=[3])])
def test_what_is_refused(bad):
    with pytest.raises(H.HartsError) as e:
        H.harts_gen_attn_index(**{**GOOD, **bad})
    assert e.value.code == -1


@pytest.mark.parametrize("bad", [dict(tree_node_ptr=[0, 1 << 28, 2]), dict(tree_node_ptr=[0, -5, 2]), dict(tree_node_ptr=[0, 0, 2]),
                                 dict(node_page_ptr=[0, 1 << 28, 2]), dict(node_page_ptr=[0, -1, 2]), dict(node_page_ptr=[0, 3, 2])])
def test_pointers_that_do_not_ascend_are_refused_before_they_are_followed(bad):
    with pytest.raises(H.HartsError) as e:
        H.harts_gen_attn_index(**{**GOOD, **bad})
    assert e.value.code == -1


W = 1 << 32


@pytest.mark.parametrize("bad", [dict(q_pos=[4 + W]), dict(q_node=[1 - W]), dict(node_len=[10, 5 + W]), dict(node_page=[3, 4 + W]), dict(tree_node_ptr=[0, 2 + W]),
                                 dict(node_parent=[-1, W]), dict(node_fork_off=[0, 10 + W]), dict(node_page_ptr=[0, 1, 2 - W]), dict(page=16 + W), dict(Hq=4 + W),
                                 dict(Hkv=2 - W), dict(grow=W), dict(q_pos=np.array([4 + W], np.uint64)), dict(q_pos=np.array([2 ** 31], np.uint32)),
                                 dict(q_pos=[4.5]), dict(q_pos=[[4]]), dict(q_pos=[float("nan")]), dict(node_page=[3.0, 1e20])])
def test_numbers_that_32_bits_do_not_hold_are_refused(bad):
    """They were cut off before: 2^32 + 4 was position 4."""
    with pytest.raises(H.HartsError) as e:
        H.harts_gen_attn_index(**{**GOOD, **bad})
    assert e.value.code == -1


@pytest.mark.parametrize("kind", [np.int8, np.int16, np.int32, np.int64, np.uint32, np.uint64, np.float32, np.float64])
def test_whole_numbers_of_any_type_are_taken(kind):
    want = H.harts_gen_attn_index(**GOOD).host
    arrays = {k: np.asarray(v, kind) for k, v in GOOD.items() if isinstance(v, list) and min(v) >= 0}
    assert np.array_equal(H.harts_gen_attn_index(**{**GOOD, **arrays}).host, want)
    strided = {k: np.repeat(v, 2)[::2] for k, v in arrays.items()}
    assert np.array_equal(H.harts_gen_attn_index(**{**GOOD, **strided}).host, want)
