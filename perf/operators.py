"""Cases of the operators that sample rollout trees: the recurrence from and into kept states, the paged cache of keys and
values, and the attention of sampled tokens on the cached tree.

A case names one path (``op``):

  la      linear attention with a decay per head on packed sequences, start and end states in a pool (one token, drafted
          tokens, turns and whole prompts)
  write   keys and values of new tokens into the pages of an 8-bit cache
  read    rows of that cache back as bf16
  attn    attention of the sampled tokens on the cached tree, a shared prefix read once for all branches below it

``run`` computes a path by elementary torch operations where ``own`` is false, and by the framework's calls where it is true.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
D = 128          # width of a cached head


# ------------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # latency of one decoding step: a few branches, few heads
        {"name": "step of 5 branches x 4 heads", "op": "la", "dtype": "bf16", "n_seq": 5, "heads": 4, "d": 128, "lo": 1, "hi": 1,
         "lens": "even"},
        # a full decoding batch: the states are all that counts
        {"name": "step of 201 branches x 32 heads", "op": "la", "dtype": "bf16", "n_seq": 201, "heads": 32, "d": 128, "lo": 1,
         "hi": 1, "lens": "even"},
        # drafted tokens on top of the last sampled one, ragged
        {"name": "drafts fp32, 96 x 16 heads", "op": "la", "dtype": "fp32", "n_seq": 96, "heads": 16, "d": 64, "lo": 1, "hi": 7,
         "lens": "spread"},
        # prompts and tool answers of one admission: lengths from one token to thousands
        {"name": "prompts of 1 to 6,000 tokens", "op": "la", "dtype": "bf16", "n_seq": 23, "heads": 16, "d": 128, "lo": 1,
         "hi": 6000, "lens": "spread"},
        # one long prompt on few heads: the length of the chain is what counts
        {"name": "prompt of 31,017 tokens x 4", "op": "la", "dtype": "bf16", "n_seq": 1, "heads": 4, "d": 128, "lo": 31017,
         "hi": 31017, "lens": "even"},
        # the cache write of a decoding step, with rows of a padded batch that are skipped
        {"name": "write 61 sampled tokens", "op": "write", "tokens": 61, "kv_heads": 8, "page": 64, "pages": 512, "skip": 0.1},
        # the cache write of a prompt
        {"name": "write 16,385 prompt tokens", "op": "write", "tokens": 16385, "kv_heads": 8, "page": 64, "pages": 768, "skip": 0.0},
        # reading a branch back, for a fork that moves to other pages
        {"name": "read 24,000 cached tokens", "op": "read", "tokens": 24000, "kv_heads": 4, "page": 32, "pages": 1536, "skip": 0.0},
        # a few branches of a short prompt: latency
        {"name": "attn, 7 branches of 700 tokens", "op": "attn", "shape": "fan", "cache": "bf16", "trees": 1, "root": 700,
         "branches": 7, "own": 90, "q_heads": 8, "kv_heads": 2, "drafts": 1, "page": 16},
        # a group of answers to one long prompt
        {"name": "attn, 64 branches of 16,421", "op": "attn", "shape": "fan", "cache": "bf16", "trees": 1, "root": 16421,
         "branches": 64, "own": 1200, "q_heads": 32, "kv_heads": 4, "drafts": 1, "page": 64},
        # agentic trees in an 8-bit cache, four drafted tokens a branch
        {"name": "attn, agentic trees, drafts, 8 bit", "op": "attn", "shape": "tree", "cache": "e4m3", "trees": 6, "root": 9000,
         "branches": 20, "own": 900, "q_heads": 16, "kv_heads": 2, "drafts": 4, "page": 64},
        # one long sequence each: nothing is shared, the work is split over the length
        {"name": "attn, 3 of 90,000 alone, 8 bit", "op": "attn", "shape": "fan", "cache": "e4m3", "trees": 3, "root": 90000,
         "branches": 1, "own": 77, "q_heads": 32, "kv_heads": 8, "drafts": 1, "page": 128},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["la", "la", "la", "write", "read", "attn", "attn", "attn"])
    if op == "la":
        kind = rng.choice(["step", "drafts", "prompts", "long"])
        dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("fp32", 64)]) if kind in ("step", "drafts") else ("bf16", 128)
        case = {"op": "la", "dtype": dtype, "d": d, "heads": rng.choice([1, 2, 4, 8, 16, 32]), "lo": 1, "hi": 1, "lens": "even"}
        if kind == "step":
            case["n_seq"] = _log(rng, 1, 200)
        elif kind == "drafts":
            case.update(n_seq=_log(rng, 1, 100), hi=rng.randint(2, 9), lens="spread")
        elif kind == "prompts":
            case.update(n_seq=_log(rng, 2, 24), heads=rng.choice([4, 8, 16]), hi=_log(rng, 100, 6000), lens="spread")
        else:
            n = _log(rng, 2000, 31000)
            case.update(n_seq=1, heads=rng.choice([1, 2, 4]), lo=n, hi=n)
        return case
    if op in ("write", "read"):
        page = rng.choice([16, 32, 64, 128])
        tokens = _log(rng, 1, 16000)
        return {"op": op, "tokens": tokens, "kv_heads": rng.choice([1, 2, 4, 8]), "page": page,
                "pages": -(-tokens // page) * 2 + rng.randint(1, 40), "skip": rng.choice([0.0, 0.0, 0.1])}
    kv = rng.choice([1, 2, 4])
    shape = rng.choice(["fan", "tree", "branchy"])
    return {"op": "attn", "shape": shape, "cache": rng.choice(["bf16", "e4m3"]), "trees": rng.randint(1, 4), "root": _log(rng, 40, 16000),
            "branches": _log(rng, 1, 24), "own": _log(rng, 8, 1000), "q_heads": kv * rng.choice([1, 3, 4, 8]), "kv_heads": kv,
            "drafts": rng.choice([1, 1, 2, 4]), "page": rng.choice([16, 32, 64, 128])}


# ------------------------------------------------------------------------------------------------------------------ inputs
def _shape_rng(case):
    """Draws what the sizes of a case's tensors depend on: the same for every seed."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """Tokens of every sequence: all ``hi`` ("even"), or spread over the logarithm from ``lo`` to ``hi``, both ends among them."""
    rng = _shape_rng(case)
    n, lo, hi = case["n_seq"], case["lo"], case["hi"]
    if case["lens"] == "even":
        return [hi] * n
    return ([lo, hi] + [_log(rng, lo, hi) for _ in range(n)])[:n]


def _forest(case, rng):
    """Parents, fork offsets and lengths of the cached nodes, node count of every tree, and the branches being sampled.

    fan: answers of about ``own`` tokens to one prompt.  tree: turns that fork at their parent's end, up to four levels, the last
    node of every path being sampled.  branchy: the same with forks at arbitrary offsets, and inner nodes sampled too."""
    par, off, ln, ptr, live = [], [], [], [0], []
    for _ in range(case["trees"]):
        nodes = [(-1, 0, case["root"])]
        depth = [0]
        while len(nodes) <= case["branches"]:
            up = [0] if case["shape"] == "fan" else [i for i in range(len(nodes)) if depth[i] < 4]
            p = rng.choice(up)
            f = rng.randint(1, nodes[p][2]) if case["shape"] == "branchy" else nodes[p][2]
            nodes.append((p, f, max(1, int(case["own"] * rng.lognormvariate(0.0, 0.5)))))
            depth.append(depth[p] + 1)
        parents = {x[0] for x in nodes}
        base = ptr[-1]
        live += [base + i for i in range(len(nodes)) if i not in parents or (case["shape"] == "branchy" and i % 3 == 0)]
        par += [x[0] for x in nodes]
        off += [x[1] for x in nodes]
        ln += [x[2] for x in nodes]
        ptr.append(base + len(nodes))
    return par, off, ln, ptr, live


def _tree_tables(case, rng):
    """The cached forest, its pages, and the sampled tokens: the last ``drafts`` of every live node (as many as it has)."""
    par, off, ln, ptr, live = _forest(case, _shape_rng(case))
    page = case["page"]
    n_pages = [-(-x // page) for x in ln]
    order = list(range(sum(n_pages) + 3))
    rng.shuffle(order)
    page_ptr = [0]
    for x in n_pages:
        page_ptr.append(page_ptr[-1] + x)
    q_node = [v for v in live for _ in range(min(case["drafts"], ln[v]))]
    q_pos = [ln[v] - c + i for v in live for c in [min(case["drafts"], ln[v])] for i in range(c)]
    base = [ptr[t] for t in range(len(ptr) - 1) for _ in range(ptr[t + 1] - ptr[t])]
    sees = {}                                  # of every sampled token: node -> how many of its tokens it sees
    for r, (v, p) in enumerate(zip(q_node, q_pos)):
        sees[r, v] = p + 1
        while par[v] >= 0:
            sees[r, base[v] + par[v]] = off[v]
            v = base[v] + par[v]
    return {"par": par, "off": off, "len": ln, "ptr": ptr, "page_ptr": page_ptr, "page": order[:page_ptr[-1]], "pages": len(order),
            "q_node": q_node, "q_pos": q_pos, "sees": sees}


def prepare(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * (seed + 1))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def ints(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")

    if case["op"] == "la":
        lens = _lengths(case)
        n, H, d, dt = case["n_seq"], case["heads"], case["d"], DTYPES[case["dtype"]]
        rows = sum(lens)
        begin = [sum(lens[:i]) for i in range(n)]
        order = list(range(2 * n))             # start states in any order, end states in others (a branch keeps its parent's)
        rng.shuffle(order)
        starts = [-1 if n > 2 and i % 5 == 4 else order[i] for i in range(n)]
        s = {"case": case, "max_len": max(lens), "begin": ints(begin), "len": ints(lens), "in": ints(starts), "out": ints(order[n:]),
             "states": normal(2 * n, H, d, d) * 0.3}
        s["q"], s["k"] = ((normal(rows, H, d) / 8).to(dt) for _ in range(2))
        s["v"] = normal(rows, H, d).to(dt)
        s["g"] = torch.nn.functional.logsigmoid(normal(rows, H) + 3.0)
        if own:                                # the work memory that a sampling program keeps
            import paper_2608_28158_b200 as hp
            s["workspace"] = torch.empty(hp.harts_gen_la_workspace_bytes(n, s["max_len"], rows, H, d, d, dt), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] in ("write", "read"):
        n, hk, page, pages = case["tokens"], case["kv_heads"], case["page"], case["pages"]
        slots = torch.randperm(pages * page, generator=gen, device="cuda")[:n].to(torch.int32)
        if case["skip"]:
            slots[torch.rand(n, generator=gen, device="cuda") < case["skip"]] = -1
        s = {"case": case, "slot": slots}
        for x in ("k", "v"):
            s[x + "_cache"] = normal(pages, hk, page, D).mul_(60).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s[x + "_exp"] = torch.randint(117, 125, (pages, hk, page), generator=gen, device="cuda").to(torch.uint8)
            if case["op"] == "write":
                s[x] = (normal(n, hk, D) * torch.exp(normal(n, hk, 1))).to(torch.bfloat16)
        return s
    t = _tree_tables(case, rng)
    hq, hk, page = case["q_heads"], case["kv_heads"], case["page"]
    slot = [pg * page + i for v, m in enumerate(t["len"]) for p in [t["page_ptr"][v]]
            for j in range(-(-m // page)) for pg in [t["page"][p + j]] for i in range(min(page, m - j * page))]
    limit = torch.zeros(len(t["q_node"]), len(t["len"]), dtype=torch.int32)
    at = list(t["sees"])
    limit[[a for a, _ in at], [b for _, b in at]] = torch.tensor([t["sees"][x] for x in at], dtype=torch.int32)
    s = {"case": case, "tables": t, "scale": 1 / math.sqrt(D), "q_pos": ints(t["q_pos"]), "slot": ints(slot, torch.int64), "limit": limit.cuda(),
         "node_of": torch.repeat_interleave(torch.arange(len(t["len"])), torch.tensor(t["len"])).cuda(),
         "at": torch.cat([torch.arange(x, dtype=torch.int32) for x in t["len"]]).cuda(),
         "q": normal(len(t["q_node"]), hq, D).to(torch.bfloat16)}
    for x in ("k", "v"):
        if case["cache"] == "bf16":
            s[x + "_cache"], s[x + "_exp"] = normal(t["pages"], hk, page, D).to(torch.bfloat16), None
        else:
            s[x + "_cache"] = normal(t["pages"], hk, page, D).mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn)
            s[x + "_exp"] = torch.randint(119, 122, (t["pages"], hk, page), generator=gen, device="cuda").to(torch.uint8)
    if own:
        # the index that a sampling program keeps while its tree has the same branches, and the work memory
        import paper_2608_28158_b200 as hp
        s["index"] = hp.harts_gen_attn_index(t["ptr"], t["par"], t["off"], t["len"], t["page_ptr"], t["page"], page, t["q_node"],
                                             t["q_pos"], hq, hk).upload()
        s["workspace"] = torch.empty(s["index"].workspace_bytes, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------------- plain forms
def _plain_la(s):
    """Chunks of up to 64 tokens: products inside a chunk, and the state before every chunk as a weighted sum of what the chunks
    ahead of it add.  Running decays in 64 bits."""
    q, k, v, g, n, H, d = s["q"], s["k"], s["v"], s["g"], s["case"]["n_seq"], s["case"]["heads"], s["case"]["d"]
    T = min(64, s["max_len"])
    C = -(-s["max_len"] // T)
    t = torch.arange(C * T, device=q.device)
    inside = t < s["len"][:, None]
    row = torch.where(inside, s["begin"][:, None] + t, 0).long()

    def chunks(x):                       # [n, H, C, T, ...], zeros behind a sequence's end
        x = torch.where(inside.view(n, C * T, *[1] * (x.dim() - 1)), x[row], 0)
        return x.view(n, C, T, *x.shape[2:]).movedim(3, 1)

    Q, K, V = (chunks(x).float() for x in (q, k, v))
    b = chunks(g.double()).reshape(n, H, C * T).cumsum(-1).view(n, H, C, T)
    end = b[..., -1]
    seen = torch.ones(T, T, dtype=torch.bool, device=q.device).tril()
    decay = torch.exp((b[..., :, None] - b[..., None, :]).masked_fill(~seen, -math.inf)).float()
    inner = (Q @ K.transpose(-1, -2) * decay) @ V
    add = (K * torch.exp(end[..., None] - b).float()[..., None]).transpose(-1, -2) @ V
    start = torch.where((s["in"] >= 0).view(n, 1, 1, 1), s["states"][s["in"].clamp(min=0).long()], 0)
    # state behind chunk c: start state and every sum up to c, decayed from there to the end of c
    upto = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    weight = torch.exp((end[..., :, None] - end[..., None, :]).masked_fill(~upto, -math.inf)).float()
    behind = (weight @ add.view(n, H, C, d * d)).view(n, H, C, d, d) + torch.exp(end).float()[..., None, None] * start[:, :, None]
    before = torch.cat([start[:, :, None], behind[:, :, :-1]], 2)
    since = torch.exp(b - torch.cat([torch.zeros_like(end[..., :1]), end[..., :-1]], -1)[..., None]).float()
    out = (inner + since[..., None] * (Q @ before)).permute(0, 2, 3, 1, 4).reshape(n, C * T, H, d)
    o = torch.empty_like(v)
    o[row[inside]] = out[inside].to(v.dtype)
    s["states"][s["out"].long()] = behind[:, :, -1]
    return {"o": o, "states": s["states"]}


def _quantise(x):
    """Values in 8 bits, and the biased exponent of a row's scale: the smallest power of two 2^e with max |x| <= 448 2^e."""
    x = x.float()
    mantissa, exponent = torch.frexp(x.abs().amax(-1))               # mantissa in [1/2, 1)
    e = (exponent - 9 + (mantissa > 0.875)).clamp(min=-126)
    return (x * _power(127 - e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _power(biased):
    """2^(biased - 127), to the bit."""
    return (biased.int() << 23).view(torch.float32)


def _values(cache, exp):
    return cache.float() if exp is None else cache.float() * _power(exp)[..., None]


def _plain_write(s):
    kept = s["slot"] >= 0
    at, page = s["slot"][kept].long(), s["case"]["page"]
    for x in ("k", "v"):
        y, e = _quantise(s[x][kept])
        s[x + "_cache"].view(torch.uint8)[at // page, :, at % page] = y.view(torch.uint8)
        s[x + "_exp"][at // page, :, at % page] = e
    return {x: s[x] for x in ("k_cache", "v_cache", "k_exp", "v_exp")}


def _plain_read(s):
    at, page = s["slot"].clamp(min=0).long(), s["case"]["page"]
    kept = (s["slot"] >= 0)[:, None, None]
    return {x: torch.where(kept, _values(s[x + "_cache"].view(torch.uint8)[at // page, :, at % page].view(torch.float8_e4m3fn),
                                         s[x + "_exp"][at // page, :, at % page]), 0).to(torch.bfloat16) for x in ("k", "v")}


def _plain_attn(s):
    q, page, hk = s["q"], s["case"]["page"], s["case"]["kv_heads"]
    n, hq, G = q.shape[0], q.shape[1], q.shape[1] // hk
    k, v = (_values(s[x + "_cache"], s[x + "_exp"]).transpose(1, 2).reshape(-1, hk, D)[s["slot"]].transpose(0, 1) for x in ("k", "v"))
    hidden = s["at"][None] >= s["limit"][:, s["node_of"]]                                # [n, cached tokens]
    x = (q.float().view(n, hk, G, D).permute(1, 2, 0, 3).reshape(hk, G * n, D) @ k.transpose(-1, -2)).view(hk, G, n, -1) * s["scale"]
    x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = torch.exp(x - top)
    total = x.sum(-1)
    o = (x.view(hk, G * n, -1) @ v).view(hk, G, n, D) / total.clamp(min=1e-30)[..., None]
    return {"o": o.permute(2, 0, 1, 3).reshape(n, hq, D).to(q.dtype), "lse": (top[..., 0] + total.log()).permute(2, 0, 1).reshape(n, hq)}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"la": _plain_la, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[op](s)
    import paper_2608_28158_b200 as hp
    if op == "la":
        o = torch.empty_like(s["v"])
        hp.harts_gen_la(s["q"], s["k"], s["v"], s["g"], o, s["states"], s["begin"], s["len"], s["in"], s["out"], s["max_len"],
                        workspace=s["workspace"])
        return {"o": o, "states": s["states"]}
    if op == "write":
        hp.harts_gen_cache_write(s["k"], s["v"], s["slot"], s["k_cache"], s["v_cache"], s["k_exp"], s["v_exp"])
        return {x: s[x] for x in ("k_cache", "v_cache", "k_exp", "v_exp")}
    if op == "read":
        n, hk = s["slot"].shape[0], s["case"]["kv_heads"]
        k, v = (torch.empty(n, hk, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        hp.harts_gen_cache_read(s["k_cache"], s["v_cache"], s["slot"], k, v, s["k_exp"], s["v_exp"])
        return {"k": k, "v": v}
    o, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    hp.harts_gen_attn(s["index"], s["q"], s["k_cache"], s["v_cache"], s["q_pos"], o, lse, s["scale"], s["workspace"], k_exp=s["k_exp"],
                      v_exp=s["v_exp"])
    return {"o": o, "lse": lse}


# -------------------------------------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == "la":
        rows, H, d, e = sum(_lengths(case)), case["heads"], case["d"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": rows * H * (4 * d * e + 4) + 2 * case["n_seq"] * H * d * d * 4, "flops": rows * H * 4 * d * d}
    if case["op"] in ("write", "read"):
        return {"bytes": case["tokens"] * (case["kv_heads"] * 2 * (2 * D + D + 1) * (1 - case["skip"]) + 4), "flops": 0}
    t = _tree_tables(case, random.Random(0))
    seen = {}
    for (_, v), m in t["sees"].items():
        seen[v] = max(seen.get(v, 0), m)
    per = 2 * (2 * D if case["cache"] == "bf16" else D + 1)
    n = len(t["q_node"])
    return {"bytes": sum(seen.values()) * case["kv_heads"] * per + n * case["q_heads"] * (4 * D + 4),
            "flops": 4 * D * case["q_heads"] * sum(t["sees"].values())}


# ------------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "la":
        # token by token, all sequences at once
        n, H, d = case["n_seq"], case["heads"], case["d"]
        q, k, v, g = (s[x].double() for x in ("q", "k", "v", "g"))
        S = s["states"][s["in"].clamp(min=0).long()].double()
        S[s["in"] < 0] = 0
        o = torch.zeros_like(v)
        begin, lens = s["begin"].tolist(), s["len"].tolist()
        by_len = sorted(range(n), key=lambda i: -lens[i])
        S = S[by_len]
        for t in range(max(lens)):
            m = sum(x > t for x in lens)
            r = torch.tensor([begin[i] + t for i in by_len[:m]], device="cuda")
            S[:m] = S[:m] * g[r].exp()[..., None, None] + k[r][..., :, None] * v[r][..., None, :]
            o[r] = (q[r][..., None, :] @ S[:m])[..., 0, :]
        states = s["states"].double()
        states[s["out"].long()[torch.tensor(by_len, device="cuda")]] = S
        return {"o": o, "states": states}
    page = case.get("page")
    if case["op"] == "write":
        out = {x + y: s[x + y].double() if y == "_cache" else s[x + y].clone() for x in ("k", "v") for y in ("_cache", "_exp")}
        kept = s["slot"] >= 0
        at = s["slot"][kept].long()
        power = torch.tensor([2.0 ** i for i in range(-300, 300)], dtype=torch.float64, device="cuda")
        tops = 448 * power[300 - 126:300 + 128]                                              # largest value of every scale
        for x in ("k", "v"):
            y = s[x][kept].double()
            e = torch.searchsorted(tops, y.abs().amax(-1).contiguous())
            y = y * power[300 + 126 - e][..., None]
            _, p = torch.frexp(y)
            step = power[300 + (p - 1).clamp(min=-6).long() - 3]                             # of the 3-bit fraction, subnormals too
            out[x + "_cache"][at // page, :, at % page] = torch.round(y / step) * step
            out[x + "_exp"][at // page, :, at % page] = (e + 1).to(torch.uint8)
        return out
    scale = {x: 1.0 if s[x + "_exp"] is None else (s[x + "_exp"].cpu().double() - 127).exp2()[..., None].cuda() for x in ("k", "v")}
    if case["op"] == "read":
        out = {}
        for x in ("k", "v"):
            y = s[x + "_cache"].double() * scale[x]
            y = y.transpose(1, 2).reshape(-1, case["kv_heads"], D)[s["slot"].clamp(min=0).long()]
            y[s["slot"] < 0] = 0
            out[x] = y
        return out
    # one sampled token at a time, over the tokens on its path
    t, hq, hk = s["tables"], case["q_heads"], case["kv_heads"]
    first = [0]
    for m in t["len"]:
        first.append(first[-1] + m)
    paths = {}
    for (r, v), m in t["sees"].items():
        paths.setdefault(r, []).append(s["slot"][first[v]:first[v] + m])
    o = torch.zeros(len(t["q_node"]), hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((len(t["q_node"]), hq), -math.inf, dtype=torch.float64, device="cuda")
    K, V = ((s[x + "_cache"].double() * scale[x]).transpose(1, 2).reshape(-1, hk, D) for x in ("k", "v"))
    for r, parts in paths.items():
        at = torch.cat(parts)
        x = torch.einsum("hgd,thd->hgt", s["q"][r].double().view(hk, hq // hk, D), K[at]) * s["scale"]
        lse[r] = torch.logsumexp(x, -1).reshape(hq)
        o[r] = torch.einsum("hgt,thd->hgd", torch.softmax(x, -1), V[at]).reshape(hq, D)
    return {"o": o, "lse": lse}
