"""The operators of a step that checks drafted tokens over the paged key/value cache, as cases that can be timed.

A server drafts a tree of tokens for every request, feeds the trees as one step, and keeps of each the path that the model's
own distributions accept.  Node 0 of a request's tree is the token that the step before gave; the tokens of a step are packed
one request after another, as everywhere with the paged cache.

A case is a dict of plain values.  ``prepare`` makes what a program holds before the call, ``run`` is one pass: with
``own`` false in plain elementary torch operations, with ``own`` true through the public entry points of
``paper_2307_15517_amd.mx``.  ``work`` is what a pass cannot do without, ``exact`` the result from the definition in 64 bits.

The kinds:

* ``tree``    parents of the nodes -> bit masks of every node's ancestors (itself among them), positions in the sequence.
* ``attend``  attention of the trees' nodes over the pages: a node sees the cached tokens and its ancestors; grouped heads.
* ``verify``  walk down the trees by given random numbers: a child is accepted by its probability under the model, with or
              without the distribution that it was drawn from; at the walk's end a token is drawn from what is left.
* ``move``    keys and values of the accepted nodes to the places that follow the cached tokens.  An MXInt cache is returned
              as the values it stands for, which the framework's own dequantizer gives.

Cache: [pages][heads][tokens of a page][dim], keys and values apart, MXInt exponents [pages][heads][page][dim/block].
"""
import math
import random

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # four requests with a chain of four drafted tokens each: the smallest step of a server
        dict(name="tree_chains_4", kind="tree", requests=4, nodes=5, least=5, branch=1, words=1),
        # two hundred requests, wide trees of up to 180 nodes: three words of mask
        dict(name="tree_wide_200", kind="tree", requests=200, nodes=180, least=1, branch=6, words=3),
        # four drafted tokens after 173 cached ones, heads of OPT-125M: latency counts
        dict(name="attend_chain_5", kind="attend", requests=1, nodes=5, least=5, branch=1, words=1, min_ctx=173, max_ctx=173, heads=12,
             group=1, dim=64, page=16, cache="mx32", type="f32"),
        # continuous batching: 16 requests of very different lengths, trees of up to 25 nodes, grouped heads, MXInt cache
        dict(name="attend_trees_16", kind="attend", requests=16, nodes=25, least=1, branch=3, words=1, min_ctx=1, max_ctx=4001, heads=8,
             group=4, dim=128, page=32, cache="mx32", type="bf16"),
        # one long sequence, a tree of 61 nodes, bfloat16 cache
        dict(name="attend_long_30011", kind="attend", requests=1, nodes=61, least=61, branch=4, words=1, min_ctx=30011, max_ctx=30011,
             heads=8, group=5, dim=128, page=64, cache="bf16", type="bf16"),
        # 24 requests of up to 8191 tokens with trees of 40 to 63 nodes, eight heads a group: the largest product
        dict(name="attend_trees_24", kind="attend", requests=24, nodes=63, least=40, branch=4, words=1, min_ctx=501, max_ctx=8191, heads=8,
             group=8, dim=128, page=64, cache="mx32", type="bf16"),
        # one request, four drafted tokens without their distributions, vocabulary of LLaMA-7B: latency counts
        dict(name="verify_chain_1", kind="verify", requests=1, nodes=5, least=5, branch=1, vocab=32000, type="f32", draft=False, greedy=0.0),
        # 24 requests, chains of up to five drafted tokens with their distributions, some requests greedy, vocabulary of OPT-125M
        dict(name="verify_chains_24", kind="verify", requests=24, nodes=6, least=1, branch=1, vocab=50272, type="f32", draft=True,
             greedy=0.2),
        # 16 trees of up to 61 nodes of the most probable tokens, a large vocabulary: the most logits
        dict(name="verify_trees_16", kind="verify", requests=16, nodes=61, least=40, branch=4, vocab=128000, type="f32", draft=False,
             greedy=0.0),
        # six trees of nodes drawn from the draft's distributions, bfloat16 logits, rows of odd length
        dict(name="verify_drawn_6", kind="verify", requests=6, nodes=25, least=10, branch=3, vocab=100003, type="bf16", draft=True, greedy=0.0),
        # one request keeps four of eight nodes, heads of OPT-125M, bfloat16 cache
        dict(name="move_1", kind="move", requests=1, nodes=8, max_ctx=200, most=4, heads=12, dim=64, page=16, cache="bf16"),
        # 96 requests early in their answers keep up to eight of 61 nodes, MXInt cache
        dict(name="move_96", kind="move", requests=96, nodes=61, max_ctx=80, most=8, heads=8, dim=128, page=32, cache="mx32"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    kind = rng.choice(["tree", "attend", "attend", "attend", "verify", "verify", "verify", "move"])
    if kind == "tree":
        nodes = _log(rng, 1, 250)
        return dict(kind=kind, requests=_log(rng, 1, 400 if nodes < 65 else 120), nodes=nodes, least=rng.randint(1, nodes),
                    branch=rng.choice([1, 2, 3, 6, 30]), words=-(-nodes // 64))
    dim = rng.choice([64, 80, 96, 112, 128, 128, 128])
    cache = rng.choice(["bf16", "mx16", "mx32"] if dim % 32 == 0 else ["bf16", "mx16"])
    if kind == "move":
        nodes = _log(rng, 1, 64)
        return dict(kind=kind, requests=_log(rng, 1, 90), nodes=nodes, max_ctx=_log(rng, 1, 90), most=rng.randint(1, min(nodes, 9)),
                    heads=rng.choice([1, 4, 8]), dim=dim, page=rng.choice([16, 32]), cache=cache)
    while True:
        nodes = rng.choice([1, _log(rng, 2, 8), _log(rng, 2, 64), _log(rng, 2, 64), _log(rng, 65, 150)])
        c = dict(kind=kind, requests=_log(rng, 1, 30), nodes=nodes, least=rng.randint(1, nodes), branch=rng.choice([1, 2, 3, 4, 8]))
        if kind == "verify":
            c.update(vocab=_log(rng, 500, 130000), type=rng.choice(["f32", "f32", "bf16"]), draft=rng.random() < 0.5,
                     greedy=rng.choice([0.0, 0.0, 0.5, 1.0]))
            if c["requests"] * nodes * c["vocab"] * (2 if c["draft"] else 1) <= 1.2e8:
                return c
            continue
        c.update(words=-(-nodes // 64), max_ctx=_log(rng, 1, 30000))
        c.update(min_ctx=rng.choice([0, c["max_ctx"] // 2, c["max_ctx"]]), heads=rng.choice([1, 2, 4, 8, 8, 12, 32]),
                 group=rng.choice([1, 1, 2, 3, 4, 5, 8]), dim=dim, page=rng.choice([16, 32, 64, 128]), cache=cache,
                 type=rng.choice(["f32", "bf16", "bf16"]))
        # no more than the largest listed ones, also where the plain form pads every request to the longest
        w, hq, long = work(c), c["heads"] * c["group"], c["max_ctx"] + nodes
        if (w["bytes"] <= 3e8 and w["flops"] <= 1e11 and c["requests"] * long * c["heads"] * dim <= 1.2e8
                and c["requests"] * hq * nodes * long <= 6e8):
            return c


# ---- sizes that follow from a case ----------------------------------------------------------------------
def _block(case):
    return {"bf16": 0, "mx16": 16, "mx32": 32}[case["cache"]]


def _sizes(case):
    """Nodes of every request's tree; the first has the most."""
    r = random.Random("%(requests)d %(nodes)d %(least)d" % case)
    return [case["nodes"]] + [r.randint(case["least"], case["nodes"]) for _ in range(case["requests"] - 1)]


def _contexts(case):
    """Tokens that every request has cached; the first has the most."""
    r = random.Random("%(requests)d %(max_ctx)d %(dim)d" % case)
    return [case["max_ctx"]] + [r.randint(case.get("min_ctx", 0), case["max_ctx"]) for _ in range(case["requests"] - 1)]


def _pages(tokens, page):
    return -(-tokens // page)


# ---- inputs ---------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(g, shape):
    """Rows of a projection: N(0, 1), 2 % of the channels (at least one) eight times as large."""
    x = torch.randn(shape, generator=g, device=DEV)
    x[..., torch.randperm(shape[-1], generator=g, device=DEV)[:max(1, round(0.02 * shape[-1]))]] *= 8.0
    return x


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _order(g, n):
    return torch.randperm(n, generator=g, device=DEV).to(torch.int32)


def _starts(sizes):
    v = [0]
    for n in sizes:
        v.append(v[-1] + n)
    return v


def _trees(case, seed):
    """Parent and rank among its siblings of every node, level by level: a node has up to ``branch`` children."""
    r, branch = random.Random("%d %d" % (seed, case["nodes"])), case["branch"]
    parents, ranks = [], []
    for n in _sizes(case):
        parent, rank, open_, at = [-1], [0], [0], 1
        while at < n:
            level, node = [], 0
            while node < len(open_) and at < n:
                for k in range(branch if node == 0 else r.randint(0, branch)):
                    if at == n:
                        break
                    parent.append(open_[node])
                    rank.append(k)
                    level.append(at)
                    at += 1
                node += 1
            open_ = level
        parents += parent
        ranks += rank
    return parents, ranks


def _masks(parents, starts, words):
    """Masks of ancestors, 64 bits a word, and depths."""
    masks, depths = [], []
    for lo, hi in zip(starts, starts[1:]):
        m, d = [], []
        for i, p in enumerate(parents[lo:hi]):
            m.append((m[p] if p >= 0 else 0) | 1 << i)
            d.append(d[p] + 1 if p >= 0 else 0)
        masks += m
        depths += d
    signed = [[(x >> 64 * w & (1 << 64) - 1) - ((x >> 64 * w + 63 & 1) << 64) for w in range(words)] for x in masks]
    return torch.tensor(signed, dtype=torch.int64, device=DEV), depths


def _pool(g, case, pages):
    """Keys (or values) of a whole cache and their exponents; every place holds something, as in a cache long in use."""
    x = _rows(g, (pages, case["heads"], case["page"], case["dim"]))
    block = _block(case)
    if not block:
        return x.to(torch.bfloat16), torch.zeros(16, dtype=torch.uint8, device=DEV)
    y = x.unflatten(-1, (-1, block))
    top = y.abs().amax(-1)
    e = (torch.frexp(top)[1] - 1).clamp(-127, 128)
    m = torch.round(torch.ldexp(y, (6 - e)[..., None])).clamp(-127, 127)
    return m.to(torch.int8).flatten(-2), (e + 127).to(torch.uint8)


def _table(g, need):
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device=DEV)
    held = torch.arange(max(need), device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None]
    table[held] = _order(g, sum(need) + 1)[:sum(need)]
    return table


def prepare(case, seed):
    g = _gen(seed)
    return dict({"tree": _prepare_tree, "attend": _prepare_attend, "verify": _prepare_verify, "move": _prepare_move}[case["kind"]](case, g, seed),
                case=dict(case))


def _prepare_tree(case, g, seed):
    parents, _ = _trees(case, seed)
    ctx = random.Random(seed)
    starts = _starts(_sizes(case))
    return dict(parents=_ints(parents), q_start=_ints(starts), ctx=_ints([ctx.randint(0, 5000) for _ in range(case["requests"])]),
                tokens=starts[-1], masks=torch.empty((starts[-1], case["words"]), dtype=torch.int64, device=DEV),
                positions=torch.empty(starts[-1], dtype=torch.int32, device=DEV))


def _prepare_attend(case, g, seed):
    sizes, ctx = _sizes(case), _contexts(case)
    starts, length = _starts(sizes), [c + n for c, n in zip(ctx, sizes)]
    need = [_pages(n, case["page"]) for n in length]
    kp, ke = _pool(g, case, sum(need) + 1)
    vp, ve = _pool(g, case, sum(need) + 1)
    q = _rows(g, (starts[-1], case["heads"] * case["group"] * case["dim"])).to(TYPES[case["type"]])
    return dict(q=q, out=torch.empty_like(q), table=_table(g, need), q_start=_ints(starts), kv_len=_ints(length), kp=kp, ke=ke, vp=vp, ve=ve,
                masks=_masks(_trees(case, seed)[0], starts, case["words"])[0], tokens=starts[-1], pages=sum(need) + 1, max_new=max(sizes),
                max_len=max(length), scale=case["dim"] ** -0.5)


def _prepare_verify(case, g, seed):
    sizes, V, B = _sizes(case), case["vocab"], case["requests"]
    starts, (parents, ranks) = _starts(sizes), _trees(case, seed)
    T, type_ = starts[-1], TYPES[case["type"]]
    # logits as a language model's: a few tokens of most rows hold most of the probability; the draft's are near them
    logits = (4.0 * torch.randn((T, V), generator=g, device=DEV)).to(type_)
    draft = (logits.float() + torch.randn((T, V), generator=g, device=DEV)).to(type_)
    r = random.Random(seed + 1)
    temperature = torch.tensor([0.0 if r.random() < case["greedy"] else r.choice([0.6, 0.8, 1.0]) for _ in range(B)], device=DEV)
    owner = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(sizes, device=DEV))
    at = torch.tensor(parents, device=DEV).clamp(min=0) + torch.tensor(starts, device=DEV)[owner]     # the row of a node's parent
    if case["draft"]:              # each child drawn from its parent's distribution
        heat = torch.where(temperature > 0, temperature, 1.0)[owner, None]
        ids = torch.cat([(draft[at[lo:lo + 64]].float() / heat[lo:lo + 64]
                          - torch.empty((min(64, T - lo), V), device=DEV).exponential_(generator=g).log()).argmax(-1)
                         for lo in range(0, T, 64)])
    else:                          # the children of a node are its draft's most probable tokens
        best = draft.float().topk(min(V, max(ranks) + 1), -1).indices
        ids = best[at, torch.tensor(ranks, device=DEV)]
    width = min(case["nodes"], 16)
    return dict(logits=logits, draft=draft if case["draft"] else None, ids=ids.to(torch.int32), parents=_ints(parents),
                q_start=_ints(starts), temperature=temperature, uniform=torch.rand(T, generator=g, device=DEV),
                noise=torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30), tokens=T, width=width, most=max(sizes),
                path=torch.empty((B, width), dtype=torch.int32, device=DEV), kept=torch.empty(B, dtype=torch.int32, device=DEV),
                next=torch.empty(B, dtype=torch.int32, device=DEV))


def _prepare_move(case, g, seed):
    r, B, most, nodes = random.Random(seed), case["requests"], case["most"], case["nodes"]
    ctx = _contexts(case)
    need = [_pages(c + nodes, case["page"]) for c in ctx]
    path, kept = [], []
    for b in range(B):
        n = most if b == 0 else r.randint(1, most)
        path.append(([0] + sorted(r.sample(range(1, nodes), n - 1)) + [-1] * most)[:most])
        kept.append(n)
    kp, ke = _pool(g, case, sum(need) + 1)
    vp, ve = _pool(g, case, sum(need) + 1)
    shape = ((sum(need) + 1) * case["heads"] * case["page"], case["dim"]) if _block(case) else (1, 1)
    return dict(ctx=_ints(ctx), table=_table(g, need), path=_ints(path), kept=_ints(kept), kp=kp, ke=ke, vp=vp, ve=ve,
                pages=sum(need) + 1, ky=torch.empty(shape, device=DEV), vy=torch.empty(shape, device=DEV))


# ---- one pass -------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if kind == "tree":
        return (_own_tree if own else _plain_tree)(state)
    if kind == "attend":
        return (_own_attend if own else _plain_attend)(state)
    if kind == "verify":
        return (_own_verify if own else _plain_verify)(state)
    return (_own_move if own else _plain_move)(state)


def _own_cache(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    block = _block(c)
    return mx.cache_format(s["pages"], c["page"], c["heads"], c["dim"], mx.fmt(block, 8) if block else None)


def _own_tree(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    mx.mx_tree_plan(s["parents"], s["q_start"], s["ctx"], c["requests"], s["tokens"], c["words"], s["masks"], s["positions"])
    return s["masks"], s["positions"]


def _own_attend(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    hq = c["heads"] * c["group"]
    if "cache" not in s:                                     # the description and the workspace, which a program keeps
        s["cache"] = _own_cache(s)
        s["workspace"] = mx.cache_tree_workspace(s["cache"], s["tokens"], c["requests"], hq, s["max_new"], s["max_len"], DEV)
    mx.mx_cache_tree_attention(s["q"], mx.MX_F32 if c["type"] == "f32" else mx.MX_BF16, s["tokens"], hq * c["dim"], hq, s["cache"],
                               s["kp"], s["ke"], s["vp"], s["ve"], s["table"], s["table"].shape[1], s["q_start"], s["kv_len"],
                               s["masks"], c["words"], c["requests"], s["max_new"], s["max_len"], s["scale"], s["workspace"], s["out"],
                               hq * c["dim"])
    return s["out"]


def _own_verify(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    if "workspace" not in s:                                 # which a program keeps
        s["workspace"] = mx.verify_workspace(s["tokens"], c["requests"], c["vocab"], DEV)
    mx.mx_verify(s["logits"], s["draft"], mx.MX_F32 if c["type"] == "f32" else mx.MX_BF16, s["tokens"], c["vocab"], c["vocab"], c["vocab"],
                 s["ids"], s["parents"], s["q_start"], c["requests"], s["temperature"], s["uniform"], s["noise"], c["vocab"],
                 s["workspace"], s["path"], s["width"], s["kept"], s["next"])
    return s["path"], s["kept"], s["next"]


def _own_move(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    if "cache" not in s:
        s["cache"] = _own_cache(s)
    mx.mx_cache_move(s["cache"], s["kp"], s["ke"], s["vp"], s["ve"], s["table"], s["table"].shape[1], s["ctx"], s["path"], c["most"],
                     s["kept"], c["requests"])
    if not _block(c):
        return s["kp"], s["vp"]
    rows, f = s["pages"] * c["heads"] * c["page"], s["cache"].f
    mx.mx_dequantize(s["kp"], s["ke"], 1, rows, c["dim"], f, s["ky"])
    mx.mx_dequantize(s["vp"], s["ve"], 1, rows, c["dim"], f, s["vy"])
    return s["ky"], s["vy"]


# ---- the plain forms ------------------------------------------------------------------------------------
def _plain_tree(s):
    c, starts, parents = s["case"], s["q_start"].long(), s["parents"].long()
    N = 64 * c["words"]
    t = torch.arange(s["tokens"], device=DEV)
    b = torch.searchsorted(starts[1:], t, right=True)
    i = t - starts[b]
    up = torch.where(parents >= 0, starts[b] + parents, s["tokens"])          # a row past the last stands for the cached context
    up = torch.cat([up, up.new_full((1,), s["tokens"])])
    seen = torch.zeros((s["tokens"] + 1, N), dtype=torch.bool, device=DEV)
    seen[t, i] = True
    for _ in range(N.bit_length()):                                           # twice as many ancestors each time
        seen = seen | seen[up]
        up = up[up]
    bits = seen[:-1].unflatten(1, (c["words"], 64)).long() << torch.arange(64, device=DEV)
    return bits.sum(-1), (s["ctx"].long()[b] + seen[:-1].sum(-1) - 1).to(torch.int32)


def _values(m, e, block):
    if not block:
        return m.float()
    return torch.ldexp(m.float().unflatten(-1, (-1, block)), (e.int() - 133)[..., None]).flatten(-2)


def _plain_attend(s):
    c = s["case"]
    B, heads, group, dim, page, N, L = c["requests"], c["heads"], c["group"], c["dim"], c["page"], s["max_new"], s["max_len"]
    starts, length = s["q_start"].long(), s["kv_len"].long()
    j = torch.arange(L, device=DEV)
    entry = s["table"].long()[:, j // page].clamp(min=0)                                   # [B, L]
    k, v = (_values(m[entry, :, j % page], e[entry, :, j % page] if _block(c) else e, _block(c)).transpose(1, 2).contiguous()
            for m, e in ((s["kp"], s["ke"]), (s["vp"], s["ve"])))                          # [B, heads, L, dim]
    i = torch.arange(N, device=DEV)
    new = starts[1:] - starts[:-1]
    rows = (starts[:-1, None] + i).clamp(max=s["tokens"] - 1)
    q = s["q"][rows].float().reshape(B, N, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(B, heads, N * group, dim)
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"]).unflatten(2, (N, group))
    at = j - (length - new)[:, None]                                                       # [B, L]: which new token a key is
    word = s["masks"][rows][:, :, None, :].expand(B, N, L, c["words"]).gather(
        3, (at // 64).clamp(0, c["words"] - 1)[:, None, :, None].expand(B, N, L, 1))[..., 0]
    seen = torch.where(at[:, None, :] < 0, True, (word >> (at % 64)[:, None, :] & 1).bool()) & (j < length[:, None])[:, None, :]
    x.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(torch.where(torch.isfinite(top), top, 0.0)))
    total = x.sum(-1, keepdim=True)
    v = torch.where((j < length[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(x.flatten(2, 3), v).unflatten(2, (N, group)) / torch.where(total > 0, total, 1.0)
    t = torch.arange(s["tokens"], device=DEV)
    b = torch.searchsorted(starts[1:], t, right=True)
    return o[b, :, t - starts[b]].reshape(s["tokens"], -1).to(s["q"].dtype)


def _soft(x, heat, owner):
    """softmax(x / heat) of every row in 64 bits (acceptance and the last draw stand at borders between numbers); heat 0: all on
    the first of the largest."""
    x, cold = x.double(), (heat <= 0)[owner, None]
    top = x.amax(-1, keepdim=True)
    e = torch.exp((x - top) / torch.where(cold, 1.0, heat.double()[owner, None]))
    place = torch.arange(x.shape[-1], device=DEV)
    first = torch.where(x == top, place, x.shape[-1]).amin(-1, keepdim=True)
    return torch.where(cold, (place == first).double(), e / e.sum(-1, keepdim=True))


def _plain_verify(s):
    c, starts, V, width = s["case"], s["q_start"].long(), s["case"]["vocab"], s["width"]
    B, T, heat, last = c["requests"], s["tokens"], s["temperature"], starts[1:] - starts[:-1]
    b = torch.arange(B, device=DEV)
    owner = torch.searchsorted(starts[1:], torch.arange(T, device=DEV), right=True)
    p = _soft(s["logits"], heat, owner)
    q = _soft(s["draft"], heat, owner) if s["draft"] is not None else None
    now, kept = torch.zeros(B, dtype=torch.long, device=DEV), torch.ones(B, dtype=torch.long, device=DEV)
    path = torch.full((B, width), -1, dtype=torch.long, device=DEV)
    path[:, 0] = 0
    r, mass = p[starts[:-1]], torch.ones(B, dtype=torch.float64, device=DEV)
    for i in range(1, s["most"]):                            # a node's children come after it, in the order that they are tried in
        t = (starts[:-1] + i).clamp(max=T - 1)
        child = (i < last) & (s["parents"][t] == now) & (kept < width)
        token = s["ids"][t].long()
        drawn = q[starts[:-1] + now] if q is not None else torch.zeros_like(r).scatter_(1, token[:, None], 1.0)
        # a greedy request's draft plays no part: its tokens are tried against the one token that it allows
        drawn = torch.where((heat <= 0)[:, None], torch.zeros_like(r).scatter_(1, token[:, None], 1.0), drawn)
        here = drawn[b, token] * mass * torch.where(heat > 0, s["uniform"][t], 0.0)
        yes = child & (here < r[b, token])
        left = (r - mass[:, None] * drawn).clamp(min=0.0) if q is not None else r * (1.0 - drawn)
        left = torch.where((heat <= 0)[:, None], r * (1.0 - drawn), left)
        mass = torch.where(yes, 1.0, torch.where(child, left.sum(-1), mass))
        r = torch.where(yes[:, None], p[t], torch.where(child[:, None], left, r))
        path[b, torch.where(yes, kept, 0)] = torch.where(yes, i, path[:, 0])
        now, kept = torch.where(yes, i, now), kept + yes
    whole = p[starts[:-1] + now]
    r = torch.where(r.amax(-1, keepdim=True) > 0, r, whole)
    score = torch.where((heat > 0)[:, None], r / s["noise"].double(), whole)
    top = score.amax(-1, keepdim=True)
    place = torch.where(score == top, torch.arange(V, device=DEV), V).amin(-1)
    return path.to(torch.int32), kept.to(torch.int32), torch.where(top[:, 0] > 0, place, -1).to(torch.int32)


def _plain_move(s):
    c, table, ctx = s["case"], s["table"].long(), s["ctx"].long()
    page, block = c["page"], _block(c)
    i = torch.arange(c["most"], device=DEV)
    b, k = torch.nonzero(i[None, :] < s["kept"][:, None], as_tuple=True)
    old, new = ctx[b] + s["path"].long()[b, k], ctx[b] + k
    at, to = table[b, old // page], table[b, new // page]
    found = []
    for m, e in ((s["kp"], s["ke"]), (s["vp"], s["ve"])):
        m[to, :, new % page] = m[at, :, old % page]
        if block:
            e[to, :, new % page] = e[at, :, old % page]
        found.append(_values(m, e, block).reshape(-1, c["dim"]) if block else m)
    return tuple(found)


# ---- what a pass cannot do without ------------------------------------------------------------------------
def _density(case):
    block = _block(case)
    return 1.0 + 1.0 / block if block else 2.0


def work(case):
    if case["kind"] == "move":
        row, ctx = 2.0 * case["heads"] * case["dim"], _contexts(case)
        kept = case["most"] + (case["requests"] - 1) * (1 + case["most"]) / 2.0 - case["requests"]      # node 0 is in place
        back = row * (_density(case) + 4.0) * case["page"] * sum(_pages(c + case["nodes"], case["page"]) for c in ctx) if _block(case) else 0.0
        return {"bytes": 2.0 * kept * row * _density(case) + 8.0 * case["requests"] + 4.0 * case["requests"] * case["most"] + back, "flops": 0.0}
    sizes = _sizes(case)
    if case["kind"] == "tree":
        return {"bytes": sum(sizes) * (4.0 + 8.0 * case["words"] + 4.0) + 8.0 * case["requests"], "flops": 0.0}
    if case["kind"] == "verify":
        # the rows that a walk comes to, about two of a tree and those of half a chain; one row of random numbers
        rows = sum(min(n, 2.0 if case["branch"] > 1 else (1.0 + n) / 2.0) for n in sizes)
        width = {"f32": 4.0, "bf16": 2.0}[case["type"]] * (2 if case["draft"] else 1)
        return {"bytes": case["vocab"] * (rows * width + 4.0 * case["requests"] * (1.0 - case["greedy"])) + 12.0 * sum(sizes),
                "flops": 0.0}
    width, row = {"f32": 4.0, "bf16": 2.0}[case["type"]], float(case["heads"] * case["dim"])
    ctx = _contexts(case)
    # a node sees the cached tokens and, of its tree, at least itself
    return {"bytes": 2.0 * width * sum(sizes) * row * case["group"] + 2.0 * sum(c + n for c, n in zip(ctx, sizes)) * row * _density(case)
            + 8.0 * sum(sizes) * case["words"],
            "flops": 4.0 * sum(n * (c + 1) for c, n in zip(ctx, sizes)) * row * case["group"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------------
def _decoded(m, e, block):
    """The numbers that cached rows stand for: mantissa times a power of two, in float64."""
    if not block:
        return m.double()
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=m.device), e.double() - 127.0 - 6.0)
    return m.double() * power.repeat_interleave(block, -1)


def exact(case, seed):
    if case["kind"] in ("tree", "verify"):                   # whole numbers only
        return None
    s = prepare(case, seed)
    block, page, heads, dim = _block(case), case["page"], case["heads"], case["dim"]
    ctx = _contexts(case)
    if case["kind"] == "move":
        found = []
        for m, e in ((s["kp"], s["ke"]), (s["vp"], s["ve"])):
            pool = _decoded(m, e, block)
            was = pool.clone()
            for b in range(case["requests"]):
                row = s["table"][b].tolist()
                for k, node in enumerate(s["path"][b].tolist()[:int(s["kept"][b])]):
                    old, new = ctx[b] + node, ctx[b] + k
                    pool[row[new // page], :, new % page] = was[row[old // page], :, old % page]
            found.append(pool.reshape(-1, dim) if block else pool)
        return tuple(found)
    sizes, parents, group = _sizes(case), _trees(case, seed)[0], case["group"]
    out, t = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV), 0
    for b, (n, c) in enumerate(zip(sizes, ctx)):
        ids = s["table"][b, :_pages(c + n, page)].long()
        k, v = (_decoded(p[ids], e[ids] if block else e, block).transpose(1, 2).reshape(-1, heads, dim)[:c + n]
                for p, e in ((s["kp"], s["ke"]), (s["vp"], s["ve"])))
        seen = torch.zeros((n, c + n), dtype=torch.bool)
        seen[:, :c] = True
        for i in range(n):
            at = i
            while at >= 0:
                seen[i, c + at] = True
                at = parents[t + at]
        hide = ~seen.to(DEV)
        q = s["q"][t:t + n].double().reshape(n, heads * group, dim)
        o = out[t:t + n].reshape(n, heads * group, dim)
        for a in range(heads * group):
            x = q[:, a] @ k[:, a // group].T.contiguous() * (dim ** -0.5)
            o[:, a] = torch.softmax(x.masked_fill(hide, float("-inf")), -1) @ v[:, a // group]
        t += n
    return out
