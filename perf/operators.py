"""The operators of the paged key/value cache, as cases that can be timed: what a serving program does between the
linear layers of a step.

A case is a dict of plain values.  ``prepare`` makes what a program holds before the call, ``run`` is one pass: with
``own`` false in plain elementary torch operations (32 bits, rounded once at the end), with ``own`` true through the
public entry points of ``paper_2307_15517_amd.mx``.  ``work`` is what a pass cannot do without, ``exact`` the result
from the definition in 64 bits.

The kinds:

* ``plan``    block tables, slot and position maps of a step, built on the GPU from the requests' lengths.
* ``append``  the new tokens' keys and values, slices of one fused projection, into their slots of the cache: bfloat16
              elements, or MXInt with 8 stored bits and blocks of 16 or 32 along the head dimension.  The MXInt cache is
              returned as the values it stands for, which the framework's own dequantizer gives.
* ``attend``  attention of every request's new tokens over its pages, causal, grouped heads, requests of different
              lengths packed one after another: single tokens (decoding), chunks of a prompt, whole prompts.

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
        # four sequences, one new token each: the smallest step of a server
        dict(name="plan_decode_4", kind="plan", requests=4, page=16, max_ctx=1936, max_new=1, single=1.0, scarce=False),
        # continuous batching: several hundred sequences decode while others bring prompts, and pages run short
        dict(name="plan_mixed_700", kind="plan", requests=700, page=32, max_ctx=8192, max_new=1024, single=0.9, scarce=True),
        # the new keys and values of eight decoding sequences, heads of LLaMA-7B, bfloat16 cache
        dict(name="append_decode_8", kind="append", tokens=8, heads=32, group=1, dim=128, page=16, pages=512, cache="bf16",
             type="f32", skip=0.0),
        # a prompt of odd length into the MXInt cache, blocks of 32, grouped heads
        dict(name="append_prompt_1999", kind="append", tokens=1999, heads=8, group=4, dim=128, page=64, pages=32, cache="mx32",
             type="f32", skip=0.0),
        # a chunk of bfloat16 activations, heads of OPT-125M, blocks of 16, padding tokens at the end
        dict(name="append_chunk_333", kind="append", tokens=333, heads=12, group=1, dim=64, page=16, pages=24, cache="mx16",
             type="bf16", skip=0.1),
        # one token of a short sequence, heads of OPT-125M: latency counts
        dict(name="attend_token_61", kind="attend", requests=1, max_new=1, single=1.0, min_len=61, max_len=61, whole=False,
             heads=12, group=1, dim=64, page=16, cache="mx32", type="f32"),
        # one new token of one sequence against 1936 cached positions, heads of LLaMA-7B
        dict(name="attend_decode_1936", kind="attend", requests=1, max_new=1, single=1.0, min_len=1936, max_len=1936,
             whole=False, heads=32, group=1, dim=128, page=16, cache="mx32", type="f32"),
        # 32 sequences of very different lengths decoding, grouped heads, MXInt cache
        dict(name="attend_decode_32", kind="attend", requests=32, max_new=1, single=1.0, min_len=1, max_len=8191, whole=False,
             heads=8, group=4, dim=128, page=32, cache="mx32", type="bf16"),
        # one long sequence decoding, bfloat16 cache: the largest read
        dict(name="attend_long_100003", kind="attend", requests=1, max_new=1, single=1.0, min_len=100003, max_len=100003,
             whole=False, heads=8, group=5, dim=128, page=64, cache="bf16", type="bf16"),
        # a chunk of 300 new tokens after 1700 cached ones, fp32 activations, heads of LLaMA-7B
        dict(name="attend_chunk_300", kind="attend", requests=1, max_new=300, single=0.0, min_len=2000, max_len=2000,
             whole=False, heads=32, group=1, dim=128, page=16, cache="mx32", type="f32"),
        # five whole prompts packed, up to 4096 tokens: the largest product
        dict(name="attend_prompts_5", kind="attend", requests=5, max_new=4096, single=0.0, min_len=300, max_len=4096,
             whole=True, heads=8, group=4, dim=128, page=64, cache="bf16", type="bf16"),
        # continuous batching: most sequences decode, a few bring chunks; head dimension 96, blocks of 16
        dict(name="attend_mixed_24", kind="attend", requests=24, max_new=500, single=0.85, min_len=7, max_len=3000,
             whole=False, heads=8, group=3, dim=96, page=16, cache="mx16", type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    kind = rng.choice(["plan", "append", "append", "attend", "attend", "attend", "attend"])
    if kind == "plan":
        single = rng.choice([1.0, 1.0, 0.9, 0.5, 0.0])
        return dict(kind=kind, requests=_log(rng, 1, 900 if single > 0.6 else 60), page=rng.choice([16, 32, 64, 128]),
                    max_ctx=_log(rng, 16, 16384), max_new=1 if single == 1.0 else _log(rng, 2, 1024), single=single,
                    scarce=rng.random() < 0.3)
    dim = rng.choice([64, 80, 96, 112, 128, 128, 128])
    cache = rng.choice(["bf16", "mx16", "mx32"] if dim % 32 == 0 else ["bf16", "mx16"])
    if kind == "append":
        tokens, page = _log(rng, 1, 2000), rng.choice([16, 32, 64, 128])
        return dict(kind=kind, tokens=tokens, heads=rng.choice([1, 4, 8, 12, 32]) if tokens < 500 else rng.choice([4, 8]),
                    group=rng.choice([1, 2, 4]), dim=dim, page=page, pages=-(-tokens * 5 // (4 * page)) + rng.randint(0, 3),
                    cache=cache, type=rng.choice(["f32", "bf16"]), skip=rng.choice([0.0, 0.0, 0.2]))
    while True:
        sort = rng.choice(["decode", "decode", "few", "chunk", "prompt", "mixed"])
        c = dict(kind=kind, requests=1, max_new=1, single=1.0, min_len=1, max_len=1, whole=sort == "prompt",
                 heads=rng.choice([1, 2, 4, 8, 8, 12, 32]), group=rng.choice([1, 1, 2, 3, 4, 5, 8]), dim=dim,
                 page=rng.choice([16, 32, 64, 128]), cache=cache, type=rng.choice(["f32", "bf16", "bf16"]))
        if sort == "prompt":
            c.update(requests=_log(rng, 1, 6), single=0.0, max_new=_log(rng, 40, 3000))
            c.update(max_len=c["max_new"], min_len=max(1, c["max_new"] // 8))
        else:
            c.update(requests=_log(rng, 1, 64 if sort == "decode" else 12), max_len=_log(rng, 20, 30000 if sort == "decode" else 6000))
            c.update(min_len=rng.choice([1, c["max_len"] // 2 + 1, c["max_len"]]))
            if sort != "decode":
                c.update(max_new=min(c["max_len"], _log(rng, 2, 8) if sort == "few" else _log(rng, 20, 700)),
                         single=0.8 if sort == "mixed" else 0.0)
        # no more than the largest listed ones, also where the plain form pads every request to the longest
        w, hq = work(c), c["heads"] * c["group"]
        if (w["bytes"] <= 4e8 and w["flops"] <= 1.5e11 and c["requests"] * c["max_len"] * c["heads"] * dim <= 1.2e8
                and c["requests"] * hq * c["max_new"] * c["max_len"] <= 1.5e9):
            return c


# ---- sizes that follow from a case ----------------------------------------------------------------------
def _block(case):
    return {"bf16": 0, "mx16": 16, "mx32": 32}[case["cache"]]


def _lengths(case):
    """(new tokens, tokens with the new ones) of every request of an attend case; the first has the largest of both."""
    r = random.Random("%(requests)d %(max_new)d %(min_len)d %(max_len)d" % case)
    new, length = [case["max_new"]], [case["max_len"]]
    while len(new) < case["requests"]:
        n = 1 if r.random() < case["single"] else r.randint(1, case["max_new"])
        m = r.randint(case["min_len"], case["max_len"])
        if case["whole"]:
            n = m = max(n, case["min_len"])
        new.append(n)
        length.append(max(n, m))
    return new, length


def _plan_lengths(case):
    """(tokens cached, new tokens) of every request of a plan case; some are idle, some bring a prompt."""
    r = random.Random("%(requests)d %(page)d %(max_ctx)d %(max_new)d" % case)
    ctx, new = [], []
    for _ in range(case["requests"]):
        one = r.random() < case["single"]
        ctx.append(r.randint(0, case["max_ctx"]) if one or r.random() < 0.5 else 0)
        new.append(1 if one else r.randint(0, case["max_new"]))
    return ctx, new


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


def _pool(g, case, pages):
    """Keys (or values) of a whole cache and their exponents; every place holds something, as in a cache long in use."""
    x = _rows(g, (pages, case["heads"], case["page"], case["dim"]))
    block = _block(case)
    if not block:
        return x.to(torch.bfloat16), torch.zeros(16, dtype=torch.uint8, device=DEV)
    return _quantized(x, block)


def prepare(case, seed):
    g = _gen(seed)
    return dict({"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend}[case["kind"]](case, g),
                case=dict(case))


def _prepare_plan(case, g):
    ctx, new = _plan_lengths(case)
    page, B = case["page"], case["requests"]
    width = _pages(case["max_ctx"] + case["max_new"], page)
    have = [_pages(c, page) for c in ctx]
    need = [_pages(c + n, page) - h for c, n, h in zip(ctx, new, have)]
    total = sum(have) + sum(need) + 8
    ids = _order(g, total)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV)[None, :] < torch.tensor(have, device=DEV)[:, None]
    table[held] = ids[:sum(have)]
    free = ids[sum(have):].contiguous()
    tokens = sum(new)
    empty = lambda n: torch.empty(max(1, n), dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(ctx=_ints(ctx), new=_ints(new), free=free, n_free=int(0.8 * sum(need)) if case["scarce"] else free.numel(),
                table=table, tokens=tokens, q_start=empty(B + 1), kv_len=empty(B), slots=empty(tokens),
                positions=empty(tokens), counts=empty(2))


def _prepare_append(case, g):
    heads, dim, tokens = case["heads"], case["dim"], case["tokens"]
    qkv = _rows(g, (tokens, (case["group"] + 2) * heads * dim)).to(TYPES[case["type"]])
    k = qkv[:, case["group"] * heads * dim:(case["group"] + 1) * heads * dim]
    v = qkv[:, (case["group"] + 1) * heads * dim:]
    slots = _order(g, case["pages"] * case["page"])[:tokens].contiguous()
    slots[tokens - int(case["skip"] * tokens):] = -1
    kp, ke = _pool(g, case, case["pages"])
    vp, ve = _pool(g, case, case["pages"])
    shape = (case["pages"] * heads * case["page"], dim) if _block(case) else (1, 1)
    return dict(qkv=qkv, k=k, v=v, slots=slots, kp=kp, ke=ke, vp=vp, ve=ve, ld=qkv.stride(0),
                ky=torch.empty(shape, device=DEV), vy=torch.empty(shape, device=DEV))


def _prepare_attend(case, g):
    new, length = _lengths(case)
    page, B, hq, dim = case["page"], case["requests"], case["heads"] * case["group"], case["dim"]
    need = [_pages(n, page) for n in length]
    pages, width, tokens = sum(need) + 1, max(need), sum(new)
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    held = torch.arange(width, device=DEV)[None, :] < torch.tensor(need, device=DEV)[:, None]
    table[held] = _order(g, pages)[:sum(need)]
    kp, ke = _pool(g, case, pages)
    vp, ve = _pool(g, case, pages)
    q = _rows(g, (tokens, hq * dim)).to(TYPES[case["type"]])
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return dict(q=q, out=torch.empty_like(q), table=table, q_start=_ints(starts), kv_len=_ints(length), kp=kp, ke=ke, vp=vp,
                ve=ve, tokens=tokens, pages=pages, max_new=max(new), max_len=max(length), scale=dim ** -0.5)


# ---- one pass -------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if kind == "plan":
        return (_own_plan if own else _plain_plan)(state)
    if kind == "append":
        return (_own_append if own else _plain_append)(state)
    return (_own_attend if own else _plain_attend)(state)


def _own_cache(s, pages):
    from paper_2307_15517_amd import mx
    c = s["case"]
    block = _block(c)
    return mx.cache_format(pages, c["page"], c["heads"], c["dim"], mx.fmt(block, 8) if block else None)


def _own_plan(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    mx.mx_cache_plan(s["ctx"], s["new"], c["requests"], c["page"], s["free"], s["n_free"], s["table"], s["table"].shape[1],
                     s["tokens"], s["q_start"], s["kv_len"], s["slots"], s["positions"], s["counts"])
    return s["table"], s["q_start"], s["kv_len"], s["slots"], s["positions"], s["counts"]


def _own_append(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    if "cache" not in s:                                     # the cache's description, which a program makes once
        s["cache"] = _own_cache(s, c["pages"])
    mx.mx_cache_append(s["k"], s["v"], mx.MX_F32 if c["type"] == "f32" else mx.MX_BF16, c["tokens"], s["ld"], s["ld"], s["cache"],
                       s["kp"], s["ke"], s["vp"], s["ve"], s["slots"])
    if not _block(c):
        return s["kp"], s["vp"]
    rows, f = c["pages"] * c["heads"] * c["page"], s["cache"].f
    mx.mx_dequantize(s["kp"], s["ke"], 1, rows, c["dim"], f, s["ky"])
    mx.mx_dequantize(s["vp"], s["ve"], 1, rows, c["dim"], f, s["vy"])
    return s["ky"], s["vy"]


def _own_attend(s):
    from paper_2307_15517_amd import mx
    c = s["case"]
    hq = c["heads"] * c["group"]
    if "cache" not in s:                                     # the description and the workspace, which a program keeps
        s["cache"] = _own_cache(s, s["pages"])
        s["workspace"] = mx.cache_workspace(s["cache"], s["tokens"], c["requests"], hq, s["max_new"], s["max_len"], DEV)
    mx.mx_cache_attention(s["q"], mx.MX_F32 if c["type"] == "f32" else mx.MX_BF16, s["tokens"], hq * c["dim"], hq, s["cache"],
                          s["kp"], s["ke"], s["vp"], s["ve"], s["table"], s["table"].shape[1], s["q_start"], s["kv_len"],
                          c["requests"], s["max_new"], s["max_len"], s["scale"], s["workspace"], s["out"], hq * c["dim"])
    return s["out"]


# ---- the plain form -------------------------------------------------------------------------------------
def _plain_plan(s):
    page, n_free, table, tokens = s["case"]["page"], s["n_free"], s["table"], s["tokens"]
    B, width = table.shape
    ctx, new = s["ctx"].long(), s["new"].long()
    have, want = (ctx + page - 1) // page, (ctx + new + page - 1) // page
    wide = want > width
    need = torch.where(wide, 0, want - have)
    upto = torch.cumsum(need, 0)
    refused = wide | ((need > 0) & (upto > n_free))
    j = torch.arange(width, device=DEV)[None, :]
    fresh = (j >= have[:, None]) & (j < want[:, None]) & ~refused[:, None]
    at = ((upto - need)[:, None] + j - have[:, None]).clamp(0, s["free"].numel() - 1)
    table = torch.where(fresh, s["free"][at], table)
    q_start = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(new, 0)])
    kv_len = torch.where(refused, 0, ctx + new)
    t = torch.arange(tokens, device=DEV)
    b = torch.searchsorted(q_start[1:], t, right=True).clamp(max=B - 1)
    position = ctx[b] + t - q_start[b]
    served = (t < q_start[-1]) & ~refused[b]
    entry = table[b, (position // page).clamp(0, width - 1)].long()
    slots = torch.where(served & (entry >= 0), entry * page + position % page, -1)
    counts = torch.stack([torch.where(refused, 0, need).sum(), refused.sum()])
    i32 = torch.int32
    return table, q_start.to(i32), kv_len.to(i32), slots.to(i32), torch.where(served, position, -1).to(i32), counts.to(i32)


def _quantized(x, block):
    """MXInt with 8 stored bits: mantissas (int8) and exponent bytes, blocks along the last axis."""
    y = x.float().unflatten(-1, (-1, block))
    top = y.abs().amax(-1)
    e = (torch.frexp(top)[1] - 1).clamp(-127, 128)
    m = torch.round(torch.ldexp(y, (6 - e)[..., None])).clamp(-127, 127)
    return m.to(torch.int8).flatten(-2), torch.where(top == 0, 0, e + 127).to(torch.uint8)


def _values(m, e, block):
    if not block:
        return m.float()
    return torch.ldexp(m.float().unflatten(-1, (-1, block)), (e.int() - 133)[..., None]).flatten(-2)


def _plain_append(s):
    c = s["case"]
    block, page, heads, dim = _block(c), c["page"], c["heads"], c["dim"]
    found = []
    last = c["tokens"] - int(c["skip"] * c["tokens"])        # those that the program knows to be padding
    for x, m, e in ((s["k"], s["kp"], s["ke"]), (s["v"], s["vp"], s["ve"])):
        x, at = x[:last].unflatten(-1, (heads, dim)), s["slots"][:last].long()
        if block:
            mant, exps = _quantized(x, block)
            m[at // page, :, at % page] = mant
            e[at // page, :, at % page] = exps
        else:
            m[at // page, :, at % page] = x.to(torch.bfloat16)
        found.append(_values(m, e, block).reshape(-1, dim) if block else m)
    return tuple(found)


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
    last = (length - new)[:, None] + i                                                    # [B, N]: the last key a row sees
    x.masked_fill_((j > last[..., None])[:, None, :, None, :], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(torch.where(torch.isfinite(top), top, 0.0)))
    total = x.sum(-1, keepdim=True)
    v = torch.where((j < length[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(x.flatten(2, 3), v).unflatten(2, (N, group)) / torch.where(total > 0, total, 1.0)
    t = torch.arange(s["tokens"], device=DEV)
    b = torch.searchsorted(starts[1:], t, right=True)
    return o[b, :, t - starts[b]].reshape(s["tokens"], -1).to(s["q"].dtype)


# ---- what a pass cannot do without ------------------------------------------------------------------------
def _density(case):
    block = _block(case)
    return 1.0 + 1.0 / block if block else 2.0


def work(case):
    if case["kind"] == "plan":
        ctx, new = _plan_lengths(case)
        page = case["page"]
        taken = sum(_pages(c + n, page) - _pages(c, page) for c, n in zip(ctx, new)) * (0.8 if case["scarce"] else 1.0)
        return {"bytes": 16.0 * case["requests"] + 8.0 * taken + 8.0 * sum(new) + 12.0, "flops": 0.0}
    width = {"f32": 4.0, "bf16": 2.0}[case["type"]]
    row = float(case["heads"] * case["dim"])
    if case["kind"] == "append":
        used = case["tokens"] - int(case["skip"] * case["tokens"])
        back = 2.0 * case["pages"] * case["page"] * row * (_density(case) + 4.0) if _block(case) else 0.0
        return {"bytes": 2.0 * used * row * (width + _density(case)) + 4.0 * case["tokens"] + back, "flops": 0.0}
    new, length = _lengths(case)
    seen = sum(n * (m - n) + n * (n + 1) / 2.0 for n, m in zip(new, length))
    return {"bytes": 2.0 * width * sum(new) * row * case["group"] + 2.0 * sum(length) * row * _density(case),
            "flops": 4.0 * seen * row * case["group"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------------
def _decoded(m, e, block):
    """The numbers that cached rows stand for: mantissa times a power of two, in float64."""
    if not block:
        return m.double()
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=m.device), e.double() - 127.0 - 6.0)
    return m.double() * power.repeat_interleave(block, -1)


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    s = prepare(case, seed)
    block, page, heads, dim = _block(case), case["page"], case["heads"], case["dim"]
    if case["kind"] == "append":
        found, used = [], case["tokens"] - int(case["skip"] * case["tokens"])
        slot = s["slots"][:used].tolist()
        where = torch.tensor([p // page for p in slot], device=DEV), torch.tensor([p % page for p in slot], device=DEV)
        for x, m, e in ((s["k"], s["kp"], s["ke"]), (s["v"], s["vp"], s["ve"])):
            pool = _decoded(m, e, block)
            x = x[:used].double().reshape(used, heads, dim)
            if block:
                y = x.reshape(used, heads, dim // block, block)
                top = y.abs().amax(-1, keepdim=True)
                step = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 6.0)
                step = torch.where(top / step >= 128.0, step * 2.0, torch.where(top / step < 64.0, step * 0.5, step))
                y = torch.clamp(torch.round(y / torch.where(top > 0, step, 1.0)), -127, 127) * step
                x = y.reshape(used, heads, dim)
            pool[where[0], :, where[1]] = x
            found.append(pool.reshape(-1, dim) if block else pool)
        return tuple(found)
    new, length = _lengths(case)
    group, out, t = case["group"], torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV), 0
    for b, (n, m) in enumerate(zip(new, length)):
        ids = s["table"][b, :_pages(m, page)].long()
        k, v = (_decoded(p[ids], e[ids] if block else e, block).transpose(1, 2).reshape(-1, heads, dim)[:m]
                for p, e in ((s["kp"], s["ke"]), (s["vp"], s["ve"])))
        q = s["q"][t:t + n].double().reshape(n, heads * group, dim)
        seen = torch.arange(m, device=DEV)[None, :] <= torch.arange(m - n, m, device=DEV)[:, None]
        o = out[t:t + n].reshape(n, heads * group, dim)
        for a in range(heads * group):
            x = q[:, a] @ k[:, a // group].T.contiguous() * (dim ** -0.5)
            p = torch.softmax(x.masked_fill(~seen, float("-inf")), -1)
            o[:, a] = p @ v[:, a // group]
        t += n
    return out
