"""The paged key/value cache: block tables and slots, append, attention over pages, against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as orc
from paper_2307_15517_amd import mx

DEV = "cuda:0"
gpu = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---- refusals (no GPU: every call returns before a launch) ------------------------------------------------
def test_cache_sizes():
    c = mx.cache_format(10, 16, 8, 128, mx.fmt(32, 8))
    assert mx.mx_cache_data_bytes(c) == 10 * 16 * 8 * 128 and mx.mx_cache_exps_bytes(c) == 10 * 16 * 8 * 4
    c = mx.cache_format(10, 64, 3, 80)
    assert mx.mx_cache_data_bytes(c) == 10 * 64 * 3 * 80 * 2 and mx.mx_cache_exps_bytes(c) == 0
    for bad in (mx.cache_format(0, 16, 8, 128), mx.cache_format(4, 24, 8, 128), mx.cache_format(4, 8, 8, 128),
                mx.cache_format(4, 2048, 8, 128), mx.cache_format(4, 16, 0, 128), mx.cache_format(4, 16, 1, 72),
                mx.cache_format(4, 16, 1, 144), mx.cache_format(1 << 27, 16, 1, 64), mx.cache_format(4, 16, 1, 48, mx.fmt(32, 8)),
                mx.cache_format(4, 16, 1, 64, mx.fmt(16, 4)), mx.cache_format(4, 16, 1, 64, mx.fmt(64, 8)),
                mx.cache_format(4, 16, 1, 64, mx.fmt(16, 8, block_rows=2))):
        assert mx.mx_cache_data_bytes(bad) == 0
        assert mx.mx_cache_attention_workspace_bytes(bad, 1, 1, 1, 1, 1) == 0


def test_plan_refusals():
    def call(ctx=256, new=256, B=2, page=16, free=256, n_free=4, table=256, width=4, tokens=8, qs=256, kv=256, slots=256, pos=256,
             counts=256):
        return mx.mx_cache_plan(ctx, new, B, page, free, n_free, table, width, tokens, qs, kv, slots, pos, counts, stream=0, check=False)
    bad, uns = mx.MX_ERR_BAD_ARG, mx.MX_ERR_UNSUPPORTED
    for kw in (dict(ctx=0), dict(new=0), dict(kv=0), dict(qs=0), dict(table=0), dict(slots=0), dict(free=0), dict(B=-1), dict(n_free=-1),
               dict(width=-1), dict(tokens=-1), dict(page=0), dict(ctx=258), dict(slots=257), dict(counts=259), dict(pos=258)):
        assert call(**kw) == bad, kw
    for kw in (dict(page=24), dict(page=8), dict(page=2048), dict(B=16385), dict(n_free=1 << 31), dict(width=1 << 31), dict(tokens=1 << 31)):
        assert call(**kw) == uns, kw


def test_append_refusals():
    f = mx.fmt(32, 8)

    def call(k=256, v=256, type=mx.MX_F32, tokens=4, ldk=128, ldv=128, c=mx.cache_format(4, 16, 2, 64, f), kd=256, ke=256, vd=256, ve=256,
             slots=256):
        return mx.mx_cache_append(k, v, type, tokens, ldk, ldv, c, kd, ke, vd, ve, slots, stream=0, check=False)
    for kw in (dict(k=0), dict(v=0), dict(kd=0), dict(vd=0), dict(ke=0), dict(ve=0), dict(slots=0), dict(type=2), dict(type=-1),
               dict(tokens=-1), dict(ldk=127), dict(ldv=127), dict(k=258), dict(v=259), dict(kd=264), dict(vd=260), dict(slots=258),
               dict(k=257, type=mx.MX_BF16), dict(c=mx.cache_format(0, 16, 2, 64, f)), dict(c=mx.cache_format(4, 16, 2, 48, f)),
               dict(c=mx.cache_format(4, 16, 2, 64, mx.fmt(32, 9)))):
        assert call(**kw) == mx.MX_ERR_BAD_ARG, kw
    for c in (mx.cache_format(4, 24, 2, 64, f), mx.cache_format(4, 16, 1, 72), mx.cache_format(4, 16, 2, 64, mx.fmt(32, 4))):
        assert call(c=c) == mx.MX_ERR_UNSUPPORTED
    assert call(tokens=0) == mx.MX_OK and call(tokens=0, k=0, v=0, slots=0) == mx.MX_OK


def test_attention_refusals():
    f = mx.fmt(32, 8)

    def call(q=256, type=mx.MX_F32, tokens=4, ldq=256, hq=4, c=mx.cache_format(4, 16, 2, 64, f), kd=256, ke=256, vd=256, ve=256, table=256,
             width=4, qs=256, kv=256, B=2, mn=1, ml=64, scale=0.125, ws=256, out=512, ldo=256):
        return mx.mx_cache_attention(q, type, tokens, ldq, hq, c, kd, ke, vd, ve, table, width, qs, kv, B, mn, ml, scale, ws, out, ldo,
                                     stream=0, check=False)
    for kw in (dict(q=0), dict(out=0), dict(ws=0), dict(ws=300), dict(kd=0), dict(vd=0), dict(ke=0), dict(ve=0), dict(table=0), dict(qs=0),
               dict(kv=0), dict(type=7), dict(tokens=-1), dict(ldq=255), dict(ldo=255), dict(hq=3), dict(hq=0), dict(width=-1), dict(B=-1),
               dict(mn=0), dict(ml=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=258), dict(out=513), dict(kd=264),
               dict(qs=258), dict(c=mx.cache_format(4, 16, 2, 48, f))):
        assert call(**kw) == mx.MX_ERR_BAD_ARG, kw
    for kw in (dict(B=16385), dict(width=1 << 27), dict(c=mx.cache_format(4, 48, 2, 64, f)), dict(c=mx.cache_format(4, 16, 2, 64, mx.fmt(64, 8))),
               dict(tokens=1 << 30)):
        assert call(**kw) == mx.MX_ERR_UNSUPPORTED, kw
    assert call(tokens=0) == mx.MX_OK


# ---- block tables and slots -------------------------------------------------------------------------------
def plan_oracle(ctx, new, page, free, table, tokens):
    """The rules of mx_cache_plan, one request after another."""
    ctx, new = [max(0, c) for c in ctx], [max(0, n) for n in new]
    table = [list(r) for r in table]
    width = len(table[0]) if table else 0
    q_start, kv_len, slots, positions, claimed, taken, refused = [0], [], [-1] * tokens, [-1] * tokens, 0, 0, 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        have, want = -(-c // page), -(-(c + n) // page)
        start = q_start[-1]
        q_start.append(start + n)
        no = want > width
        if not no:
            claimed += want - have
            no = want > have and claimed > len(free)
        if no:
            refused += 1
            kv_len.append(0)
            continue
        for j in range(have, want):
            table[b][j] = free[claimed - (want - have) + j - have]
        taken += want - have
        kv_len.append(c + n)
        for i in range(n):
            if start + i < tokens:
                positions[start + i] = c + i
                e = table[b][(c + i) // page]
                slots[start + i] = e * page + (c + i) % page if e >= 0 else -1
    return table, q_start, kv_len, slots, positions, [taken, refused]


def run_plan(ctx, new, page, free, table, tokens, **kw):
    B, width = len(ctx), len(table[0]) if table else 0
    t = ints(table).reshape(B, width)
    out = [torch.full((n,), -7, dtype=torch.int32, device=DEV) for n in (B + 1, max(B, 1), max(tokens, 1), max(tokens, 1), 2)]
    mx.mx_cache_plan(ints(ctx), ints(new), B, page, ints(free), len(free), t, width, tokens, *out, **kw)
    torch.cuda.synchronize()
    return [t.tolist()] + [o.tolist()[:n] for o, n in zip(out, (B + 1, B, tokens, tokens, 2))]


def plan_case(B, page, max_ctx, max_new, free, spare_tokens, seed, width=None):
    r = np.random.default_rng(seed)
    ctx, new = r.integers(0, max_ctx + 1, B).tolist(), r.integers(0, max_new + 1, B).tolist()
    width = width or -(-(max_ctx + max_new) // page) + 1
    have = [-(-c // page) for c in ctx]
    need = sum(-(-(c + n) // page) - h for c, n, h in zip(ctx, new, have))
    ids = r.permutation(sum(have) + need + 3).tolist()
    table, at = [], 0
    for h in have:
        row = (ids[at:at + h] + [-1] * width)[:width]
        at += h
        table.append(row)
    return ctx, new, page, ids[at:at + max(0, int(free * need))], table, max(0, sum(new) + spare_tokens)


@gpu
@pytest.mark.parametrize("case", [
    (1, 16, 0, 1, 1.0, 0), (1, 16, 15, 2, 1.0, 0), (3, 16, 40, 0, 1.0, 4), (4, 16, 1936, 1, 1.0, 0), (5, 32, 100, 70, 1.0, 9),
    (64, 128, 1000, 300, 0.5, 0), (255, 16, 64, 3, 0.9, -5), (256, 64, 64, 3, 0.0, 0), (257, 16, 50, 40, 1.0, 1), (700, 32, 3000, 90, 0.8, 7),
    (2049, 1024, 5000, 5, 0.7, 0), (16384, 16, 30, 2, 0.95, 3)])
def test_plan_matches_the_rules(case):
    args = plan_case(*case, seed=sum(case[:4]))
    assert run_plan(*args) == list(plan_oracle(*args))


@gpu
def test_plan_edges():
    # rows that are too short claim nothing and do not hold back the others; idle requests are served when pages ran out
    ctx, new = [0, 31, 100, 16, 5, -3], [33, 1, 1, 0, 40, 7]
    table = [[-1] * 3, [4, 9, -1], [1, 1, 1], [7, -1, -1], [8, -1, -1], [-1] * 3]
    for free in ([], [20], [20, 21, 22], [20, 21, 22, 23, 24, 25], list(range(30, 60))):
        args = (ctx, new, 16, free, table, 90)
        assert run_plan(*args) == list(plan_oracle(*args)), free
    # no requests: only padding tokens; no tokens; entries that were never allocated give no slot
    assert run_plan([], [], 16, [3], [], 5)[1:] == [[0], [], [-1] * 5, [-1] * 5, [0, 0]]
    assert run_plan([4], [2], 16, [], [[3]], 0)[1:3] == [[0, 2], [6]]
    assert run_plan([4], [2], 16, [], [[-1]], 2)[3] == [-1, -1]
    # positions and counts are optional
    ctx_t, new_t, tab = ints([3, 3]), ints([1, 2]), ints([[5], [6]])
    qs, kv, slots = (torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(3))
    mx.mx_cache_plan(ctx_t, new_t, 2, 16, None, 0, tab, 1, 3, qs, kv, slots, None, None)
    assert slots.tolist() == [83, 99, 100] and qs.tolist() == [0, 1, 3]
    # lengths whose sums pass 32 bits are refused by their rows and keep their places
    big = 2 ** 31 - 1
    got = run_plan([big, 0, 0], [big, big, 1], 16, [1, 2], [[-1] * 2] * 3, 4)
    assert got[1] == [0, big, big, big] and got[2] == [0, 0, 1] and got[5] == [1, 2]


# ---- append -----------------------------------------------------------------------------------------------
def cached(cache, f, c):
    """The two tensors of a cache as [pages][heads][page][dim] mantissas (or bfloat16 bits) and exponents."""
    shape = (c.pages, c.heads, c.page)
    if f is None:
        return [t.view(torch.int16).reshape(*shape, c.dim).cpu().numpy() for t in (cache.k, cache.v)], None
    return ([t.view(torch.int8).reshape(*shape, c.dim).cpu().numpy() for t in (cache.k, cache.v)],
            [t.reshape(*shape, -1).cpu().numpy() for t in (cache.k_exps, cache.v_exps)])


@gpu
@pytest.mark.parametrize("f", [None, (16, 8, mx.MX_RNE), (32, 8, mx.MX_RNE), (32, 8, mx.MX_RTZ), (16, 5, mx.MX_RNE)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,heads,dim,page,pages,lead,tail", [
    (1, 1, 64, 16, 1, 0, 0), (8, 32, 128, 16, 5, 256, 0), (333, 3, 96, 64, 7, 1, 2), (70, 12, 64, 1024, 1, 8, 3), (37, 5, 32, 32, 2, 0, 0)])
def test_append_bits(f, dtype, tokens, heads, dim, page, pages, lead, tail):
    fm = None if f is None else mx.fmt(f[0], 8, exp_bits=f[1], rounding=f[2])
    r = np.random.default_rng(tokens + dim)
    cache = mx.Cache(pages, page, heads, dim, fm, DEV)
    for t in (cache.k, cache.v, cache.k_exps, cache.v_exps):
        if t is not None:
            t.fill_(0x5A)
    total = lead + 2 * heads * dim + tail                                  # k and v are slices of one projection
    x = (r.standard_normal((tokens, total)) * 10.0 ** r.integers(-3, 3, (tokens, total))).astype(np.float32)
    x[0, lead:lead + 32] = 0.0
    x[-1, lead:lead + 4] = [2.0 ** -140, -2.0 ** -130, 2.0 ** -127, 0.0]   # subnormal values
    x[-1, -1 - tail] = 3.0e38
    xd = torch.from_numpy(x).to(DEV).to(dtype)
    k, v = xd[:, lead:lead + heads * dim], xd[:, lead + heads * dim:lead + 2 * heads * dim]
    slots = r.permutation(pages * page)[:tokens].astype(np.int32)
    slots = np.resize(slots, tokens)
    slots[len(slots) // 2] = -1
    if tokens > 3:
        slots[1], slots[2] = pages * page, 2 ** 31 - 1
    seen = {}
    for t, s in enumerate(slots):                                          # of tokens that share a slot any may stay
        if 0 <= s < pages * page:
            assert s not in seen
            seen[s] = t
    mx.cache_append(cache, k, v, ints(slots.tolist()))
    torch.cuda.synchronize()
    data, exps = cached(cache, fm, cache.c)
    for w, src in enumerate((k, v)):
        rows = src.float().cpu().numpy().reshape(tokens, heads, dim)
        want = np.full(data[w].shape, 0x5A if fm else 0x5A5A, data[w].dtype)
        if fm:
            q, e = orc.quantize(rows.reshape(tokens * heads, dim), fm.block, 8, fm.exp_bits, fm.rounding)
            q, e = np.asarray(q).reshape(tokens, heads, dim), np.asarray(e).reshape(tokens, heads, -1)
            want_e = np.full(exps[w].shape, 0x5A, np.uint8)
        else:
            q = src.contiguous().cpu().to(torch.bfloat16).view(torch.int16).numpy().reshape(tokens, heads, dim)
        for s, t in seen.items():
            want[s // page, :, s % page] = q[t]
            if fm:
                want_e[s // page, :, s % page] = e[t]
        assert np.array_equal(data[w], want)
        if fm:
            assert np.array_equal(exps[w], want_e)


@gpu
def test_append_keeps_infinities_and_nan_in_bfloat16():
    cache = mx.Cache(1, 16, 1, 16, None, DEV)
    x = torch.zeros((1, 16), device=DEV)
    x[0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.4e38], device=DEV)
    mx.cache_append(cache, x, -x, ints([3]))
    got = cache.k.view(torch.bfloat16).reshape(16, 16)
    assert torch.equal(got[3].isnan(), x[0].isnan()) and got[3, 1:4].tolist() == [float("inf"), -float("inf"), float("inf")]
    assert not got[torch.arange(16, device=DEV) != 3].any()


@gpu
def test_append_then_dequantize_reads_the_cache_back():
    f = mx.fmt(32, 8)
    cache = mx.Cache(3, 16, 2, 64, f, DEV)
    x = torch.randn((40, 128), generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    mx.cache_append(cache, x, x, torch.arange(40, dtype=torch.int32, device=DEV))
    y = mx.dequantize(cache.k, cache.k_exps, 1, 3 * 2 * 16, 64, f).reshape(3, 2, 16, 64).transpose(1, 2).reshape(48, 128)
    m, e = mx.quantize(x, f)
    assert torch.equal(y[:40], mx.dequantize(m, e, 1, 40, 128, f)[0]) and not y[40:].any()


# ---- attention --------------------------------------------------------------------------------------------
class Step:
    """A cache with random pages, and a step's requests: lens = [(new, cached with the new ones), ...]."""

    def __init__(self, lens, heads, group, dim, page, f, dtype, seed, pad=0, lead=0, qpad=0, spread=1.0, garbage=True, pages=None):
        r = np.random.default_rng(seed)
        self.lens, self.heads, self.group, self.dim, self.page, self.f, self.dtype = lens, heads, group, dim, page, f, dtype
        need = [-(-m // page) for _, m in lens]
        total = pages or sum(need) + 2
        ids = (r.permutation(min(total, 1 << 20)) + max(0, total - (1 << 20)))[:sum(need)]
        self.width = max(need + [1]) + 1
        table = np.full((len(lens), self.width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
        self.cache = mx.Cache(total, page, heads, dim, f, DEV)
        if garbage:                                          # memory that no request has written: NaN, or MXInt that is no number
            for t, byte in ((self.cache.k, 0xFF if f is None else 0x7F), (self.cache.v, 0xFF if f is None else 0x7F),
                            (self.cache.k_exps, 0xFF), (self.cache.v_exps, 0xFF)):
                if t is not None:
                    t.fill_(byte)
        self.table = torch.from_numpy(table).to(DEV)
        n_kv = sum(m for _, m in lens)
        kv = r.standard_normal((2, max(1, n_kv), heads * dim)).astype(np.float32) * spread
        kv[0, :, 3 % dim::dim] *= 4.0
        self.slots = np.concatenate([table[b, np.arange(m) // page].astype(np.int64) * page + np.arange(m) % page
                                     for b, (_, m) in enumerate(lens)] + [np.zeros(0, np.int64)])
        self.kv = torch.from_numpy(kv).to(DEV)
        if n_kv:
            mx.cache_append(self.cache, self.kv[0], self.kv[1], torch.from_numpy(self.slots.astype(np.int32)).to(DEV))
        self.tokens = lead + sum(n for n, _ in lens) + pad
        self.starts = [lead]
        for n, _ in lens:
            self.starts.append(self.starts[-1] + n)
        self.q_start, self.kv_len = ints(self.starts), ints([m for _, m in lens] or [0])[:len(lens)]
        row = heads * group * dim
        self.q = torch.from_numpy(r.standard_normal((max(1, self.tokens), row + qpad)).astype(np.float32)).to(DEV).to(dtype)[:self.tokens, :row]
        self.max_new = max([n for n, _ in lens] + [1])
        self.max_len = max([m for _, m in lens] + [1])

    def run(self, scale=None, max_new=None, max_len=None, opad=0, workspace=None):
        row = self.heads * self.group * self.dim
        out = torch.full((max(1, self.tokens), row + opad), 77.0, device=DEV, dtype=self.dtype)
        mx.cache_attention(self.cache, self.q, self.table, self.q_start, self.kv_len, max_new or self.max_new, max_len or self.max_len,
                           scale, workspace, out[:self.tokens, :row])
        torch.cuda.synchronize()
        assert bool((out[:, row:] == 77.0).all())
        return out[:self.tokens, :row]

    def values(self):
        """Cached keys and values of every request in float64, from the bits of the cache."""
        at = torch.from_numpy(self.slots).to(DEV)
        found = []
        for m, e in ((self.cache.k, self.cache.k_exps), (self.cache.v, self.cache.v_exps)):
            if self.f is None:
                x = m.view(torch.bfloat16).reshape(-1, self.heads, self.page, self.dim)[at // self.page, :, at % self.page].double()
            else:
                q = m.view(torch.int8).reshape(-1, self.heads, self.page, self.dim)[at // self.page, :, at % self.page].double()
                x = e.reshape(-1, self.heads, self.page, self.dim // self.f.block)[at // self.page, :, at % self.page].double()
                x = q * torch.exp2(x - (2 ** (self.f.exp_bits - 1) - 1) - 6).repeat_interleave(self.f.block, -1)
            found.append(x.cpu().numpy())
        return found

    def reference(self, scale=None):
        """(output, how far the kernel may be from it), from the definition in 64 bits."""
        scale = self.dim ** -0.5 if scale is None else scale
        K, V = self.values()
        q = self.q.double().cpu().numpy().reshape(self.tokens, self.heads * self.group, self.dim)
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        at = 0
        for b, (n, m) in enumerate(self.lens):
            k, v = K[at:at + m], V[at:at + m]
            at += m
            for a in range(self.heads * self.group if n else 0):
                x = q[self.starts[b]:self.starts[b] + n, a]
                s = scale * (x @ k[:, a // self.group].T)
                seen = np.arange(m)[None, :] <= (m - n + np.arange(n))[:, None]
                if m == 0:
                    continue
                s = np.where(seen, s, -np.inf)
                top = s.max(-1, keepdims=True)
                p = np.where(seen, np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
                total = p.sum(-1, keepdims=True)
                p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
                o = p @ v[:, a // self.group]
                # Scores: dim products summed in fp32, q cut at 24 bits, then scale * log2(e), its rounding and exp2's argument:
                # (dim + 8) units of 2^-24 of sum |q||k| and 4 of the largest score.  It enters numerator and sum.  Sums over the
                # keys: an fp32 rounding a term and rescaling at most, (m + 64) units of 2^-24.  bfloat16: a probability and
                # the result are rounded to 8 bits.  A probability below the smallest normal float may count as zero.
                mag = abs(scale) * (np.abs(x) @ np.abs(k[:, a // self.group]).T)
                mag = np.where(seen, mag, 0.0).max(-1, keepdims=True)
                eps = 2 * 2.0 ** -24 * ((self.dim + 8) * mag + 4 * mag) + 2 * (m + 64) * 2.0 ** -24
                size = p @ np.abs(v[:, a // self.group])
                t = eps * size + 2.0 ** -126 * (1.0 + np.abs(v[:, a // self.group]).sum(0))
                if self.dtype == torch.bfloat16:
                    t = t + 2.0 ** -9 * size + 2.0 ** -8 * np.abs(o)
                out[self.starts[b]:self.starts[b] + n, a], tol[self.starts[b]:self.starts[b] + n, a] = o, t
        return out.reshape(self.tokens, -1), tol.reshape(self.tokens, -1)

    def check(self, scale=None, **kw):
        got = self.run(scale, **kw)
        want, tol = self.reference(scale)
        err = np.abs(got.double().cpu().numpy() - want)
        assert not np.isnan(err).any()
        worst = (err - tol).max() if err.size else 0.0
        assert worst <= 0.0, (worst, err.max(), np.unravel_index((err - tol).argmax(), err.shape))
        return got


FORMATS = {"bf16": None, "mx16": mx.fmt(16, 8), "mx32": mx.fmt(32, 8)}
DECODE = [(1, 61)]
RAGGED = [(1, 1), (1, 2), (1, 15), (1, 16), (1, 17), (1, 33), (1, 700), (1, 128), (1, 129)]
FEW = [(3, 3), (2, 40), (7, 500), (1, 64), (5, 31), (16, 16)]
CHUNKS = [(40, 100), (129, 129), (1, 77), (17, 300), (200, 201)]
PROMPT = [(333, 333)]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
@pytest.mark.parametrize("lens,heads,group,dim,page", [
    (DECODE, 12, 1, 64, 16), (DECODE, 2, 5, 128, 64), (RAGGED, 2, 4, 128, 16), (RAGGED, 3, 1, 96, 32), (FEW, 2, 3, 64, 16), (FEW, 1, 8, 128, 128),
    (CHUNKS, 2, 2, 128, 16), (CHUNKS, 1, 1, 32, 16), (CHUNKS, 1, 7, 96, 1024), (PROMPT, 2, 1, 128, 32), (PROMPT, 1, 4, 64, 64)])
def test_attention(dtype, kind, lens, heads, group, dim, page):
    Step(lens, heads, group, dim, page, FORMATS[kind], dtype, seed=dim + len(lens)).check()


@gpu
@pytest.mark.parametrize("dim", [16, 48, 80, 112])
@pytest.mark.parametrize("kind", ["bf16", "mx16"])
def test_attention_head_dimensions(dim, kind):
    Step(FEW + CHUNKS, 2, 2, dim, 16, FORMATS[kind], torch.float32, seed=dim).check()
    Step(FEW + CHUNKS, 1, 3, dim, 32, FORMATS[kind], torch.bfloat16, seed=dim).check()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx32"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_split_over_a_long_axis(dtype, kind):
    Step([(1, 9001)], 1, 4, 128, 64, FORMATS[kind], dtype, seed=3).check()
    Step([(1, 5000), (2, 17), (1, 300), (4, 4999)], 2, 2, 64, 16, FORMATS[kind], dtype, seed=4).check()
    Step([(33, 6000)], 1, 2, 128, 16, FORMATS[kind], dtype, seed=5).check()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_rows_without_keys_and_padding(dtype):
    """Idle requests, requests without cached tokens (refused ones), more new tokens than cached ones, padding at both ends."""
    for lens in ([(0, 40), (3, 0), (5, 2), (1, 50), (0, 0)], [(2, 0)], [(40, 39), (70, 100), (64, 1)], [(0, 17)], []):
        s = Step(lens, 2, 2, 64, 16, FORMATS["mx32"], dtype, seed=6, pad=5, lead=3)
        got = s.check()
        assert not got[:3].any() and not got[s.tokens - 5:].any()


@gpu
@pytest.mark.parametrize("lead,qpad,opad", [(0, 0, 1), (1, 3, 5), (0, 64, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_strides(dtype, lead, qpad, opad):
    for lens in (RAGGED, CHUNKS):
        Step(lens, 2, 2, 64, 16, FORMATS["mx16"], dtype, seed=8, qpad=qpad, lead=lead).check(opad=opad)


@gpu
@pytest.mark.parametrize("lens", [RAGGED, FEW, CHUNKS, [(1, 4000)]])
def test_attention_bounds_on_lengths_only_shape_the_launch(lens):
    for dtype in (torch.float32, torch.bfloat16):
        s = Step(lens, 2, 2, 128, 16, FORMATS["mx32"], dtype, seed=9)
        for mn, ml in ((1, 1), (10000, 100000), (1, 100000), (500, 1)):
            s.check(max_new=mn, max_len=ml)


@gpu
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1.0, 3.0])
@pytest.mark.parametrize("lens", [FEW, CHUNKS])
def test_attention_scales(scale, lens):
    Step(lens, 2, 2, 64, 16, FORMATS["mx32"], torch.float32, seed=10).check(scale)
    Step(lens, 2, 2, 64, 16, FORMATS["bf16"], torch.bfloat16, seed=10).check(scale)


@gpu
def test_attention_exponent_bits_and_spread():
    for f in (mx.fmt(16, 8, exp_bits=4), mx.fmt(32, 8, exp_bits=6, rounding=mx.MX_RTZ)):
        Step(FEW + CHUNKS, 2, 2, 64, 16, f, torch.float32, seed=11).check()
    for spread in (1e-6, 30.0):
        Step(FEW + CHUNKS, 2, 2, 64, 16, FORMATS["mx32"], torch.float32, seed=12, spread=spread).check()
        Step(FEW + CHUNKS, 2, 2, 64, 16, FORMATS["bf16"], torch.bfloat16, seed=12, spread=spread).check()


@gpu
def test_attention_offsets_past_32_bits():
    """A pool whose bytes and whose rows' offsets pass 32 bits, with the pages in use at its end."""
    s = Step([(1, 200), (40, 70)], 8, 2, 128, 16, None, torch.bfloat16, seed=13, garbage=False, pages=(1 << 20) + 200000)
    assert int(s.table.max()) * 16 * 8 * 128 * 2 > 1 << 32
    s.check()
    s = Step([(1, 200), (40, 70)], 8, 2, 128, 16, FORMATS["mx32"], torch.float32, seed=13, garbage=False, pages=(1 << 20) + 200000)
    s.check()


@gpu
def test_attention_bad_indices_do_not_reach_memory():
    """Page indices outside the pool read page 0, lengths stop at the table row, token ranges at the packed tokens."""
    s = Step([(2, 60), (30, 64)], 2, 2, 64, 16, FORMATS["mx32"], torch.float32, seed=14)
    s.table[0, :4] = ints([2 ** 31 - 1, -5, s.cache.c.pages, -2 ** 31])
    s.kv_len.fill_(2 ** 31 - 1)
    s.q_start.copy_(ints([-4, 2, 2 ** 31 - 1]))
    for lens in ((1, 1), (100, 100000)):
        assert s.run(max_new=lens[0], max_len=lens[1]).shape == (32, 256)


@gpu
def test_attention_same_inputs_same_bits_also_on_another_stream():
    s = Step(CHUNKS + [(1, 5000)], 2, 4, 128, 16, FORMATS["mx32"], torch.float32, seed=15)
    ws = mx.cache_workspace(s.cache.c, s.tokens, len(s.lens), 8, s.max_new, s.max_len, DEV)
    first = s.check(workspace=ws)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        again = s.run(workspace=ws)
    assert torch.equal(first, again) and not ws[:65536].any()


@gpu
def test_step_in_a_graph():
    """Plan, append and attention of a decode step, captured once and replayed on new lengths and rows."""
    B, heads, group, dim, page = 5, 2, 4, 64, 16
    f = FORMATS["mx32"]
    cache = mx.Cache(64, page, heads, dim, f, DEV)
    table = torch.full((B, 8), -1, dtype=torch.int32, device=DEV)
    free = torch.arange(64, dtype=torch.int32, device=DEV)
    ctx, new = ints([0] * B), ints([1] * B)
    k, v, q = (torch.zeros((B, n * dim), device=DEV) for n in (heads, heads, heads * group))
    ws = mx.cache_workspace(cache.c, B, B, heads * group, 1, 128, DEV)
    out = torch.empty_like(q)

    def step():
        q_start, kv_len, slots, _, _ = mx.cache_plan(ctx, new, page, free, table, B)
        mx.cache_append(cache, k, v, slots)
        mx.cache_attention(cache, q, table, q_start, kv_len, 1, 128, None, ws, out)

    g = torch.cuda.CUDAGraph()
    step()
    table.fill_(-1)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    rng = torch.Generator(DEV).manual_seed(2)
    for at in range(20):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=rng, device=DEV))
        ctx.fill_(at)
        free.copy_(torch.arange(64, dtype=torch.int32, device=DEV).roll(-B * (-(-at // page))))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and got.isfinite().all()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_batches_whose_tiles_are_split_unevenly(dtype, kind):
    """Row tiles of one run next to tiles of many, and requests of a few rows beside both; more than sixteen runs of a tile; a
    tile whose first rows see nothing."""
    Step([(300, 3000), (1, 2000), (300, 310), (20, 60), (3, 900)], 2, 2, 96, 16, FORMATS[kind], dtype, seed=16).check()
    Step([(1, 4), (40, 9000), (1, 5000), (25, 64)], 1, 2, 64, 32, FORMATS[kind], dtype, seed=17).check()
    Step([(90, 4000), (1, 3000), (70, 40), (200, 7)], 1, 1, 80, 16, FORMATS[kind], dtype, seed=18).check()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("requests,heads,group,most_new,longest", [(40, 8, 4, 1, 4000), (40, 8, 4, 4, 41000), (64, 12, 1, 2, 600),
                                                                 (65, 8, 1, 1, 700), (300, 4, 1, 1, 200), (150, 2, 1, 30, 90)])
def test_attention_many_requests(dtype, requests, heads, group, most_new, longest):
    """The longest requests first, however they stand; parts joined by a launch of their own; more requests than a wave has lanes."""
    r = np.random.default_rng(requests + longest)
    lens = [(int(r.integers(0, most_new + 1)), int(r.integers(1, min(longest, 400) + 1))) for _ in range(requests)]
    lens[requests // 2], lens[requests // 3] = (most_new, longest), (1, longest)
    Step(lens, heads, group, 64, 16, FORMATS["mx32"], dtype, seed=requests).check()


@gpu
@pytest.mark.parametrize("f", [None, FORMATS["mx32"]])
def test_serving_example(f):
    """The example's steps against attention in float64 over the keys and values that its cache holds."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    r = np.random.default_rng(5)
    waiting = [ex.Request(r.integers(0, ex.VOCAB, n), m) for n, m in ((100, 4), (1, 9), (49, 2), (16, 3), (30, 1), (7, 5), (64, 2))]
    lengths = sorted(x.stop + 1 for x in waiting)
    server = ex.Server(batch=4, pages=64, page=16, max_len=160, chunk=48, f=f)
    finished = []
    for _ in range(40):
        server.admit(waiting)
        if all(x is None for x in server.places):
            break
        finished += server.step()
        q, o, q_start, kv_len = server.last
        c, found = server.cache.c, []
        for data, exps in ((server.cache.k, server.cache.k_exps), (server.cache.v, server.cache.v_exps)):
            x = data.view(torch.bfloat16) if f is None else mx.dequantize(data, exps, 1, c.pages * c.heads * c.page, c.dim, f)
            found.append(x.reshape(c.pages, c.heads, c.page, c.dim).double().cpu())
        table, q, o, q_start, kv_len = (t.cpu() for t in (server.table, q.double(), o.double(), q_start, kv_len))
        for b in range(4):
            n, m = int(q_start[b + 1] - q_start[b]), int(kv_len[b])
            if n == 0:
                continue
            pages = table[b, :-(-m // 16)].long()
            k, v = (x[pages].transpose(0, 1).reshape(c.heads, -1, c.dim)[:, :m] for x in found)
            rows = slice(int(q_start[b]), int(q_start[b + 1]))
            for a in range(ex.HEADS_Q):
                x, h = q[rows, a * 64:(a + 1) * 64], a // (ex.HEADS_Q // ex.HEADS)
                s = (x @ k[h].T) / 8.0
                s = s.masked_fill(torch.arange(m)[None, :] > (m - n + torch.arange(n))[:, None], -np.inf)
                # fp32 throughout: as in Step.reference, with |s| <= |q||k|/8
                mag = (x.abs() @ k[h].abs().T).max() / 8.0
                eps = 2 * 2.0 ** -24 * (64 + 12) * mag + 2 * (m + 64) * 2.0 ** -24
                p = torch.softmax(s, -1)
                assert ((o[rows, a * 64:(a + 1) * 64] - p @ v[h]).abs() <= eps * (p @ v[h].abs()) + 2.0 ** -120).all()
    assert sorted(len(x.tokens) for x in finished) == lengths and sorted(server.free) == list(range(64))


@gpu
@pytest.mark.parametrize("lens", [RAGGED, CHUNKS, [(300, 2000)]])
def test_attention_takes_any_bounds(lens):
    """Bounds as large as the type holds: no sum or product of the host's arithmetic may leave its range."""
    for dtype in (torch.float32, torch.bfloat16):
        s = Step(lens, 2, 2, 64, 16, FORMATS["mx32"], dtype, seed=19)
        for bound in (2 ** 31 - 1, 2 ** 40, 2 ** 63 - 1):
            s.check(max_new=bound, max_len=bound)
