"""Trees, attention, verification and moved rows together, as a server runs them: the example, whole steps against plain ones, graphs."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

from paper_2307_15517_amd import mx
from test_cache import DEV, FORMATS, ints
from test_tree import random_parents
from test_verify import walk

gpu = pytest.mark.gpu


def example(name):
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", name + ".py")
    spec = importlib.util.spec_from_file_location(name, path)
    ex = importlib.util.module_from_spec(spec)
    sys.modules[name] = ex
    spec.loader.exec_module(ex)
    return ex


def serve(server, waiting, steps=500):
    finished = []
    for _ in range(steps):
        server.admit(waiting)
        if all(x is None for x in server.places):
            return finished
        finished += server.step()
    raise AssertionError("not done")


def requests(ex, r, lengths):
    return [ex.Request(r.integers(0, ex.VOCAB, n).tolist(), m) for n, m in lengths]


LENGTHS = [(100, 24), (1, 39), (49, 12), (16, 30), (30, 1), (7, 25), (64, 18), (15, 33), (33, 20)]


@gpu
@pytest.mark.parametrize("f", [None, FORMATS["mx32"]])
@pytest.mark.parametrize("nodes,branch", [(8, 2), (1, 1), (5, 1), (40, 5), (70, 9)])
def test_greedy_speculation_gives_the_same_tokens(f, nodes, branch):
    """Every request's tokens are those that one token a step gives, whatever is drafted; all pages come back."""
    plain, ex = example("paged_serving"), example("speculative_serving")
    served = []
    for server in (plain.Server(batch=4, pages=80, max_len=160, f=f, seed=3),
                   ex.Speculative(nodes, branch, batch=4, pages=80, max_len=160, f=f, seed=3)):
        waiting = requests(plain, np.random.default_rng(5), LENGTHS)
        order = list(waiting)
        finished = serve(server, waiting)
        assert len(finished) == len(LENGTHS) and sorted(server.free) == list(range(80))
        served.append([x.tokens for x in order])
        drafts = {a: b for a, b in getattr(server, "followers", {}).items()}
    for a, b in zip(*served):
        assert a == b
    assert drafts and (server.made >= server.steps > 0)
    if nodes > 1:
        assert server.made > server.steps                        # some drafts were right


@gpu
def test_sampled_speculation_runs():
    ex = example("speculative_serving")
    server = ex.Speculative(12, 3, 0.8, batch=3, pages=60, max_len=160, f=FORMATS["mx16"], seed=4)
    waiting = requests(ex, np.random.default_rng(6), LENGTHS)
    finished = serve(server, waiting)
    assert sorted(len(x.tokens) for x in finished) == sorted(n + m + 1 for n, m in LENGTHS) and sorted(server.free) == list(range(60))
    with pytest.raises(ValueError):
        server.admit([ex.Request([1] * 150, 20)])


class Loop:
    """One speculative step on fixed buffers, of trees of up to `nodes` nodes: what a graph holds."""

    def __init__(self, f, dtype, B=3, nodes=12, heads=2, group=2, dim=64, page=16, vocab=999, draft=True, spaces=None):
        self.B, self.nodes, self.page, self.T = B, nodes, page, B * nodes
        self.cache = mx.Cache(40, page, heads, dim, f, DEV)
        self.table = torch.full((B, 10), -1, dtype=torch.int32, device=DEV)
        self.ctx, self.new = ints([0] * B), ints([nodes] * B)
        self.free = torch.arange(40, dtype=torch.int32, device=DEV)
        self.parents, self.ids = ints([-1] * self.T), ints([0] * self.T)
        self.q = torch.zeros((self.T, heads * group * dim), device=DEV, dtype=dtype)
        self.k, self.v = (torch.zeros((self.T, heads * dim), device=DEV, dtype=dtype) for _ in range(2))
        self.logits = torch.zeros((self.T, vocab), device=DEV)
        self.draft = torch.zeros((self.T, vocab), device=DEV) if draft else None
        self.temperature, self.uniform = torch.ones(B, device=DEV), torch.zeros(self.T, device=DEV)
        self.noise = torch.ones((B, vocab), device=DEV)
        self.spaces = spaces or (mx.cache_tree_workspace(self.cache.c, self.T, B, heads * group, nodes, 160, DEV),
                                 mx.verify_workspace(self.T, B, vocab, DEV))

    def step(self):
        q_start, kv_len, slots, _, _ = mx.cache_plan(self.ctx, self.new, self.page, self.free, self.table, self.T)
        masks, positions = mx.tree_plan(self.parents, q_start, self.ctx, 1)
        mx.cache_append(self.cache, self.k, self.v, slots)
        o = mx.cache_tree_attention(self.cache, self.q, self.table, q_start, kv_len, masks, self.nodes, 160, None, self.spaces[0])
        path, kept, following = mx.verify(self.logits, self.ids, self.parents, q_start, self.temperature, self.uniform, self.noise, 6,
                                          self.draft, self.spaces[1])
        mx.cache_move(self.cache, self.table, self.ctx, path, kept)
        return masks, positions, o, path, kept, following

    def state(self):
        return [t for t in (self.cache.k, self.cache.v, self.cache.k_exps, self.cache.v_exps, self.table) if t is not None]

    def fill(self, seed, ctx):
        g, r = torch.Generator(DEV).manual_seed(seed), np.random.default_rng(seed)
        for t in (self.q, self.k, self.v, self.logits, self.draft):
            if t is not None:
                t.copy_(torch.randn(t.shape, generator=g, device=DEV) * (4.0 if t is self.logits or t is self.draft else 1.0))
        self.uniform.copy_(torch.rand(self.T, generator=g, device=DEV))
        self.noise.exponential_(generator=g).clamp_(min=1e-30)
        sizes = [int(n) for n in r.integers(0, self.nodes + 1, self.B)]
        parents = [p for n in sizes for p in random_parents(r, n, 3)[:n]]
        self.parents.copy_(ints(parents + [-1] * (self.T - len(parents))))
        self.new.copy_(ints(sizes))
        self.ctx.fill_(ctx)
        near = (self.logits if self.draft is None else self.draft).topk(3).indices
        rows = [sum(sizes[:b]) + max(p, 0) for b, n in enumerate(sizes) for p in parents[sum(sizes[:b]):sum(sizes[:b + 1])]]
        self.ids.zero_()
        if rows:
            self.ids[:len(rows)] = near[torch.tensor(rows, device=DEV), torch.from_numpy(r.integers(0, 3, len(rows))).to(DEV)].int()
        have = -(-ctx // self.page)
        self.table.fill_(-1)
        if have:
            self.table[:, :have] = torch.arange(self.B * have, dtype=torch.int32, device=DEV).reshape(self.B, have)
        self.free.copy_(torch.arange(40, dtype=torch.int32, device=DEV).roll(-self.B * have))
        return sizes, parents


@gpu
@pytest.mark.parametrize("f", [None, FORMATS["mx16"]])
@pytest.mark.parametrize("draft", [False, True])
def test_two_graphs_on_one_workspace(f, draft):
    """Two captured steps of different sizes that share their workspaces, replayed in turn on new inputs, against eager steps."""
    big = Loop(f, torch.float32, draft=draft)
    small = Loop(f, torch.bfloat16, B=2, nodes=5, vocab=64, draft=draft, spaces=big.spaces)
    loops, graphs, outs = (big, small), [], []
    for x in loops:
        x.fill(1, 0)
        x.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(x.step())
        graphs.append(g)
    for at in range(12):
        for x, g, out in zip(loops, graphs, outs):
            x.fill(100 + at, 7 * at % 120)
            before = [t.clone() for t in x.state()]
            g.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in list(out) + x.state()]
            for t, b in zip(x.state(), before):
                t.copy_(b)
            again = list(x.step()) + x.state()
            torch.cuda.synchronize()
            live = int(x.new.sum())
            for n, (a, b) in enumerate(zip(got, again)):
                assert torch.equal(a[:live], b[:live]) if n == 2 else torch.equal(a, b), (at, n)
    assert not big.spaces[0][:65536].any()


@gpu
@pytest.mark.parametrize("draft", [False, True])
def test_a_step_against_plain_ones(draft):
    """Outputs, path and moved rows of steps against the definitions in 64 bits."""
    x = Loop(None, torch.float32, nodes=20, vocab=300, draft=draft)
    for seed, ctx in ((1, 0), (2, 16), (3, 61), (4, 100)):
        sizes, parents = x.fill(seed, ctx)
        x.cache.k.view(torch.bfloat16).normal_()
        x.cache.v.view(torch.bfloat16).normal_()
        old = [t.view(torch.bfloat16).reshape(40, 2, 16, 64).double().cpu() for t in (x.cache.k, x.cache.v)]
        masks, positions, o, path, kept, following = (t.cpu() for t in x.step())
        new = [t.view(torch.bfloat16).reshape(40, 2, 16, 64).double().cpu() for t in (x.cache.k, x.cache.v)]
        table, t0 = x.table.cpu().long(), 0
        for b, n in enumerate(sizes):
            at = torch.arange(ctx + n)
            place = table[b, at // 16], at % 16
            rows = [w[place[0], :, place[1]] for w in old]           # [ctx + n, heads, dim], the new ones to come
            for w, src in zip(rows, (x.k, x.v)):
                w[ctx:] = src[t0:t0 + n].to(torch.bfloat16).double().cpu().reshape(n, 2, 64)
            for i in range(n):
                line, node = [], i
                while node >= 0:
                    line.append(node)
                    node = parents[t0 + node]
                assert int(positions[t0 + i]) == ctx + len(line) - 1
                assert int(masks[t0 + i, 0]) == sum(1 << j for j in line)
                seen = torch.tensor(list(range(ctx)) + [ctx + j for j in line])
                for a in range(4):
                    s = rows[0][seen, a // 2] @ x.q[t0 + i, a * 64:(a + 1) * 64].double().cpu() / 8.0
                    want = torch.softmax(s, 0) @ rows[1][seen, a // 2]
                    # fp32 throughout, as in test_cache.Step.reference; |s| <= |q||k| / 8 < 200, |v| < 6: 2 * 2^-24 * 76 * 200 * 6 < 0.011
                    assert (o[t0 + i, a * 64:(a + 1) * 64].double() - want).abs().max() <= 2 * 2.0 ** -24 * (76 * 200 + len(seen) + 64) * 6
            rng = slice(t0, t0 + n)
            got = walk(x.logits[rng].double().cpu().numpy(), None if x.draft is None else x.draft[rng].double().cpu().numpy(),
                       x.ids[rng].tolist(), parents[rng], 1.0, x.uniform[rng].double().cpu().numpy(), x.noise[b].double().cpu().numpy(), 6)
            if got[2]:
                assert path[b, :int(kept[b])].tolist() == got[0] and int(following[b]) == got[1]
            for k, node in enumerate(path[b, :int(kept[b])].tolist()):
                for w, row in zip(new, rows):
                    assert torch.equal(w[table[b, (ctx + k) // 16], :, (ctx + k) % 16], row[ctx + node])
            t0 += n


@gpu
@pytest.mark.parametrize("draft", [False, True])
def test_the_walks_of_steps_are_decided_and_right(draft):
    """Paths, their lengths, the rest of their rows and the tokens after them against 64 bits, in steps whose decisions stand clear of their borders."""
    x, unsure, steps = Loop(None, torch.float32, B=5, nodes=16, vocab=300, draft=draft), 0, 12
    for seed in range(steps):
        sizes, parents = x.fill(60 + seed, 16 * (seed % 4))
        _, _, _, path, kept, following = (t.cpu() for t in x.step())
        t0 = 0
        for b, n in enumerate(sizes):
            rng = slice(t0, t0 + n)
            want, token, sure = walk(x.logits[rng].double().cpu().numpy(), None if x.draft is None else x.draft[rng].double().cpu().numpy(),
                                     x.ids[rng].tolist(), parents[rng], 1.0, x.uniform[rng].double().cpu().numpy(),
                                     x.noise[b].double().cpu().numpy(), 6)
            t0 += n
            if not sure:
                unsure += 1
                continue
            assert int(kept[b]) == len(want) and path[b].tolist() == want + [-1] * (6 - len(want)) and int(following[b]) == token
    assert unsure <= 2, unsure                                   # of 60 walks
