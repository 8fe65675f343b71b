"""The serving loop of paged_serving.py with drafted tokens: several tokens of a request in one step.

    python examples/speculative_serving.py [--requests 12] [--nodes 8] [--branch 2] [--temperature 0]

Drafts are looked up: what has followed a token in any request so far is drafted after it, the latest first, as a tree whose node 0
is the token that the step before gave.  A step is: the fused projection of all nodes, block tables and slots (mx.cache_plan), the
trees' masks (mx.tree_plan), keys and values into the pages (mx.cache_append), attention of the trees (mx.cache_tree_attention), the
output projection, the walk down the trees (mx.verify), the accepted rows moved together (mx.cache_move).  At temperature 0
the tokens are those of paged_serving.py.  While a prompt is being read all requests take that program's steps.
"""

from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paged_serving import DIM, HEADS, HEADS_Q, VOCAB, Request, Server, mx  # noqa: E402


class Speculative(Server):
    """A server whose steps check up to ``nodes`` tokens of a request, ``branch`` drafted ones after each."""

    def __init__(self, nodes=8, branch=2, temperature=0.0, max_len=512, batch=8, page=16, seed=0, **kw):
        super().__init__(max_len=max_len + nodes, batch=batch, page=page, seed=seed, **kw)
        self.nodes, self.branch, self.limit = nodes, branch, max_len
        self.temperature = torch.full((batch,), float(temperature), device=self.device)
        self.random = torch.Generator(self.device).manual_seed(seed + 1)
        self.tree_space = mx.cache_tree_workspace(self.cache.c, batch * nodes, batch, HEADS_Q, nodes, max_len + nodes, self.device)
        self.walk_space = mx.verify_workspace(batch * nodes, batch, VOCAB, self.device)
        self.followers = {}              # token -> those that followed it, the latest first
        self.steps = self.made = 0       # speculative steps of a request, tokens that they gave

    def _pages_of(self, request):
        return -(-(request.stop + self.nodes) // self.page)

    def admit(self, waiting):
        for request in waiting:
            if request.stop > self.limit:
                raise ValueError("a request of 1 to %d tokens is wanted" % self.limit)
        super().admit(waiting)

    def _note(self, tokens):
        for a, b in zip(tokens, tokens[1:]):
            row = self.followers.setdefault(a, [])
            if b in row:
                row.remove(b)
            row.insert(0, b)

    def draft(self, request):
        """(tokens, parents) of a request's tree, level by level."""
        ids, parents = [request.tokens[-1]], [-1]
        node = 0
        while node < len(ids) and len(ids) < self.nodes:
            for token in self.followers.get(ids[node], [])[:self.branch]:
                if len(ids) < self.nodes:
                    ids.append(token)
                    parents.append(node)
            node += 1
        return ids, parents

    def step(self):
        if any(r is not None and len(r.tokens) - r.done > 1 for r in self.places):
            done = super().step()
            for r in done + [r for r in self.places if r is not None and len(r.tokens) - r.done == 1]:
                self._note(r.tokens)
            return done
        trees = [([], []) if r is None else self.draft(r) for r in self.places]
        new, ctx = [len(ids) for ids, _ in trees], [0 if r is None else r.done for r in self.places]
        ids, parents = (sum((t[k] for t in trees), []) for k in (0, 1))

        def up(v):
            return torch.tensor(v, dtype=torch.int32).to(self.device)
        ctx_len, tokens = up(ctx), up(ids)
        q_start, kv_len, slots, _, counts = mx.cache_plan(ctx_len, up(new), self.page, up(self.free), self.table, len(ids))
        tree = up(parents)
        masks, _ = mx.tree_plan(tree, q_start, ctx_len, -(-self.nodes // 64))
        y = self.qkv(self.embedding[tokens.long()])
        q, k, v = y[:, :HEADS_Q * DIM], y[:, HEADS_Q * DIM:(HEADS_Q + HEADS) * DIM], y[:, (HEADS_Q + HEADS) * DIM:]
        mx.cache_append(self.cache, k, v, slots)
        o = mx.cache_tree_attention(self.cache, q, self.table, q_start, kv_len, masks, max(new), self.max_len, None, self.tree_space)
        logits = self.out(o) @ self.embedding.T
        uniform = torch.rand(len(ids), generator=self.random, device=self.device)
        noise = torch.empty((self.batch, VOCAB), device=self.device).exponential_(generator=self.random).clamp_(min=1e-30)
        path, kept, following = mx.verify(logits, tokens, tree, q_start, self.temperature, uniform, noise, self.nodes,
                                          workspace=self.walk_space)
        mx.cache_move(self.cache, self.table, ctx_len, path, kept)
        path, kept, following = path.tolist(), kept.tolist(), following.tolist()
        if counts.tolist()[1]:
            raise RuntimeError("out of pages")
        done = []
        for i, r in enumerate(self.places):
            if r is None:
                continue
            lacks = -(-(ctx[i] + new[i]) // self.page) - -(-ctx[i] // self.page)
            self.owned[i] += self.free[:lacks]                         # the rule by which the pages were handed out
            del self.free[:lacks]
            r.done += kept[i]
            r.tokens += [trees[i][0][node] for node in path[i][1:kept[i]]] + [following[i]]
            self.steps += 1
            self.made += kept[i]
            self._note(r.tokens[-kept[i] - 1:])
            if len(r.tokens) > r.stop:
                del r.tokens[r.stop + 1:]
                done.append(r)
                r.done = 0
            spare = 0 if r in done else -(-r.done // self.page)        # pages behind the last token that stays
            self.free += self.owned[i][spare:]
            del self.owned[i][spare:]
            if r in done:
                self.places[i] = None
        return done


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--requests", type=int, default=12)
    p.add_argument("--nodes", type=int, default=8)
    p.add_argument("--branch", type=int, default=2)
    p.add_argument("--temperature", type=float, default=0.0)
    p.add_argument("--cache-block", type=int, default=32, choices=(0, 16, 32), help="0: bfloat16 cache")
    a = p.parse_args()
    r = np.random.default_rng(0)
    waiting = [Request(r.integers(0, VOCAB, int(r.integers(1, 300))).tolist(), int(r.integers(1, 60))) for _ in range(a.requests)]
    server = Speculative(a.nodes, a.branch, a.temperature, pages=512, f=mx.fmt(a.cache_block, 8) if a.cache_block else None)
    finished = 0
    while True:
        server.admit(waiting)
        if all(x is None for x in server.places):
            break
        finished += len(server.step())
    print("%d requests finished, %.2f tokens a speculative step" % (finished, server.made / max(1, server.steps)))


if __name__ == "__main__":
    main()
