"""One attention layer served with continuous batching over a paged MXInt key/value cache.

    python examples/paged_serving.py [--requests 12] [--steps 60] [--page 16] [--cache-block 32]

Requests bring prompts of different lengths, which enter in chunks while the requests before them decode; finished requests hand
their pages back and their places go to the next.  A step is: the fused projection of the packed tokens (MXInt weights), the block
tables (mx.cache_plan), the new keys and values into their pages (mx.cache_append), the attention over the pages
(mx.cache_attention), the output projection.  The weights are random; a request's next token follows from its last output.
"""

from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2307_15517_amd import mx  # noqa: E402

HIDDEN, HEADS_Q, HEADS, DIM, VOCAB = 768, 12, 4, 64, 1000
QKV = (HEADS_Q + 2 * HEADS) * DIM


class Linear:
    """y = x W^T with weights MXInt(32, 8, 3) and activations MXInt(32, 8, 7)."""

    def __init__(self, w: torch.Tensor):
        self.n, self.k = w.shape
        self.fx, self.fw = mx.fmt(32, 8), mx.fmt(32, 4)
        self.w = mx.quantize_pack(w, self.fw, mx.MX_LAYOUT_MATRIX)

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        packed = mx.quantize_pack(x, self.fx, mx.MX_LAYOUT_MATRIX)
        return mx.gemm(packed, self.fx, self.w, self.fw, x.shape[0], self.n, self.k, layout=mx.MX_LAYOUT_MATRIX)[0]


class Request:
    def __init__(self, prompt, answer: int):
        self.tokens = list(prompt)       # the prompt, then what was generated
        self.done = 0                    # tokens in the cache
        self.stop = len(self.tokens) + answer


class Server:
    """Places for ``batch`` requests, their block tables, the cache's pages and the layer's weights."""

    def __init__(self, batch=8, pages=256, page=16, max_len=512, chunk=48, f=None, device="cuda", seed=0):
        g = torch.Generator(device).manual_seed(seed)

        def matrix(rows, cols):
            return torch.randn((rows, cols), generator=g, device=device) * cols ** -0.5
        self.device, self.batch, self.pages, self.page, self.chunk, self.max_len = device, batch, pages, page, chunk, max_len
        self.embedding = torch.randn((VOCAB, HIDDEN), generator=g, device=device)
        self.qkv, self.out = Linear(matrix(QKV, HIDDEN)), Linear(matrix(HIDDEN, HEADS_Q * DIM))
        self.cache = mx.Cache(pages, page, HEADS, DIM, f, device)
        self.width = -(-max_len // page)
        self.table = torch.full((batch, self.width), -1, dtype=torch.int32, device=device)
        self.places = [None] * batch
        self.free = list(range(pages))
        self.owned = [[] for _ in range(batch)]       # the host's own list of the pages that a place holds
        # of the largest step; smaller ones need no more
        self.workspace = mx.cache_workspace(self.cache.c, batch * chunk, batch, HEADS_Q, chunk, max_len, device)

    def _pages_of(self, request):
        """The pages that a request holds at its end."""
        return -(-request.stop // self.page)

    def admit(self, waiting):
        """Gives places to the first that wait, as long as the pages cover what all with a place will hold at their ends."""
        for request in waiting:
            if not request.tokens or request.stop > self.max_len or self._pages_of(request) > self.pages:
                raise ValueError("a request of 1 to %d tokens is wanted" % min(self.max_len, self.pages * self.page))
        lacking = sum(self._pages_of(r) - len(o) for r, o in zip(self.places, self.owned) if r is not None)
        for i in range(self.batch):
            if self.places[i] is None and waiting and lacking + self._pages_of(waiting[0]) <= len(self.free):
                self.places[i] = waiting.pop(0)
                lacking += self._pages_of(self.places[i])

    def step(self):
        """Feeds every request its next chunk or token.  Returns the finished requests."""
        new = [0 if r is None else min(self.chunk, len(r.tokens) - r.done) for r in self.places]
        ctx = [0 if r is None else r.done for r in self.places]
        ids = [t for r, n in zip(self.places, new) if r is not None for t in r.tokens[r.done:r.done + n]]

        def up(v):
            return torch.tensor(v, dtype=torch.int32).to(self.device)
        q_start, kv_len, slots, _, counts = mx.cache_plan(up(ctx), up(new), self.page, up(self.free), self.table, len(ids))
        y = self.qkv(self.embedding[torch.tensor(ids).to(self.device)])
        q, k, v = y[:, :HEADS_Q * DIM], y[:, HEADS_Q * DIM:(HEADS_Q + HEADS) * DIM], y[:, (HEADS_Q + HEADS) * DIM:]
        mx.cache_append(self.cache, k, v, slots)
        o = mx.cache_attention(self.cache, q, self.table, q_start, kv_len, max(new), self.max_len, None, self.workspace)
        self.last = (q, o, q_start, kv_len)                           # for a look at the step from outside
        last = [sum(new[:i + 1]) - 1 for i in range(self.batch) if new[i]]
        answers = iter((self.out(o[last]) @ self.embedding.T).argmax(-1).tolist())
        taken, refused = counts.tolist()
        if refused:
            raise RuntimeError("out of pages")
        done = []
        for i, r in enumerate(self.places):
            if r is None:
                continue
            lacks = -(-(ctx[i] + new[i]) // self.page) - -(-ctx[i] // self.page)
            self.owned[i] += self.free[:lacks]                         # the rule by which the pages were handed out
            del self.free[:lacks]
            taken -= lacks
            r.done += new[i]
            answer = next(answers)
            if r.done == len(r.tokens):
                r.tokens.append(answer)
                if len(r.tokens) > r.stop:
                    done.append(r)
                    self.free += self.owned[i]
                    self.owned[i], self.places[i] = [], None
        assert taken == 0
        return done


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--requests", type=int, default=12)
    p.add_argument("--steps", type=int, default=1000, help="at most")
    p.add_argument("--page", type=int, default=16)
    p.add_argument("--cache-block", type=int, default=32, choices=(0, 16, 32), help="0: bfloat16 cache")
    a = p.parse_args()
    r = np.random.default_rng(0)
    waiting = [Request(r.integers(0, VOCAB, int(r.integers(1, 300))), int(r.integers(1, 60))) for _ in range(a.requests)]
    server = Server(page=a.page, pages=8192 // a.page, f=mx.fmt(a.cache_block, 8) if a.cache_block else None)
    finished = 0
    for step in range(a.steps):
        server.admit(waiting)
        if all(x is None for x in server.places):
            break
        for x in server.step():
            finished += 1
            print("step %d: a request of %d tokens is done, %d pages free" % (step, len(x.tokens), len(server.free)), flush=True)
    print("%d requests finished" % finished)


if __name__ == "__main__":
    main()
