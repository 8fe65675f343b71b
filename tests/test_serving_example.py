"""The serving example over the paged cache: pools that run short, requests that cannot be served, sizes of its workspace."""
import importlib.util
import os

import numpy as np
import pytest

from paper_2307_15517_amd import mx

gpu = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    return ex


def serve(ex, server, waiting, steps=400):
    finished = []
    for _ in range(steps):
        server.admit(waiting)
        if all(x is None for x in server.places):
            break
        finished += server.step()
    return finished


@gpu
@pytest.mark.parametrize("batch,pages,max_len,chunk", [(8, 10, 160, 48), (8, 12, 160, 16), (4, 25, 160, 48), (3, 1, 16, 5)])
def test_a_pool_smaller_than_all_places(batch, pages, max_len, chunk):
    """More places than the pool can fill at once: requests wait, none runs out of pages on its way."""
    ex, r = example(), np.random.default_rng(batch + pages)
    lengths = [int(r.integers(1, min(max_len, 16 * pages) - 9)) if pages > 1 else 7 for _ in range(9)]
    waiting = [ex.Request(r.integers(0, ex.VOCAB, n), 9) for n in lengths]
    server = ex.Server(batch=batch, pages=pages, page=16, max_len=max_len, chunk=chunk, f=mx.fmt(32, 8))
    finished = serve(ex, server, waiting)
    assert not waiting and sorted(len(x.tokens) for x in finished) == sorted(n + 10 for n in lengths)
    assert sorted(server.free) == list(range(pages))


@gpu
@pytest.mark.parametrize("batch,max_len,chunk", [(2, 4096, 4), (3, 2000, 3), (1, 1000, 300)])
def test_steps_of_few_tokens_on_the_workspace_of_the_largest(batch, max_len, chunk):
    """Steps whose keys are split more often than the largest step's; outputs against those on a workspace of their own."""
    ex, r = example(), np.random.default_rng(batch)
    server = ex.Server(batch=batch, pages=-(-max_len // 16) * batch, page=16, max_len=max_len, chunk=chunk, f=mx.fmt(32, 8))
    waiting = [ex.Request(r.integers(0, ex.VOCAB, n), 3) for n in (3 * chunk, 2 * chunk + 1, 2, 1)]
    while True:
        server.admit(waiting)
        if all(x is None for x in server.places):
            break
        server.step()
        q, o, q_start, kv_len = server.last
        again = mx.cache_attention(server.cache, q, server.table, q_start, kv_len, int((q_start[1:] - q_start[:-1]).max()), max_len)
        assert bool((again == o).all())
    assert not server.workspace[:65536].any()


@gpu
def test_requests_that_cannot_be_served_are_refused():
    ex = example()
    server = ex.Server(batch=2, pages=4, page=16, max_len=60, chunk=16, f=mx.fmt(32, 8))
    for prompt, answer in (([1] * 60, 1), ([1] * 40, 25), ([], 3)):
        waiting = [ex.Request([1, 2, 3], 2), ex.Request(prompt, answer)]
        with pytest.raises(ValueError):
            server.admit(waiting)
        assert len(waiting) == 2 and server.places == [None, None] and len(server.free) == 4
    server = ex.Server(batch=2, pages=2, page=16, max_len=60, chunk=16, f=mx.fmt(32, 8))
    with pytest.raises(ValueError):
        server.admit([ex.Request([1] * 30, 3)])
