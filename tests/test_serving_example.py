"""The serving example over the paged cache."""
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
