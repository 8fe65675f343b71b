"""The workspace of attention over the paged cache: one made for a batch serves every smaller batch."""
import itertools
import random

import pytest
import torch

from paper_2307_15517_amd import mx
from test_cache import DEV, FORMATS, Step

gpu = pytest.mark.gpu


def size(heads, group, dim, tokens, requests, max_new, max_len):
    return mx.mx_cache_attention_workspace_bytes(mx.cache_format(4, 16, heads, dim), tokens, requests, heads * group, max_new, max_len)


def test_smaller_batches_need_no_more():
    steps = ([1, 2, 4, 12, 48, 64, 300, 2000, 4096, 8192, 36000], [1, 2, 3, 8, 16, 64, 255, 700, 4096],
             [1, 2, 3, 4, 15, 17, 48, 500, 1024, 4096], [1, 64, 128, 129, 1936, 4096, 4097, 8192, 100003, 1 << 20, 1 << 33])
    for heads, group, dim in ((1, 1, 64), (4, 3, 64), (8, 4, 128), (12, 1, 64), (32, 1, 128), (2, 16, 16)):
        found = {at: size(heads, group, dim, *(s[i] for s, i in zip(steps, at)))
                 for at in itertools.product(*(range(len(s)) for s in steps))}
        for at, n in found.items():
            for axis in range(4):
                if at[axis]:
                    less = at[:axis] + (at[axis] - 1,) + at[axis + 1:]
                    assert found[less] <= n, (heads, group, dim, less, at)
        assert 65536 <= min(found.values()) and max(found.values()) < 600e6


def test_sizes_that_grew_when_the_batch_shrank():
    # two requests of three and one new tokens against a bound of four; a server's largest step against its smaller ones
    assert size(4, 3, 64, 4, 2, 3, 4096) <= size(4, 3, 64, 8, 2, 4, 4096)
    large = size(8, 4, 128, 8192, 16, 512, 8192)
    assert size(8, 4, 128, 2000, 16, 500, 8192) <= large and size(8, 4, 128, 64, 16, 48, 8192) <= large
    assert size(8, 4, 128, 8, 8, 1, 2048) <= size(8, 4, 128, 64, 64, 1, 2048)


def test_sizes_at_random():
    r = random.Random(5)
    for _ in range(20000):
        heads, group, dim = r.randint(1, 40), r.randint(1, 20), 16 * r.randint(1, 8)
        top = [int(2 ** r.uniform(0, e)) for e in (18, 13, 14, 21)]
        less = [r.choice([v, r.randint(1, v)]) for v in top]
        assert size(heads, group, dim, *less) <= size(heads, group, dim, *top), (heads, group, dim, less, top)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,group,dim", [(4, 3, 64), (8, 4, 128), (2, 2, 96)])
def test_one_workspace_for_all_steps(dtype, heads, group, dim):
    """Steps of many kinds on the workspace of the largest, with a guard behind it that none of them may touch."""
    most = (700, 12, 300, 6000)
    need = size(heads, group, dim, *most)
    guard = 64 << 20
    space = torch.zeros(need + guard, dtype=torch.uint8, device=DEV)
    space[need:] = 0xA5
    for lens in ([(1, 5000)], [(3, 4096), (1, 4090)], [(1, 900)] * 8, [(2, 700)] * 12, [(4, 300), (1, 6000), (30, 31)], [(300, 2000)],
                 [(1, 1)], [(9, 5000), (17, 5000)], [(290, 6000), (300, 310), (100, 5000)], [(40, 50)] * 12, [(60, 60), (0, 9), (5, 2)]):
        step = Step(lens, heads, group, dim, 16, FORMATS["mx32"], dtype, seed=len(lens) + lens[0][0])
        for max_new, max_len in ((step.max_new, step.max_len), (300, 6000)):
            assert step.tokens <= most[0] and len(lens) <= most[1] and max_new <= most[2] and max_len <= most[3]
            step.check(workspace=space[:need], max_new=max_new, max_len=max_len)
        assert bool((space[need:] == 0xA5).all()) and not space[:65536].any()


@gpu
def test_a_workspace_that_does_not_fit_is_refused():
    step = Step([(1, 5000), (20, 300)], 4, 3, 64, 16, FORMATS["mx32"], torch.float32, seed=3)
    need = size(4, 3, 64, step.tokens, 2, step.max_new, step.max_len)
    whole = torch.zeros(2 * need, dtype=torch.uint8, device=DEV)
    for bad in (whole[:need - 1], whole[:65536], whole[::2], torch.zeros(need, dtype=torch.uint8), whole[:0]):
        with pytest.raises(mx.MxError) as e:
            step.run(workspace=bad)
        assert e.value.status == mx.MX_ERR_BAD_ARG
    step.check(workspace=whole[:need])
    step.check(workspace=torch.zeros(need // 4 + 1, dtype=torch.int32, device=DEV))
    with pytest.raises(mx.MxError):                          # enough for its own numbers, not for larger bounds
        step.run(workspace=whole[:need], max_new=1000, max_len=50000)
