"""Block tables and slots at the ends of 32 bits."""
import pytest
import torch

from paper_2307_15517_amd import mx
from test_cache import DEV, ints, run_plan

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_page_indices_whose_slots_pass_32_bits_give_none(page):
    """The largest page with slots below 2^31, the next, those that would come out at page 0 and 1 again, and negative ones; taken
    from the free list (three tokens of a new request) and from the table (the next token of an old one)."""
    last = (1 << 31) // page - 1
    for entry in (last, last + 1, 2 * last + 1, 2 * last + 2, 2 * last + 3, 2 ** 31 - 1, -1, -2 ** 31):
        if not -2 ** 31 <= entry < 2 ** 31:
            continue
        table, _, kv_len, slots, positions, _ = run_plan([0, 5], [3, 1], page, [entry], [[-1], [entry]], 4)
        assert table == [[entry], [entry]] and kv_len == [3, 6] and positions == [0, 1, 2, 5]
        assert slots == ([entry * page + i for i in (0, 1, 2, 5)] if 0 <= entry <= last else [-1] * 4), entry


@gpu
def test_positions_past_32_bits_stay_at_the_last():
    """A request whose new tokens take it past 2^31 positions, in a table row wide enough for them."""
    page, have = 16, (1 << 27) - 1                           # pages of the 2^31 - 20 cached tokens
    table = torch.full((1, have + 4), 7, dtype=torch.int32, device=DEV)
    q_start, kv_len, slots, positions, counts = mx.cache_plan(ints([2 ** 31 - 20]), ints([40]), page, ints([1, 2, 3, 4]), table, 40)
    at = [2 ** 31 - 20 + i for i in range(40)]
    pages = [7 if p // page < have else 1 + p // page - have for p in at]
    assert positions.tolist() == [min(p, 2 ** 31 - 1) for p in at] and kv_len.tolist() == [2 ** 31 - 1]
    assert slots.tolist() == [e * page + p % page for e, p in zip(pages, at)]
    assert counts.tolist() == [3, 0] and table[0, have - 1:].tolist() == [7, 1, 2, 3, 7]


@gpu
def test_a_step_without_requests_clears_more_tokens_than_a_launch_has_workgroups():
    cache = mx.Cache(1, 16, 1, 16, None, DEV)
    none = ints([])
    for tokens in (70001, (1 << 24) + 5):
        q = torch.zeros((tokens, 16), dtype=torch.bfloat16, device=DEV)
        out = torch.ones((tokens, 24), dtype=torch.bfloat16, device=DEV)
        mx.cache_attention(cache, q, none.reshape(0, 1), ints([0]), none, 1, 1, out=out[:, :16])
        assert not out[:, :16].any() and bool((out[:, 16:] == 1.0).all())
