"""Attention over the paged cache of bfloat16 activations at the ends of its range and where P V cancels, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2307_15517_amd import mx
from test_cache import CHUNKS, DEV, FEW, FORMATS, Step

gpu = pytest.mark.gpu
LENS = FEW + CHUNKS + [(1, 3000)]


def rewritten(step, change):
    """The step with its keys and values ([2][cached token][heads][dim]) changed in place and stored again."""
    kv = step.kv.clone()
    change(kv.view(2, -1, step.heads, step.dim))
    mx.cache_append(step.cache, kv[0], kv[1], torch.from_numpy(step.slots.astype(np.int32)).to(DEV))
    return step


def close(step, scale=None):
    """As Step.check, but with what bfloat16 calls do round: the result, to 8 bits, and in tiles of many rows a probability, whose
    two pieces leave 2^-16 of it at most (a bfloat16 rounding each).  Step's own bound takes 2^-9 for a probability."""
    got = step.run(scale).double().cpu().numpy()
    want, wide = step.reference(scale)
    step.dtype = torch.float32
    fine = step.reference(scale)[1]                             # of fp32 scores, statistics and sums
    step.dtype = torch.bfloat16
    size = 2.0 ** 9 * (wide - fine - 2.0 ** -8 * np.abs(want))  # sum p|v|
    tol = fine + 2.0 ** -16 * size
    tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    at = np.unravel_index((np.abs(got - want) - tol).argmax(), got.shape)
    assert (np.abs(got - want) <= tol).all(), (at, got[at], want[at], tol[at])


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
@pytest.mark.parametrize("power", [-100, -75, -69, -66, -62, -59, -30, 60, 79, 90, 110])
def test_values_of_any_size(kind, power):
    """Keys of ordinary size, values about 2^power."""
    def change(kv):
        kv[1] *= 2.0 ** power
    rewritten(Step(LENS, 2, 2, 64, 16, FORMATS[kind], torch.bfloat16, seed=31), change).check()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
@pytest.mark.parametrize("down", [12, 25, 28, 32, 37, 45, 80])
def test_values_far_below_others_of_their_keys(kind, down):
    """Half the channels 2^-down of the others: in MXInt, blocks of far exponents next to each other."""
    def change(kv):
        kv[1, ..., 32:] *= 2.0 ** -down
    rewritten(Step(LENS, 2, 2, 64, 32, FORMATS[kind], torch.bfloat16, seed=32), change).check()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("up", [26, 40, 70, 100])
def test_later_tokens_do_not_change_what_earlier_ones_give(kind, dim, up):
    """Whole prompts whose last token has values of 2^up: the rows before it do not see it, and keep all their bits."""
    lens = [(100, 100), (33, 64), (250, 250), (40, 48)]
    ends = (np.cumsum([m for _, m in lens]) - 1).tolist()

    def change(kv):
        kv[1, ends] *= 2.0 ** up
    rewritten(Step(lens, 1, 2, dim, 16, FORMATS[kind], torch.bfloat16, seed=33), change).check()


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
def test_a_run_of_keys_far_below_the_next(kind):
    """Sixteen keys with small values between sixteen with large ones, and keys that draw most of the weight with values of zero."""
    def change(kv):
        place = torch.arange(kv.shape[1], device=DEV)
        kv[1, place // 16 % 2 == 0] *= 2.0 ** -35
        kv[0, place % 64 == 5] *= 3.0
        kv[1, place % 64 == 5] = 0.0
    rewritten(Step(LENS, 2, 2, 64, 16, FORMATS[kind], torch.bfloat16, seed=34), change).check()
    rewritten(Step(LENS, 1, 2, 128, 16, FORMATS[kind], torch.bfloat16, seed=34), change).check(1.0)


@gpu
@pytest.mark.parametrize("lens,group", [([(1, 64)], 2), ([(1, 64)], 32), ([(40, 104)], 1), ([(1, 200)], 24)])
def test_probabilities_keep_their_bits_where_the_products_cancel(lens, group):
    """The last visible key's values are what makes P V nearly zero, so that rounding the result hides nothing.  Small scores and a
    head dimension of 16 keep the fp32 part of the bound near 2^-15 of sum p|v|; probabilities of 8 bits miss it several times."""
    n, m = lens[0]
    step = Step(lens, 1, group, 16, 16, None, torch.bfloat16, seed=35)
    step.q[:] = step.q[:1, :16].repeat(1, group) * 0.25          # every row the same: their weights differ by what they see only
    x = step.q[0, :16].double().cpu().numpy() @ step.values()[0][:, 0].T * 0.25

    def change(kv):
        p = np.exp(x - x.max())
        v = kv[1, :, 0].to(torch.bfloat16).double().cpu().numpy()
        seen = m - n + 1                                         # of the first row
        v[seen - 1] = -(p[:seen - 1, None] * v[:seen - 1]).sum(0) / p[seen - 1]
        for later in range(seen, m):
            v[later] = 0.0
        kv[1, :, 0] = torch.from_numpy(v).to(DEV).float()
    close(rewritten(step, change))


@gpu
@pytest.mark.parametrize("kind", ["bf16", "mx16", "mx32"])
def test_bfloat16_calls_within_their_own_roundings(kind):
    close(Step(LENS, 2, 2, 64, 16, FORMATS[kind], torch.bfloat16, seed=36))
    close(Step(LENS, 1, 4, 128, 32, FORMATS[kind], torch.bfloat16, seed=37))
    close(Step([(1, 5), (2, 3)], 1, 4, 128, 32, FORMATS[kind], torch.bfloat16, seed=38))
