"""Where calls of several tokens change over from the streaming kernel (sets of 16 rows) to the large tiles, and uneven
batches that the mean number of rows sends to the streaming kernel."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests.test_gpu_paged import BF, FP, ints, pages, randn
from tests.test_gpu_paged_prefill import check, prefill, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("group", [1, 2, 3, 5, 6, 7, 8])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_calls_around_the_change(dtype, group, more):
    """The most tokens that the streaming kernel takes, one fewer and one more, in one long sequence beside short ones: sets that
    end inside a token, sequences of many sets, pieces that span sets and CTAs."""
    batch, hkv = 6, 2
    n = 16 * batch // group + more
    new = [n - 7, 1, 0, 2, 3, 1]
    past = [9000, 30, 500, 0, 1700, 64]
    c = pages([a + b for a, b in zip(new, past)], hkv, 16, dtype, 131)
    cu, q = starts(new), randn(n, hkv * group, 128, dtype=dtype, seed=132)
    for opt in (dict(), dict(window=700, prefix_len=ints([40, 0, 9, 1, 2000, 5])), dict(cap=20.0)):
        for workspace in (False, True):
            check(c, q, cu, prefill(c, q, cu, workspace, **opt), **opt)
    assert mq.moqae_paged_poll_status(c) == 0


@pytest.mark.parametrize("new, past, hq, hkv", [([1] * 60 + [900], [40] * 60 + [4000], 4, 4), ([1] * 63 + [190], [300] * 63 + [8000], 32, 8),
                                                ([190] + [1] * 63, [8000] + [2000] * 63, 8, 2), ([0] * 30 + [90] + [0] * 30, [9] * 61, 10, 2)])
def test_one_long_sequence_beside_single_tokens(new, past, hq, hkv):
    c = pages([a + b for a, b in zip(new, past)], hkv, 16, BF, 141)
    cu, n = starts(new), sum(new)
    assert n * (hq // hkv) <= 16 * len(new)                   # the streaming kernel takes it
    q = randn(n, hq, 128, dtype=BF, seed=142)
    for workspace in (False, True):
        check(c, q, cu, prefill(c, q, cu, workspace))
