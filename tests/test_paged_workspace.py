"""One workspace for calls of several sizes: what the sizes that the library asks for have to do with one another."""
import ctypes as C

import pytest

from paper_2506_07533_b200 import binding as mq
from paper_2506_07533_b200 import build as mqbuild
from tests.test_paged_host import cache

TOKENS = [0, 1, 2, 4, 5, 15, 16, 17, 40, 128, 129, 300, 512, 1000, 4000, 5000, 16300, 16384, 16385, 40000, 1 << 20, 1 << 24]


def size(batch, heads, group, n):
    out, c = C.c_int64(0), cache(batch=batch, n_kv_heads=heads)
    assert mq.lib().moqae_paged_prefill_attn_workspace(C.byref(c), heads * group, n, C.byref(out)) == mq.OK
    return out.value


@pytest.mark.parametrize("heads, group", [(1, 1), (2, 4), (8, 4), (8, 8), (40, 1), (8, 3), (200, 1), (600, 1)])
def test_a_buffer_for_the_largest_call_serves_the_smaller_ones(heads, group):
    mqbuild.build()
    batches = [1, 2, 3, 8, 64, 65, 70, 500, 5000]
    for i, batch in enumerate(batches):
        sizes = [size(batch, heads, group, n) for n in TOKENS]
        assert sizes == sorted(sizes), (batch, sizes)
        if i:
            assert all(a <= b for a, b in zip(before, sizes)), (batch, before, sizes)
        before = sizes
        one, c = C.c_int64(0), cache(batch=batch, n_kv_heads=heads)
        fits = batch * heads <= 1 << 18                       # (what a call of one token per sequence takes)
        assert mq.lib().moqae_paged_decode_attn_workspace(C.byref(c), heads * group, C.byref(one)) == (mq.OK if fits else mq.ERR_UNSUPPORTED)
        assert one.value <= sizes[0]
