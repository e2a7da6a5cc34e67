"""Paged 4-bit cache without a GPU: the sizes that its documentation allows, and the next ones."""
import ctypes as C

import pytest

from paper_2506_07533_b200 import binding as mq

from .test_paged4_host import cache, lib  # noqa: F401


@pytest.mark.parametrize("page, max_pages, batch, heads, code", [
    (16, 1 << 14, 1 << 12, 32, mq.ERR_UNSUPPORTED),           # 2^17 * (2^18 + 64): above
    (16, (1 << 14) - 4, 1 << 12, 32, mq.ERR_UNSUPPORTED),     # 2^17 * 2^18 = 2^35: not below
    (16, (1 << 14) - 5, 1 << 12, 32, mq.OK),
    (256, (1 << 10) - 1, 1 << 12, 32, mq.OK),
    (16, 4, 1 << 13, 32, mq.OK),                              # 2^18 pairs
    (16, 4, (1 << 13) + 1, 32, mq.ERR_UNSUPPORTED)])
def test_one_token_calls_at_the_limits(lib, page, max_pages, batch, heads, code):  # noqa: F811
    c = cache(page_size=page, max_pages=max_pages, batch=batch, n_kv_heads=heads, head_stride=160 * page, page_stride=160 * page * heads)
    n = C.c_int64(0)
    assert lib.moqae_paged4_decode_attn_workspace(C.byref(c), heads, C.byref(n)) == code
