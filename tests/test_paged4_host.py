"""Paged 4-bit cache and plans without a GPU: the refusals of the entry points, all of which are decided on the host
before anything is launched."""
import ctypes as C

import pytest

from paper_2506_07533_b200 import binding as mq
from paper_2506_07533_b200 import build as mqbuild

A = 1 << 20                      # a 16-byte aligned address that no refused call may follow


@pytest.fixture(scope="module")
def lib():
    mqbuild.build()
    return mq.lib()


def cache(**kw):
    c = mq.MoqaePaged4Cache(A, 2 * 2560, 2560, A, A, A, 10, 16, 2, mq.DT_BF16, 3, 5)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def rows(heads, **kw):
    r = mq.MoqaeRows(A, heads * 128, 128, heads)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def options(**kw):
    o = mq.MoqaeAttnOptions(None, None, 0.0, 0.0, 0)
    for name, value in kw.items():
        setattr(o, name, value)
    return o


BAD_CACHES = [
    (dict(dtype=2), mq.ERR_UNSUPPORTED), (dict(page_size=24), mq.ERR_UNSUPPORTED), (dict(page_size=8), mq.ERR_UNSUPPORTED),
    (dict(page_size=512), mq.ERR_UNSUPPORTED), (dict(page_size=0), mq.ERR_UNSUPPORTED), (dict(n_pages=-1), mq.ERR_INVALID_ARG),
    (dict(n_kv_heads=0), mq.ERR_INVALID_ARG), (dict(batch=-1), mq.ERR_INVALID_ARG), (dict(max_pages=-1), mq.ERR_INVALID_ARG),
    (dict(max_pages=(1 << 26) + 1), mq.ERR_UNSUPPORTED), (dict(page_stride=0), mq.ERR_INVALID_ARG), (dict(head_stride=-16), mq.ERR_INVALID_ARG),
    (dict(page_stride=5128), mq.ERR_MISALIGNED), (dict(head_stride=2568), mq.ERR_MISALIGNED), (dict(head_stride=2544), mq.ERR_INVALID_ARG),
    (dict(page_stride=2544), mq.ERR_INVALID_ARG), (dict(page_size=32), mq.ERR_INVALID_ARG),       # pages that would lie in one another
    (dict(pages=None), mq.ERR_INVALID_ARG), (dict(pages=A + 8), mq.ERR_MISALIGNED), (dict(block_table=None), mq.ERR_INVALID_ARG),
    (dict(kv_len=None), mq.ERR_INVALID_ARG), (dict(kv_len=A + 2), mq.ERR_MISALIGNED), (dict(status=A + 4), mq.ERR_MISALIGNED),
]


@pytest.mark.parametrize("change, code", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(lib, change, code):
    c, n = C.byref(cache(**change)), C.c_int64(0)
    q, k = C.byref(rows(8)), C.byref(rows(2))
    assert lib.moqae_paged4_append(c, None, k, k, None, None, A, A, 3, None) == code
    assert lib.moqae_paged4_read(c, k, k, A, A, 3, None) == code
    assert lib.moqae_paged4_decode_attn(c, q, q, None, A, 1 << 40, None) == code
    assert lib.moqae_paged4_prefill_attn(c, q, A, 3, q, None, A, 1 << 40, None) == code
    assert lib.moqae_paged4_decode_attn_workspace(c, 8, C.byref(n)) == code
    assert lib.moqae_paged4_prefill_attn_workspace(c, 8, 3, C.byref(n), None) == code


def test_missing_arguments(lib):
    c, n = C.byref(cache()), C.c_int64(0)
    q, k = C.byref(rows(8)), C.byref(rows(2))
    bad = mq.ERR_INVALID_ARG
    assert lib.moqae_paged4_append(None, None, k, k, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged4_append(c, None, None, k, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged4_append(c, None, k, None, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged4_append(c, None, k, k, q, None, A, A, 3, None) == bad
    assert lib.moqae_paged4_append(c, None, k, k, None, None, None, A, 3, None) == bad
    assert lib.moqae_paged4_append(c, None, k, k, None, None, A, A, -1, None) == bad
    assert lib.moqae_paged4_append(c, None, q, k, None, None, A, A, 3, None) == bad             # head counts
    assert lib.moqae_paged4_read(c, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged4_read(c, k, q, A, A, 3, None) == bad
    assert lib.moqae_paged4_read(c, k, k, None, A, 3, None) == bad
    assert lib.moqae_paged4_read(c, C.byref(rows(2, token_stride=0)), k, A, A, 3, None) == bad   # output rows in one another
    assert lib.moqae_paged4_read(c, k, k, A + 1, A, 3, None) == mq.ERR_MISALIGNED
    assert lib.moqae_paged4_decode_attn(c, None, q, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged4_decode_attn(c, q, None, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged4_decode_attn(c, q, q, None, None, 1 << 40, None) == bad
    assert lib.moqae_paged4_decode_attn(c, q, q, None, A + 8, 1 << 40, None) == mq.ERR_MISALIGNED
    assert lib.moqae_paged4_decode_attn(c, q, q, None, A, (1 << 20) - 1, None) == mq.ERR_WORKSPACE_TOO_SMALL
    assert lib.moqae_paged4_prefill_attn(c, q, None, 3, q, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged4_prefill_attn(c, q, A, 3, q, None, None, 1 << 40, None) == bad
    assert lib.moqae_paged4_prefill_attn(c, q, A, -1, q, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged4_prefill_attn(c, q, A, (1 << 24) + 1, q, None, A, 1 << 40, None) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged4_prefill_attn(c, q, A, 3, q, None, A, (1 << 20) - 1, None) == mq.ERR_WORKSPACE_TOO_SMALL
    assert lib.moqae_paged4_decode_attn_workspace(c, 8, None) == bad
    assert lib.moqae_paged4_decode_attn_workspace(c, 3, C.byref(n)) == bad
    assert lib.moqae_paged4_decode_attn_workspace(c, 18, C.byref(n)) == mq.ERR_UNSUPPORTED       # groups of nine
    assert lib.moqae_paged4_decode_attn(c, q, C.byref(rows(4)), None, A, 1 << 40, None) == bad


@pytest.mark.parametrize("change, code", [
    (dict(scale=float("nan")), mq.ERR_INVALID_ARG), (dict(cap=-1.0), mq.ERR_INVALID_ARG), (dict(cap=1e-5), mq.ERR_UNSUPPORTED),
    (dict(window=-1), mq.ERR_INVALID_ARG), (dict(slopes=A + 1), mq.ERR_MISALIGNED), (dict(prefix_len=A + 2), mq.ERR_MISALIGNED)])
def test_bad_options(lib, change, code):
    c, q, o = C.byref(cache()), C.byref(rows(8)), C.byref(options(**change))
    assert lib.moqae_paged4_decode_attn(c, q, q, o, A, 1 << 40, None) == code
    assert lib.moqae_paged4_prefill_attn(c, q, A, 3, q, o, A, 1 << 40, None) == code


def test_batches_that_the_counters_cannot_hold(lib):
    n = C.c_int64(0)
    assert lib.moqae_paged4_decode_attn_workspace(C.byref(cache(batch=1 << 18)), 8, C.byref(n)) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged4_decode_attn_workspace(C.byref(cache(batch=100000, max_pages=60000)), 8, C.byref(n)) == mq.ERR_UNSUPPORTED


def test_workspaces_serve_every_smaller_call(lib):
    def sizes(batch, tokens, heads=8, **kw):
        n, low = C.c_int64(0), C.c_int64(0)
        assert lib.moqae_paged4_prefill_attn_workspace(C.byref(cache(batch=batch, **kw)), heads, tokens, C.byref(n), C.byref(low)) == 0
        one = C.c_int64(0)
        assert lib.moqae_paged4_decode_attn_workspace(C.byref(cache(batch=batch, **kw)), heads, C.byref(one)) == 0
        assert (1 << 20) < one.value <= low.value <= n.value
        return low.value, n.value
    for kw in (dict(), dict(max_pages=8192), dict(n_kv_heads=1, page_stride=2560), dict(max_pages=0)):
        shape = [(b, t) for b in (1, 2, 3, 40, 300) for t in (1, 2, 15, 64, 300, 5000, 40000)]
        got = {s: sizes(*s, **kw) for s in shape}
        for b, t in shape:
            for c, u in shape:
                if c >= b and u >= t:
                    assert got[c, u][0] >= got[b, t][0] and got[c, u][1] >= got[b, t][1], (b, t, c, u)
    assert sizes(1000, 8, max_pages=8192)[1] - sizes(1000, 8, max_pages=8192)[0] <= 1 << 30
    n = C.c_int64(0)
    assert lib.moqae_paged4_prefill_attn_workspace(C.byref(cache()), 8, 3, None, None) == mq.ERR_INVALID_ARG
    assert lib.moqae_paged4_prefill_attn_workspace(C.byref(cache()), 8, -1, C.byref(n), None) == mq.ERR_INVALID_ARG


def plan(lib, **kw):
    a = dict(past=A, n_new=A, batch=3, page=16, width=5, table=A, kv_len=A, ring=A, state=A, n_pages=10, before=None, cu=A, pos=A, seq=A,
             rows=7, status=A, pool=True)
    a.update(kw)
    pool = C.byref(mq.MoqaePagePool(a["ring"], a["state"], a["n_pages"])) if a["pool"] else None
    return lib.moqae_paged_plan(a["past"], a["n_new"], a["batch"], a["page"], a["width"], a["table"], a["kv_len"], pool, a["before"], a["cu"],
                                a["pos"], a["seq"], a["rows"], a["status"], None)


@pytest.mark.parametrize("change, code", [
    (dict(pool=False), mq.ERR_INVALID_ARG), (dict(batch=-1), mq.ERR_INVALID_ARG), (dict(width=-1), mq.ERR_INVALID_ARG),
    (dict(rows=-1), mq.ERR_INVALID_ARG), (dict(n_pages=-1), mq.ERR_INVALID_ARG), (dict(page=24), mq.ERR_UNSUPPORTED),
    (dict(page=512), mq.ERR_UNSUPPORTED), (dict(page=0), mq.ERR_UNSUPPORTED), (dict(width=(1 << 26) + 1), mq.ERR_UNSUPPORTED),
    (dict(rows=(1 << 24) + 1), mq.ERR_UNSUPPORTED), (dict(batch=(1 << 24) + 1), mq.ERR_UNSUPPORTED), (dict(n_pages=(1 << 24) + 1), mq.ERR_UNSUPPORTED),
    (dict(past=None), mq.ERR_INVALID_ARG), (dict(n_new=None), mq.ERR_INVALID_ARG), (dict(table=None), mq.ERR_INVALID_ARG),
    (dict(kv_len=None), mq.ERR_INVALID_ARG), (dict(ring=None), mq.ERR_INVALID_ARG), (dict(state=None), mq.ERR_INVALID_ARG),
    (dict(cu=None), mq.ERR_INVALID_ARG), (dict(pos=None), mq.ERR_INVALID_ARG), (dict(seq=None), mq.ERR_INVALID_ARG),
    (dict(past=A + 1), mq.ERR_MISALIGNED), (dict(n_new=A + 2), mq.ERR_MISALIGNED), (dict(table=A + 3), mq.ERR_MISALIGNED),
    (dict(kv_len=A + 1), mq.ERR_MISALIGNED), (dict(ring=A + 2), mq.ERR_MISALIGNED), (dict(state=A + 4), mq.ERR_MISALIGNED),
    (dict(before=A + 2), mq.ERR_MISALIGNED), (dict(cu=A + 1), mq.ERR_MISALIGNED), (dict(pos=A + 1), mq.ERR_MISALIGNED),
    (dict(seq=A + 1), mq.ERR_MISALIGNED), (dict(status=A + 8), mq.ERR_MISALIGNED)])
def test_bad_plans(lib, change, code):
    assert plan(lib, **change) == code
