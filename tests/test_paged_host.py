"""Paged 16-bit cache without a GPU: the table validator and the refusals of the entry points, all of which
are decided on the host before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from paper_2506_07533_b200 import build as mqbuild

A = 1 << 20                      # a 16-byte aligned address that no refused call may follow


@pytest.fixture(scope="module")
def lib():
    mqbuild.build()
    return mq.lib()


def cache(**kw):
    c = mq.MoqaePagedCache(A, A, (C.c_int64 * 3)(2 * 16 * 128, 16 * 128, 128), (C.c_int64 * 3)(2 * 16 * 128, 16 * 128, 128), A, A, A,
                           10, 16, 2, mq.DT_BF16, 3, 5)
    for name, value in kw.items():
        setattr(c, name, (C.c_int64 * 3)(*value) if name.endswith("stride") else value)
    return c


def rows(heads, **kw):
    r = mq.MoqaeRows(A, heads * 128, 128, heads)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def rope(**kw):
    r = mq.MoqaeRope(A, A, A, 100, 128, 0, 1e-6)
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
    (dict(max_pages=(1 << 26) + 1), mq.ERR_UNSUPPORTED),                 # more than 2^30 tokens
    (dict(k_stride=(4096, 0, 128)), mq.ERR_INVALID_ARG), (dict(v_stride=(4096, 2048, -128)), mq.ERR_INVALID_ARG),
    (dict(k_stride=(4096, 2048, 132)), mq.ERR_MISALIGNED), (dict(v_stride=(4100, 2048, 128)), mq.ERR_MISALIGNED),
    (dict(k_pages=None), mq.ERR_INVALID_ARG), (dict(v_pages=A + 2), mq.ERR_MISALIGNED), (dict(block_table=None), mq.ERR_INVALID_ARG),
    (dict(kv_len=None), mq.ERR_INVALID_ARG), (dict(kv_len=A + 2), mq.ERR_MISALIGNED), (dict(status=A + 4), mq.ERR_MISALIGNED),
]


@pytest.mark.parametrize("change, code", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(lib, change, code):
    c, n = C.byref(cache(**change)), C.c_int64(0)
    q, k = C.byref(rows(8)), C.byref(rows(2))
    assert lib.moqae_paged_append(c, None, k, k, None, None, A, A, 3, None) == code
    assert lib.moqae_paged_decode_attn(c, q, q, None, A, 1 << 40, None) == code
    assert lib.moqae_paged_prefill_attn(c, q, A, 3, q, None, None, 0, None) == code
    assert lib.moqae_paged_decode_attn_workspace(c, 8, C.byref(n)) == code
    assert lib.moqae_paged_prefill_attn_workspace(c, 8, 3, C.byref(n)) == code


def test_missing_arguments(lib):
    c, n = C.byref(cache()), C.c_int64(0)
    q, k = C.byref(rows(8)), C.byref(rows(2))
    bad = mq.ERR_INVALID_ARG
    assert lib.moqae_paged_append(None, None, k, k, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged_append(c, None, None, k, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged_append(c, None, k, None, None, None, A, A, 3, None) == bad
    assert lib.moqae_paged_append(c, None, k, k, q, None, A, A, 3, None) == bad
    assert lib.moqae_paged_append(c, None, k, k, None, None, None, A, 3, None) == bad
    assert lib.moqae_paged_append(c, None, k, k, None, None, A, A, -1, None) == bad
    assert lib.moqae_paged_append(c, None, q, k, None, None, A, A, 3, None) == bad            # 8 key heads, 2 in the cache
    assert lib.moqae_paged_append(c, None, k, k, q, k, A, A, 3, None) == bad                  # queries into fewer heads
    assert lib.moqae_paged_append(c, None, k, k, None, None, A + 2, A, 3, None) == mq.ERR_MISALIGNED
    assert lib.moqae_paged_decode_attn(None, q, q, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged_decode_attn(c, None, q, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged_decode_attn(c, q, None, None, A, 1 << 40, None) == bad
    assert lib.moqae_paged_decode_attn(c, q, q, None, None, 1 << 40, None) == bad
    assert lib.moqae_paged_decode_attn(c, q, q, None, A + 8, 1 << 40, None) == mq.ERR_MISALIGNED
    assert lib.moqae_paged_decode_attn_workspace(c, 8, C.byref(n)) == mq.OK and n.value > 0
    assert lib.moqae_paged_decode_attn(c, q, q, None, A, n.value - 1, None) == mq.ERR_WORKSPACE_TOO_SMALL
    assert lib.moqae_paged_decode_attn_workspace(c, 8, None) == bad
    many = C.byref(cache(batch=(1 << 17) + 1))
    assert lib.moqae_paged_decode_attn_workspace(many, 8, C.byref(n)) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged_decode_attn(many, q, q, None, A, 1 << 40, None) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged_prefill_attn(c, q, None, 3, q, None, None, 0, None) == bad
    assert lib.moqae_paged_prefill_attn(c, q, A, -3, q, None, None, 0, None) == bad
    assert lib.moqae_paged_prefill_attn(c, q, A, 3, k, None, None, 0, None) == bad
    assert lib.moqae_paged_prefill_attn_workspace(c, 8, -1, C.byref(n)) == bad
    assert lib.moqae_paged_prefill_attn_workspace(c, 8, (1 << 24) + 1, C.byref(n)) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged_prefill_attn(c, q, A, (1 << 24) + 1, q, None, None, 0, None) == mq.ERR_UNSUPPORTED
    assert lib.moqae_paged_prefill_attn_workspace(c, 8, 3, C.byref(n)) == mq.OK and n.value > 0
    assert lib.moqae_paged_prefill_attn(c, q, A, 3, q, None, A, n.value - 1, None) == mq.ERR_WORKSPACE_TOO_SMALL
    assert lib.moqae_paged_poll_status(None, None, None) == bad


@pytest.mark.parametrize("batch, heads, max_pages, page, code", [
    (1 << 18, 1, 1, 16, mq.OK), ((1 << 18) + 1, 1, 1, 16, mq.ERR_UNSUPPORTED), (1 << 14, 1, 8192 * 16 - 3, 16, mq.OK),
    (1 << 14, 1, 8192 * 16, 16, mq.ERR_UNSUPPORTED), (1 << 5, 1, 1 << 22, 256, mq.ERR_UNSUPPORTED), (31, 1, 1 << 22, 256, mq.OK),
    (4, 8, 1 << 22, 256, mq.ERR_UNSUPPORTED), (3, 8, 1 << 22, 256, mq.OK)])
def test_decode_sizes_that_its_counters_hold(lib, batch, heads, max_pages, page, code):
    assert (batch * heads * (max_pages * page // 16 + 2) < 1 << 31 and batch * heads <= 1 << 18) == (code == mq.OK)
    n = C.c_int64(0)
    c = cache(batch=batch, n_kv_heads=heads, max_pages=max_pages, page_size=page)
    assert lib.moqae_paged_decode_attn_workspace(C.byref(c), heads, C.byref(n)) == code
    if code != mq.OK:
        q = C.byref(rows(heads))
        assert lib.moqae_paged_decode_attn(C.byref(c), q, q, None, A, 1 << 40, None) == code


@pytest.mark.parametrize("heads, code", [(0, mq.ERR_INVALID_ARG), (-8, mq.ERR_INVALID_ARG), (7, mq.ERR_INVALID_ARG),
                                         (18, mq.ERR_UNSUPPORTED), (32, mq.ERR_UNSUPPORTED)])
def test_head_counts(lib, heads, code):
    n = C.c_int64(0)
    q = C.byref(rows(heads))
    assert lib.moqae_paged_decode_attn_workspace(C.byref(cache()), heads, C.byref(n)) == code
    assert lib.moqae_paged_decode_attn(C.byref(cache()), q, q, None, A, 1 << 40, None) == code
    assert lib.moqae_paged_prefill_attn(C.byref(cache()), q, A, 3, q, None, None, 0, None) == code


@pytest.mark.parametrize("change, code", [
    (dict(data=None), mq.ERR_INVALID_ARG), (dict(data=A + 8), mq.ERR_MISALIGNED), (dict(token_stride=1028), mq.ERR_MISALIGNED),
    (dict(head_stride=-128), mq.ERR_INVALID_ARG), (dict(head_stride=64), mq.ERR_INVALID_ARG), (dict(token_stride=0), mq.ERR_INVALID_ARG)])
def test_output_rows(lib, change, code):
    q, bad = C.byref(rows(8)), C.byref(rows(8, **change))
    assert lib.moqae_paged_decode_attn(C.byref(cache()), q, bad, None, A, 1 << 40, None) == code
    assert lib.moqae_paged_prefill_attn(C.byref(cache()), q, A, 3, bad, None, None, 0, None) == code
    assert lib.moqae_norm_rope(C.byref(rope()), 1, q, None, bad, None, A, 3, None, None) == code
    assert lib.moqae_paged_append(C.byref(cache()), None, C.byref(rows(2)), C.byref(rows(2)), q, bad, A, None, 3, None) == code


@pytest.mark.parametrize("change, code", [
    (dict(rot_dim=-16), mq.ERR_INVALID_ARG), (dict(rot_dim=144), mq.ERR_INVALID_ARG), (dict(rot_dim=72), mq.ERR_UNSUPPORTED),
    (dict(interleaved=2), mq.ERR_INVALID_ARG), (dict(cos_sin=None), mq.ERR_INVALID_ARG), (dict(cos_sin=A + 4), mq.ERR_MISALIGNED),
    (dict(n_positions=-1), mq.ERR_INVALID_ARG), (dict(eps=-1.0), mq.ERR_INVALID_ARG), (dict(eps=float("nan")), mq.ERR_INVALID_ARG),
    (dict(q_weight=A + 2), mq.ERR_MISALIGNED), (dict(k_weight=A + 8), mq.ERR_MISALIGNED)])
def test_rope_arguments(lib, change, code):
    r, q, k = C.byref(rope(**change)), C.byref(rows(8)), C.byref(rows(2))
    assert lib.moqae_norm_rope(r, 1, q, k, q, k, A, 3, None, None) == code
    assert lib.moqae_paged_append(C.byref(cache()), r, k, k, None, None, A, A, 3, None) == code


def test_norm_rope_arguments(lib):
    r, q, k = C.byref(rope()), C.byref(rows(8)), C.byref(rows(2))
    bad = mq.ERR_INVALID_ARG
    assert lib.moqae_norm_rope(None, 1, q, k, q, k, A, 3, None, None) == bad
    assert lib.moqae_norm_rope(r, 2, q, k, q, k, A, 3, None, None) == mq.ERR_UNSUPPORTED
    assert lib.moqae_norm_rope(r, 1, q, k, q, None, A, 3, None, None) == bad
    assert lib.moqae_norm_rope(r, 1, None, None, None, None, A, 3, None, None) == bad
    assert lib.moqae_norm_rope(r, 1, q, k, k, q, A, 3, None, None) == bad
    assert lib.moqae_norm_rope(r, 1, q, k, q, k, None, 3, None, None) == bad
    assert lib.moqae_norm_rope(r, 1, q, k, q, k, A, -1, None, None) == bad
    assert lib.moqae_norm_rope(r, 1, q, k, q, k, A, 3, A + 4, None) == mq.ERR_MISALIGNED


@pytest.mark.parametrize("change, code", [
    (dict(cap=-1.0), mq.ERR_INVALID_ARG), (dict(cap=1e-5), mq.ERR_UNSUPPORTED), (dict(cap=float("inf")), mq.ERR_INVALID_ARG), (dict(cap=float("nan")), mq.ERR_INVALID_ARG),
    (dict(scale=float("nan")), mq.ERR_INVALID_ARG), (dict(scale=float("inf")), mq.ERR_INVALID_ARG), (dict(window=-1), mq.ERR_INVALID_ARG),
    (dict(slopes=A + 2), mq.ERR_MISALIGNED), (dict(prefix_len=A + 1), mq.ERR_MISALIGNED)])
def test_attention_options(lib, change, code):
    o, q = C.byref(options(**change)), C.byref(rows(8))
    assert lib.moqae_paged_decode_attn(C.byref(cache()), q, q, o, A, 1 << 40, None) == code
    assert lib.moqae_paged_prefill_attn(C.byref(cache()), q, A, 3, q, o, None, 0, None) == code


def test_table_validator_on_host_arrays(lib):
    rng = np.random.RandomState(0)
    table = rng.randint(0, 50, size=(4, 7)).astype(np.int32)
    length = np.array([0, 1, 16 * 7, 33], np.int32)
    ok = (mq.OK, -1, -1)
    assert mq.moqae_paged_validate_host(table, length, 50, 16) == ok
    spare = table.copy()
    spare[0, :] = -1                       # entries behind the last used page may hold anything
    spare[1, 1:] = 99
    spare[3, 3:] = -7
    assert mq.moqae_paged_validate_host(spare, length, 50, 16) == ok
    for b, i, page in ((1, 0, -1), (2, 6, 50), (3, 2, 1 << 30)):
        bad = table.copy()
        bad[b, i] = page
        assert mq.moqae_paged_validate_host(bad, length, 50, 16) == (mq.ERR_CORRUPT_TABLE, b, i)
    for n in (-1, 16 * 7 + 1):
        bad = length.copy()
        bad[2] = n
        assert mq.moqae_paged_validate_host(table, bad, 50, 16) == (mq.ERR_CORRUPT_TABLE, 2, -1)
    assert mq.moqae_paged_validate_host(np.zeros((0, 0)), np.zeros(0), 0, 16) == ok
    assert mq.moqae_paged_validate_host(table, length, 50, 0)[0] == mq.ERR_INVALID_ARG


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):
    """The library only takes device memory; a host tensor is refused before any pointer is passed on."""
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    table, length = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(mq.MoqaeError) as e:
        mq.moqae_paged_bind(k, k, table, length)
    assert e.value.code == mq.ERR_INVALID_ARG
    with pytest.raises(mq.MoqaeError):
        mq.make_rope(torch.zeros(10, 128), 128)
    with pytest.raises(mq.MoqaeError):
        mq.make_rope(None, 64)
    with pytest.raises(mq.MoqaeError):
        mq.moqae_norm_rope(mq.make_rope(None, 0), torch.zeros(3, 8, 128, dtype=torch.float16), None, torch.zeros(3, dtype=torch.int32))


def test_rope_table():
    t = mq.rope_table(5, 64, device="cpu")
    assert t.shape == (5, 64) and t.dtype == torch.float32
    i = torch.arange(32, dtype=torch.float64)
    a = 4 * 10000.0 ** (-2 * i / 64)
    assert torch.equal(t[4], torch.cat([a.cos(), a.sin()]).float()) and torch.equal(t[0], torch.tensor([1.0] * 32 + [0.0] * 32))
