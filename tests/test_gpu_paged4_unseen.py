"""Paged 4-bit cache on the GPU: tokens that no query sees may hold anything, and their pages may have been given back, whichever kernel reads
the sequence."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .test_gpu_paged4 import DTYPES, generator, make_cache, randn, space

pytestmark = pytest.mark.gpu


def hide(cache, b, first, last):
    """Tokens first .. last - 1 of sequence b: all bytes 0xff (scales and zeros are NaN); pages that hold nothing else leave the table."""
    page = cache.pages.shape[2] // 160
    key, key_s, value, value_s = ref.places("cuda")
    for entry in range(first // page, (last + page - 1) // page):
        p, at = int(cache.block_table[b, entry]), entry * page
        for tile in range(page // 16):
            t = torch.arange(16, device="cuda") + at + 16 * tile
            t = ((t >= first) & (t < last)).nonzero().flatten()
            gone = torch.zeros(2560, dtype=torch.bool, device="cuda")
            for x in (key, key_s, key_s + 1, key_s + 8, key_s + 9, value, value_s, value_s + 1, value_s + 16, value_s + 17):
                gone[x[t].flatten()] = True
            cache.pages[p, :, 2560 * tile:2560 * tile + 2560].masked_fill_(gone, 255)
        if at >= first and at + page <= last:
            cache.block_table[b, entry] = -1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decode_reads_only_what_is_seen(dtype, page):
    gen = generator(page)
    cache = make_cache(gen, [1000, 70], 2, page, dtype)
    q, opt = randn(gen, 2, 8, 128, dtype=dtype), mq.make_attn_options(window=100, prefix_len=torch.tensor([10, 0], dtype=torch.int32, device="cuda"))
    want, out, work = torch.empty_like(q), torch.empty_like(q), space(mq.moqae_paged4_decode_attn_workspace(cache, 8))
    mq.moqae_paged4_decode_attn(cache, q, want, work, opt)
    hide(cache, 0, 10, 900)
    mq.moqae_paged4_decode_attn(cache, q, out, work, opt)
    assert torch.equal(out, want) and mq.moqae_paged_poll_status(cache) == mq.OK


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("new", [[50, 3], [5, 2], [200, 40]], ids=lambda x: str(x[0]))
def test_prompts_read_only_what_is_seen(dtype, page, new):
    """50 and 200 tokens of a group of four go to the large tiles, the others to the streaming kernel; blocks expanded in the workspace, inside the
    tiles (no room), and some of each."""
    gen = generator(page + new[0])
    lens = [4000, 700]
    cache = make_cache(gen, lens, 2, page, dtype)
    n = sum(new)
    q, cu = randn(gen, n, 8, 128, dtype=dtype), torch.tensor([0, new[0], n], dtype=torch.int32, device="cuda")
    opt = mq.make_attn_options(window=300, prefix_len=torch.tensor([20, 0], dtype=torch.int32, device="cuda"))
    full, least = (mq.moqae_paged4_prefill_attn_workspace(cache, 8, n, least=x) for x in (False, True))
    want, out = torch.empty_like(q), torch.empty_like(q)
    mq.moqae_paged4_prefill_attn(cache, q, cu, want, space(full), opt)
    for b in range(2):
        hide(cache, b, 20 if b == 0 else 0, lens[b] - new[b] - 299)       # up to the first token that the first query sees
    for size in (full, least, (full + least) // 2):
        out.fill_(3.0)
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(size), opt)
        assert torch.equal(out, want), size
        assert mq.moqae_paged_poll_status(cache) == mq.OK, (size, cache.status.tolist())


def test_a_seen_page_that_does_not_exist_is_still_reported():
    """Beside pages that were given back, one that some query sees: it is the one that the status names."""
    gen = generator(5)
    cache = make_cache(gen, [4000], 2, 16, torch.float16)
    q, cu = randn(gen, 50, 8, 128, dtype=torch.float16), torch.tensor([0, 50], dtype=torch.int32, device="cuda")
    opt = mq.make_attn_options(window=300)
    hide(cache, 0, 0, 4000 - 50 - 299)
    cache.block_table[0, 240] = -1
    out = torch.empty_like(q)
    for least in (False, True):
        cache.status.zero_()
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, 8, 50, least=least)), opt)
        assert cache.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, 0, 240] and torch.isfinite(out.float()).all()
