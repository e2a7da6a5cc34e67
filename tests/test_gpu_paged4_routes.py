"""Paged 4-bit cache on the GPU: which kernel takes a sequence goes by its own rows, not by the mean of the batch."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from .test_gpu_paged4 import DTYPES, check, generator, make_cache, randn, space

pytestmark = pytest.mark.gpu


def attend(cache, q, cu, **kw):
    out = torch.full_like(q, 9.0)
    mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, q.shape[1], q.shape[0], **kw)))
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq, hkv, piece", [(2, 2, 256), (4, 1, 64)])
def test_a_piece_of_a_prompt_beside_single_tokens(dtype, hq, hkv, piece):
    """256 rows behind 3000 tokens beside 31 sequences of one new token: on average few rows each, but the piece fills a tile.  The large tiles and the
    streaming kernel round differently, so the piece has the bits that it has alone exactly where the same kernel takes it.  (One full row tile: the
    blocks are shared out alike.)"""
    gen = generator(hq)
    past, new = [40 + 3 * b for b in range(15)] + [3000] + [200 - b for b in range(16)], [1] * 15 + [piece] + [1] * 16
    cache = make_cache(gen, [a + b for a, b in zip(past, new)], hkv, 16, dtype)
    n = sum(new)
    q, cu = randn(gen, n, hq, 128, dtype=dtype), torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    out = attend(cache, q, cu)
    check(cache, q, new, out, None, None)
    one = mq.moqae_paged4_bind(cache.pages, cache.block_table[15:16], cache.kv_len[15:16], dtype)
    alone = attend(one, q[15:15 + piece].contiguous(), torch.tensor([0, piece], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[15:15 + piece], alone)
    assert cache.status[0].item() == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_bound_on_the_new_tokens_changes_no_result(dtype):
    """Even batches with a bound that holds; an uneven one with a bound that does not: the kernels may change, the results stay within their error."""
    gen = generator(3)
    for new in ([4] * 40, [24, 3] * 9, [1] * 20 + [200] + [2] * 20):
        cache = make_cache(gen, [300 + 5 * b + n for b, n in enumerate(new)], 2, 16, dtype)
        n = sum(new)
        q, cu = randn(gen, n, 8, 128, dtype=dtype), torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
        work = space(mq.moqae_paged4_prefill_attn_workspace(cache, 8, n))
        for bound in (0, 24, 200, 1 << 40):
            out = torch.full_like(q, 9.0)
            mq.moqae_paged4_prefill_attn(cache, q, cu, out, work, mq.make_attn_options(max_new=bound))
            check(cache, q, new, out, None, None, what=f"bound {bound}")
        assert cache.status[0].item() == 0 and (work[:1 << 20] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_row_tile_beside_many_single_tokens_is_cut(dtype):
    """256 rows behind 3000 tokens beside 600 single tokens: the long walk is cut into pieces as it is alone, which its bits show."""
    gen = generator(4)
    past, new = [10 + b % 50 for b in range(300)] + [3000] + [20 + b % 40 for b in range(300)], [1] * 300 + [64] + [1] * 300
    cache = make_cache(gen, [a + b for a, b in zip(past, new)], 1, 16, dtype)
    n = sum(new)
    q, cu = randn(gen, n, 4, 128, dtype=dtype), torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    out = attend(cache, q, cu)
    check(cache, q, new, out, None, None)
    one = mq.moqae_paged4_bind(cache.pages, cache.block_table[300:301], cache.kv_len[300:301], dtype)
    assert torch.equal(out[300:364], attend(one, q[300:364].contiguous(), torch.tensor([0, 64], dtype=torch.int32, device="cuda")))
