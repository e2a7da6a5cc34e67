"""Paged 4-bit cache on the GPU: which blocks of several-token calls are expanded in the workspace.  Only the blocks that some query sees take room, and a
sequence that finds none leaves it to those behind it."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from .test_gpu_paged4 import DTYPES, check, generator, make_cache, randn, space

pytestmark = pytest.mark.gpu
MARK = 0xA5


def attend(cache, q, cu, opt, blocks):
    """The result with room for `blocks` blocks, and which 16-byte units of that room were written."""
    n, hq = q.shape[0], q.shape[1]
    least = mq.moqae_paged4_prefill_attn_workspace(cache, hq, n, least=True)
    block_bytes = 2 * cache.pages.shape[1] * 128 * 128 * 2
    work = space(least + blocks * block_bytes)
    work[least:] = MARK
    out = torch.full_like(q, 9.0)
    mq.moqae_paged4_prefill_attn(cache, q, cu, out, work, opt)
    assert (work[:1 << 20] == 0).all() and cache.status[0].item() == 0
    return out, (work[least:].view(-1, 16) != MARK).any(1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_blocks_before_the_windows_take_no_room(dtype):
    """20000 tokens, 50 of them new, window of 300 and prefix of 20: block 0, and blocks 153 .. 156.  900 tokens, 40 new: blocks 4 .. 7.  500 tokens of which the prefix and
    the window leave nothing out: 4 blocks."""
    gen = generator(51)
    lens, new = [20000, 900, 500], [50, 40, 30]
    cache, n = make_cache(gen, lens, 2, 16, dtype), sum(new)
    q, cu = randn(gen, n, 8, 128, dtype=dtype), torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    prefix = torch.tensor([20, 0, 250], dtype=torch.int32, device="cuda")
    opt = mq.make_attn_options(window=300, prefix_len=prefix)
    inside, _ = attend(cache, q, cu, opt, 0)
    check(cache, q, new, inside, None, prefix, window=300)
    out, written = attend(cache, q, cu, opt, 13)
    assert written.all() and torch.equal(out, inside)
    out, written = attend(cache, q, cu, opt, 12)             # the last sequence finds no room
    assert torch.equal(out, inside) and not written.all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("before, lens, new", [(0, [6000, 500, 400], [50, 30, 60]), (297, [6000, 500, 400], [50, 30, 60]),
                                               (0, [6000, 500, 380, 250, 500, 120], [30] * 6), (253, [6000, 500, 380, 250, 500, 120], [30] * 6)])
def test_a_sequence_without_room_stops_nobody(dtype, before, lens, new):
    """Eight blocks: 47 do not fit, then 4 and 4 do; or 4 and 3 do, 2 and 4 do not, 1 does; the same behind sequences that bring nothing (which are looked at 256
    at a time)."""
    gen = generator(52 + before)
    lens, new = [0] * before + lens, [0] * before + new
    cache, n = make_cache(gen, lens, 1, 32, dtype), sum(new)
    q, cu = randn(gen, n, 4, 128, dtype=dtype), torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    inside, _ = attend(cache, q, cu, None, 0)
    check(cache, q, new, inside, None, None)
    out, written = attend(cache, q, cu, None, 8)
    assert written.all() and torch.equal(out, inside)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window, prefix, new", [(2500, 0, 200), (2500, 700, 200), (4096, 130, 1500), (127, 128, 129), (129, 1, 700), (6000, 9000, 300)])
def test_long_windows(dtype, window, prefix, new):
    """Windows of thousands of tokens: blocks of the prefix, blocks from the first window on, and the gap between them."""
    gen = generator(window + prefix)
    cache = make_cache(gen, [9000, 150], 2, 64, dtype)
    n = new + 100
    q, cu = randn(gen, n, 4, 128, dtype=dtype), torch.tensor([0, new, n], dtype=torch.int32, device="cuda")
    lens = torch.tensor([prefix, prefix], dtype=torch.int32, device="cuda")
    opt = mq.make_attn_options(window=window, prefix_len=lens)
    inside, _ = attend(cache, q, cu, opt, 0)
    check(cache, q, [new, 100], inside, None, lens, window=window)
    for blocks in (200, 60, 7):
        out, _ = attend(cache, q, cu, opt, blocks)
        assert torch.equal(out, inside), blocks
