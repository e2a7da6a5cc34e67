"""Paged caches on the GPU: one row tile of one kv head over a long context is cut into pieces whatever else the batch holds."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from .test_gpu_paged4 import DTYPES, check, generator, make_cache, randn, space

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits, batch", [(4, 2), (4, 4), (4, 5), (4, 40), (16, 2), (16, 4), (16, 5)])
def test_a_lone_row_tile_is_cut_as_it_is_alone(dtype, batch, bits):
    """256 rows over a long context; the others bring nothing.  (4-bit pages: so long that the streaming kernel does not take them.)  A cut tile adds up its pieces, one that is walked by a single CTA does not, so the bits show
    which it was."""
    gen = generator(batch)
    piece, past, hq = 64, 33000 if bits == 4 else 3000, 4
    q = randn(gen, piece, hq, 128, dtype=dtype)
    if bits == 4:
        cache = make_cache(gen, [past + piece] + [40] * (batch - 1), 1, 16, dtype)
        one = mq.moqae_paged4_bind(cache.pages, cache.block_table[:1].contiguous(), cache.kv_len[:1], dtype)
        size, attend = mq.moqae_paged4_prefill_attn_workspace, mq.moqae_paged4_prefill_attn
    else:
        pages = [randn(gen, 200, 1, 16, 128, dtype=dtype) for _ in range(2)]
        table, lens = torch.arange(200, dtype=torch.int32, device="cuda").repeat(batch, 1), torch.full((batch,), past + piece, dtype=torch.int32, device="cuda")
        cache, one = mq.moqae_paged_bind(*pages, table, lens), mq.moqae_paged_bind(*pages, table[:1], lens[:1])
        size, attend = mq.moqae_paged_prefill_attn_workspace, mq.moqae_paged_prefill_attn
    got, alone = torch.empty_like(q), torch.empty_like(q)
    attend(cache, q, torch.tensor([0] + [piece] * batch, dtype=torch.int32, device="cuda"), got, space(size(cache, hq, piece)))
    attend(one, q, torch.tensor([0, piece], dtype=torch.int32, device="cuda"), alone, space(size(one, hq, piece)))
    if bits == 4:
        check(cache, q, [piece] + [0] * (batch - 1), got, None, None)
    assert torch.equal(got, alone) and cache.status[0].item() == 0
