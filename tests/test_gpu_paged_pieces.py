"""What a CTA of the paged prefill attention hands from one piece of work to the next."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests.test_gpu_paged import BF, FP, pages, randn
from tests.test_gpu_paged_prefill import check, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype, opt", [(BF, {}), (FP, dict(scale=0.2)), (BF, dict(window=90))])
def test_full_row_tiles_followed_by_tiles_without_work(dtype, opt, workspace):
    """More uncut pieces than SMs, full ones (256 rows) beside ends of 44 rows (the second tile has none), sequences whose first
    tile sees nothing (more queries than tokens) and sequences without tokens: a warp with nothing to do for its
    tile goes on to the next piece while its partner may still be sending out rows of the last one."""
    new, past = [300, 256, 256, 40] * 15, [0, -156, 0, -40] * 15
    c = pages([max(0, a + b) for a, b in zip(new, past)], 8, 16, dtype, 101)
    cu, n = starts(new), sum(new)
    q = randn(n, 8, 128, dtype=dtype, seed=102)
    options = mq.make_attn_options(**opt)
    ws = torch.zeros(mq.moqae_paged_prefill_attn_workspace(c, 8, n), dtype=torch.uint8, device="cuda") if workspace else None
    want = None
    for _ in range(40):
        out = torch.full((n, 8, 128), 7.0, dtype=dtype, device="cuda")
        mq.moqae_paged_prefill_attn(c, q, cu, out, ws, options)
        if want is None:
            check(c, q, cu, out, **opt)
            want = out
        assert torch.equal(out, want)
    assert mq.moqae_paged_poll_status(c) == 0
