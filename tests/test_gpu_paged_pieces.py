"""What a CTA of the paged prefill attention hands from one piece of work to the next."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests.test_gpu_paged import BF, FP, ints, pages, randn
from tests.test_gpu_paged_prefill import check, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype, opt", [(BF, {}), (FP, dict(scale=0.2)), (BF, dict(window=90)), (FP, dict(cap=30.0))])
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


@pytest.mark.parametrize("hq", [8, 24])                     # query groups of 1 and 3 (tiles of 128 and of 126 rows)
@pytest.mark.parametrize("opt", [dict(cap=30.0), dict(cap=30.0, slopes=True), dict(cap=30.0, window=20), dict(cap=30.0, prefix=True)])
def test_capped_results_do_not_depend_on_what_nobody_sees(opt, hq):
    """The same call to the bit, whatever stands behind a sequence's last token, in the rows behind the last query, and in
    shared memory from the call before: the tanh of a score is taken in one of three forms, chosen by the scores that are seen."""
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = 2.0 ** (-torch.arange(1, hq + 1, device="cuda").float() / 4)
    if opt.pop("prefix", False):
        opt["prefix_len"] = ints([12, 30])
    lengths = [40, 70]
    c = pages(lengths, 8, 16, FP, 111)
    cu, options = starts(lengths), mq.make_attn_options(**opt)
    q = randn(190, hq, 128, dtype=FP, seed=112)              # 80 rows behind the last query
    before = pages([1500] * 4, 8, 16, FP, 113)
    q_before, cu_before = randn(1600, hq, 128, dtype=FP, seed=114), starts([400] * 4)
    want = None
    for rest in (0.0, 3e4, float("nan")):
        for x in (before.k_pages, before.v_pages):
            x.normal_().mul_(1.0 if rest == 0.0 else 100.0)
        for b, n in enumerate(lengths):
            last = int(c.block_table[b, n // 16])
            c.k_pages[last, :, n % 16:] = rest
        q[110:] = rest
        out = torch.full_like(q, 7.0)
        mq.moqae_paged_prefill_attn(before, q_before, cu_before, torch.empty_like(q_before), None, options if opt.get("prefix_len") is None else mq.make_attn_options(cap=30.0))
        mq.moqae_paged_prefill_attn(c, q, cu, out, None, options)
        if want is None:
            check(c, q, cu, out, **opt)
            want = out
        assert torch.equal(out, want), f"{rest}: {int((out != want).sum())} values differ"


def test_a_workspace_for_the_largest_call_serves_the_smaller_ones():
    """Prompts, pieces, few rows and single tokens with one buffer that was sized once, for the most tokens and sequences."""
    shapes = [([5000], [0]), ([512], [3000]), ([900] * 5, [10] * 5), ([3, 1, 0], [700, 9, 50]), ([1] * 5, [40, 3000, 7, 0, 333]), ([17], [9000])]
    most = pages([5000] + [0] * 4, 8, 16, BF, 121)
    ws = torch.zeros(mq.moqae_paged_prefill_attn_workspace(most, 32, 5000), dtype=torch.uint8, device="cuda")
    for new, past in shapes:
        c = pages([a + b for a, b in zip(new, past)], 8, 16, BF, 122)
        cu, q = starts(new), randn(sum(new), 32, 128, dtype=BF, seed=123)
        out = torch.full_like(q, 7.0)
        mq.moqae_paged_prefill_attn(c, q, cu, out, ws)
        check(c, q, cu, out)
        if set(new) == {1}:
            one = torch.empty_like(q)
            mq.moqae_paged_decode_attn(c, q, one, ws)
            check(c, q, cu, one)
    assert (ws[:1 << 20] == 0).all()
