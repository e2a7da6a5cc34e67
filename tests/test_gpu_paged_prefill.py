"""Attention of several new tokens per sequence over a paged 16-bit cache, against its definition in 64 bits."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests import paged_reference as R
from tests.test_gpu_paged import BF, FP, decode, ints, pages, randn

pytestmark = pytest.mark.gpu


def prefill(c, q, cu, workspace=True, **opt):
    """The call twice with and without a workspace (which shares the tokens of few queries out); all must agree
    with the definition, calls with the same workspace to the bit."""
    options = mq.make_attn_options(**opt) if opt else None
    ws = torch.zeros(mq.moqae_paged_prefill_attn_workspace(c, q.shape[1], q.shape[0]), dtype=torch.uint8, device="cuda") if workspace else None
    outs = []
    for _ in range(2):
        out = torch.full(tuple(q.shape), 7.0, dtype=q.dtype, device="cuda")
        mq.moqae_paged_prefill_attn(c, q, cu, out, ws, options)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    return outs[0]


def check(c, q, cu, out, what="", heads=None, **opt):
    prefix = opt.pop("prefix_len", None)
    at = cu.tolist()
    for b, total in enumerate(c.kv_len.tolist()):
        n = at[b + 1] - at[b]
        k, v = (R.gather(x, c.block_table[b], total) for x in (c.k_pages, c.v_pages))
        want, tol = R.attention(q[at[b]:at[b + 1]], k, v, total - n, prefix=0 if prefix is None else max(int(prefix[b]), 0), split_weights=False, **opt)
        R.close(out[at[b]:at[b + 1]], want, tol, f"{what} sequence {b}: {n} of {total}")
    assert (out[at[-1]:] == 7.0).all()                        # rows behind the last sequence


def starts(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return ints(cu)


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (8, 2), (6, 2), (7, 1), (8, 1), (3, 3)])
@pytest.mark.parametrize("page, order", [(16, "hsd"), (64, "shd"), (256, "hsd")])
def test_prefill_head_layouts(dtype, hq, hkv, page, order, workspace):
    new, past = [1, 130, 5, 64, 300], [0, 0, 700, 127, 33]
    c = pages([a + b for a, b in zip(new, past)], hkv, page, dtype, hq, order)
    cu = starts(new)
    q = randn(sum(new) + 3, hq, 128, dtype=dtype, seed=5)     # a padded batch
    check(c, q, cu, prefill(c, q, cu, workspace))
    assert mq.moqae_paged_poll_status(c) == 0


@pytest.mark.parametrize("new, past", [([1], [0]), ([1], [5000]), ([2], [131000]), ([127], [1]), ([128], [0]), ([129], [0]), ([257], [255]),
                                       ([1200], [0]), ([512], [9000]), ([0, 3, 0, 0, 9], [4, 0, 0, 50, 0]), ([1] * 40, [77] * 40), ([3, 400] * 20, [2000, 0] * 20)])
def test_prefill_lengths(new, past):
    c = pages([a + b for a, b in zip(new, past)], 2, 32, BF, 21)
    cu = starts(new)
    q = randn(sum(new), 8, 128, dtype=BF, seed=6)
    for workspace in (False, True):
        check(c, q, cu, prefill(c, q, cu, workspace))


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("dtype, hq, hkv", [(BF, 8, 2), (FP, 3, 3)])
@pytest.mark.parametrize("opt", [dict(cap=30.0), dict(cap=0.5), dict(window=1), dict(window=100), dict(window=129, cap=50.0), dict(scale=0.3),
                                 dict(slopes=True), dict(slopes=True, cap=20.0, window=200, prefix=True), dict(prefix=True),
                                 dict(window=64, prefix=True), dict(window=1 << 30)])
def test_prefill_options(dtype, hq, hkv, opt, workspace):
    new, past = [200, 1, 400, 10, 70], [0, 300, 900, 2000, 60]
    c = pages([a + b for a, b in zip(new, past)], hkv, 16, dtype, 31)
    cu = starts(new)
    q = randn(sum(new), hq, 128, dtype=dtype, seed=7)
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = 2.0 ** (-torch.arange(1, hq + 1, device="cuda").float())
    if opt.pop("prefix", False):
        opt["prefix_len"] = ints([150, 64, 1000, -3, 129])
    check(c, q, cu, prefill(c, q, cu, workspace, **opt), **opt)


@pytest.mark.parametrize("cap", [1e-4, 0.01, 1.0, 3.0, 500.0, 1e5, 1e20])
def test_prefill_caps(cap):
    """Caps far below and far above the scores: an all but uniform and an all but plain softmax."""
    c = pages([700, 333], 2, 16, FP, 35)
    cu, q = starts([150, 300]), randn(450, 8, 128, dtype=FP, seed=9, scale=3.0)
    check(c, q, cu, prefill(c, q, cu, cap=cap), cap=cap)


FEW = [dict(), dict(cap=30.0), dict(window=1), dict(window=100), dict(window=33, cap=50.0), dict(scale=0.3), dict(slopes=True), dict(prefix=True),
       dict(slopes=True, cap=20.0, window=60, prefix=True), dict(window=64, prefix=True)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (8, 2), (6, 2), (7, 1), (8, 1), (10, 10)])
@pytest.mark.parametrize("opt", FEW)
def test_prefill_few_rows(dtype, hq, hkv, opt):
    """A few tokens per sequence: one, more than a set of 16 rows holds, none, a sequence that is all new, one with more
    queries than tokens."""
    group = hq // hkv
    new = [1, 2, 40 // group, 0, 5, 16 // group + 1, 3] + [0] * 6
    past = [700, 0, 130, 50, 2000, 15, -2] + [0, 20, 0, 0, 33, 1]
    c = pages([a + b for a, b in zip(new, past)], hkv, 16, dtype, 33)
    cu = starts(new)
    q = randn(sum(new) + 2, hq, 128, dtype=dtype, seed=7)
    assert sum(new) * group <= 12 * len(new)                  # the form for few rows
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = 2.0 ** (-torch.arange(1, hq + 1, device="cuda").float())
    if opt.pop("prefix", False):
        opt["prefix_len"] = ints([150, 64, 1000, -3, 129, 8, 1] + [5] * 6)
    check(c, q, cu, prefill(c, q, cu, **opt), **opt)
    assert mq.moqae_paged_poll_status(c) == 0


@pytest.mark.parametrize("new, past", [([1], [100000]), ([8], [20000]), ([3] * 100, [77] * 100), ([1, 0] * 60, [9, 3000] * 60), ([2, 5, 1] * 7, [0, 4000, 16] * 7)])
def test_prefill_few_rows_lengths(new, past):
    c = pages([a + b for a, b in zip(new, past)], 2, 32, BF, 23)
    cu, q = starts(new), randn(sum(new), 8, 128, dtype=BF, seed=6)
    check(c, q, cu, prefill(c, q, cu))


@pytest.mark.parametrize("window", list(range(900, 1160, 17)))
def test_prefill_windows_of_uneven_row_tiles(window):
    """Few row tiles over a long window, which are cut into pieces; the tiles between the first and the last of a
    sequence may see a block more than either."""
    c = pages([5000 + window], 2, 16, BF, 91)
    cu, q = starts([150]), randn(150, 8, 128, dtype=BF, seed=window)
    check(c, q, cu, prefill(c, q, cu, window=window), window=window)


def test_prefill_tokens_before_every_window_may_hold_anything():
    c = pages([4000], 2, 16, BF, 41)
    cu, q = starts([50]), randn(50, 8, 128, dtype=BF, seed=8)
    opt = dict(window=300, prefix_len=ints([20]))
    want = [prefill(c, q, cu, w, **opt) for w in (False, True)]
    first = 4000 - 50 - 299                                   # first token that the first query sees
    for p in range(250):
        rows = [r for r in range(16) if 20 <= 16 * p + r < first]
        page = int(c.block_table[0, p])
        c.k_pages[page, :, rows] = float("nan")
        c.v_pages[page, :, rows] = float("inf")
        if len(rows) == 16:
            c.block_table[0, p] = -1                          # the page may have been given back
    for w, x in zip((False, True), want):
        assert torch.equal(prefill(c, q, cu, w, **opt), x)
    assert mq.moqae_paged_poll_status(c) == 0


def test_prefill_rows_that_see_nothing():
    """More queries than tokens: the first have positions below 0 and see nothing, or only the prefix."""
    c = pages([40, 0, 200], 2, 16, BF, 51)
    cu, q = starts([100, 30, 20]), randn(150, 8, 128, dtype=BF, seed=9)
    for w in (False, True):
        out = prefill(c, q, cu, w)
        assert (out[:60] == 0).all() and (out[100:130] == 0).all()
        check(c, q, cu, out)
        opt = dict(prefix_len=ints([7, 5, 0]), window=3)
        out = prefill(c, q, cu, w, **opt)
        check(c, q, cu, out, **opt)


def test_prefill_large_scores_and_values():
    """Scores that rise or fall by far more than the reference may lag behind, and large values."""
    for sign in (1, -1):
        c = pages([2000], 1, 16, BF, 61)
        ramp = torch.linspace(0, 60.0 * sign, 2000, device="cuda")
        for p in range(125):
            c.k_pages[int(c.block_table[0, p]), 0] = (ramp[16 * p:16 * p + 16, None] / 128 ** 0.5).to(BF).expand(16, 128)
            c.v_pages[int(c.block_table[0, p]), 0] *= 1e4
        q = torch.ones(700, 4, 128, dtype=BF, device="cuda") * torch.tensor([1.0, 4.0, -1.0, 0.0], device="cuda", dtype=BF)[None, :, None]
        cu = starts([700])
        for w in (False, True):
            check(c, q, cu, prefill(c, q, cu, w))


def test_prefill_bad_tables():
    c = pages([300, 60], 2, 16, FP, 71)
    cu, q = starts([50, 20]), randn(70, 4, 128, dtype=FP, seed=9)
    good = prefill(c, q, cu)
    c.block_table[0, 2] = c.k_pages.shape[0]
    out = prefill(c, q, cu)
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE and c.status.tolist()[1:3] == [0, 2]
    assert torch.equal(out[50:], good[50:]) and torch.isfinite(out.float()).all()
    c.status.zero_()
    c.kv_len[0] = -9                                          # counts as 0
    out = prefill(c, q, cu)
    assert torch.equal(out[50:], good[50:]) and (out[:50] == 0).all()
    # offsets that leave the rows of q or fall are held inside them
    c = pages([300, 60], 2, 16, FP, 71)
    out = prefill(c, q, ints([0, 50, 1 << 30]))
    assert torch.equal(out, good)
    out = prefill(c, q, ints([-5, 50, 20]))
    assert torch.equal(out[:50], good[:50]) and (out[50:] == 7.0).all()
    # a cache without pages or tokens
    e = mq.moqae_paged_bind(c.k_pages[:0], c.v_pages[:0], c.block_table[:, :0].contiguous(), ints([0, 0]))
    assert (prefill(e, q, cu) == 0).all()
    assert (prefill(mq.moqae_paged_bind(c.k_pages, c.v_pages, c.block_table[:0], ints([])), q, ints([0])) == 7.0).all()


@pytest.mark.parametrize("n, batch", [(700, 40), (60, 40)])      # large tiles, few rows per sequence
@pytest.mark.parametrize("workspace", [False, True])
def test_prefill_sequences_that_share_rows(n, batch, workspace):
    """Offsets that go back and forth: the sequences' tokens would be more than the call has."""
    c = pages([800] * batch, 8, 16, BF, 91)
    q = randn(n, 8, 128, dtype=BF, seed=92)
    out = prefill(c, q, ints([0, n] * (batch // 2) + [0]), workspace)
    assert mq.moqae_paged_poll_status(c) == mq.ERR_INVALID_ARG and (out == 7.0).all()
    c.status.zero_()
    cu = ints([0] * batch + [n])                                # the same buffers serve the next call
    check(c, q, cu, prefill(c, q, cu, workspace))
    assert mq.moqae_paged_poll_status(c) == 0


def test_sequences_that_share_pages():
    c = pages([500, 500, 500, 230], 2, 16, FP, 93)
    c.block_table[1, :20] = c.block_table[0, :20]
    c.block_table[2] = c.block_table[0]
    c.block_table[3, :14] = c.block_table[0, :14]
    cu = starts([200, 180, 500, 9])
    q = randn(889, 8, 128, dtype=FP, seed=94)
    check(c, q, cu, prefill(c, q, cu))
    q1 = randn(4, 8, 128, dtype=FP, seed=95)
    out = decode(c, q1)
    for b, n in enumerate(c.kv_len.tolist()):
        want, tol = R.attention(q1[b:b + 1], R.gather(c.k_pages, c.block_table[b], n), R.gather(c.v_pages, c.block_table[b], n), n - 1)
        R.close(out[b:b + 1], want, tol)


def test_calls_on_two_streams_at_once():
    """Each with its own workspace: prompts that fill the GPU, steps and few rows side by side."""
    c = pages([2100, 900, 40, 3000], 8, 16, BF, 96)
    q, cu = randn(1500, 32, 128, dtype=BF, seed=97), starts([1000, 400, 0, 100])
    few, cu_few = randn(9, 32, 128, dtype=BF, seed=98), starts([3, 1, 0, 5])
    step = randn(4, 32, 128, dtype=BF, seed=99)
    want = [prefill(c, q, cu), prefill(c, few, cu_few), decode(c, step)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    room = [torch.zeros(max(mq.moqae_paged_prefill_attn_workspace(c, 32, 1500), mq.moqae_paged_prefill_attn_workspace(c, 32, 9)),
                        dtype=torch.uint8, device="cuda") for _ in streams]
    outs = [[torch.empty_like(w) for w in want] for _ in streams]
    torch.cuda.synchronize()
    for turn in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                for call in range(3):
                    kind = (call + i + turn) % 3
                    if kind == 0:
                        mq.moqae_paged_prefill_attn(c, q, cu, outs[i][0], room[i])
                    elif kind == 1:
                        mq.moqae_paged_prefill_attn(c, few, cu_few, outs[i][1], room[i])
                    else:
                        mq.moqae_paged_decode_attn(c, step, outs[i][2], room[i])
    torch.cuda.synchronize()
    for got in outs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_one_workspace_for_all_calls():
    """One-token calls, calls for few and for many rows, cut and whole row tiles, all in one buffer, in turn and twice."""
    shapes = [([1, 1, 1], [4000, 20, 333]), ([300, 7, 200], [0, 900, 60]), ([40], [20000]), ([900] * 3, [100] * 3), ([2, 1, 3], [50, 7000, 1])]
    calls = []
    for new, past in shapes:
        c = pages([a + b for a, b in zip(new, past)], 2, 16, BF, 95)
        q = randn(sum(new), 8, 128, dtype=BF, seed=len(new) + sum(new))
        size = [mq.moqae_paged_prefill_attn_workspace(c, 8, q.shape[0])]
        size += [mq.moqae_paged_decode_attn_workspace(c, 8)] if max(new) == 1 else []
        calls.append((c, q, starts(new), prefill(c, q, starts(new)), decode(c, q) if max(new) == 1 else None, size))
    ws = torch.zeros(max(max(x[-1]) for x in calls), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for c, q, cu, want, one, _size in calls + calls[::-1]:
            out = torch.empty_like(q)
            mq.moqae_paged_prefill_attn(c, q, cu, out, ws)
            assert torch.equal(out, want)
            if one is not None:
                mq.moqae_paged_decode_attn(c, q, out, ws)
                assert torch.equal(out, one)
    assert (ws[:1 << 20] == 0).all()                          # the counters are at rest


def test_prefill_strided_rows_other_stream_and_graph():
    new, past = [33, 1, 140], [500, 40, 0]
    c = pages([a + b for a, b in zip(new, past)], 2, 16, BF, 81)
    cu = starts(new)
    n = sum(new)
    wide = randn(n, 12, 128, dtype=BF, seed=10)
    q = wide[:, 2:10]
    want = prefill(c, q.contiguous(), cu)
    big = torch.full((n, 20, 128), 7.0, dtype=BF, device="cuda")
    ws = torch.zeros(mq.moqae_paged_prefill_attn_workspace(c, 8, n), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mq.moqae_paged_prefill_attn(c, q, cu, big[:, 4:12], ws)
    stream.synchronize()
    assert torch.equal(big[:, 4:12], want) and (big[:, :4] == 7).all() and (big[:, 12:] == 7).all()
    out = torch.full((n, 8, 128), 7.0, dtype=BF, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.moqae_paged_prefill_attn(c, q, cu, out, ws)
    for lengths, rows in (([533, 41, 140], new), ([100, 20, 3], [100, 0, 3]), ([530, 0, 1], [1, 0, 1])):
        c.kv_len.copy_(ints(lengths))
        cu.copy_(starts(rows))
        out.fill_(7.0)
        graph.replay()
        check(c, q, cu, out)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new", [[300], [3], [1], [2] * 40, [140, 3, 1, 700]])
def test_a_row_of_one_token_is_its_value(dtype, new):
    """p v / p with one p, as rounded for the product: v after any rounding of p (an unrounded norm would be off by p's)."""
    c = pages(new, 2, 16, dtype, 77)
    cu = starts(new)
    q = 3 * randn(sum(new), 8, 128, dtype=dtype, seed=78)
    for workspace in (False, True):
        out = prefill(c, q, cu, workspace)
        check(c, q, cu, out)
        for b, n in enumerate(new):
            v = R.gather(c.v_pages, c.block_table[b], 1)[0]
            assert torch.equal(out[cu[b]], v.repeat_interleave(4, 0))


@pytest.mark.parametrize("hq, hkv", [(8, 2), (6, 2)])
def test_prefill_broadcast_queries(hq, hkv):
    """Queries with a stride of zero (one row for every token, or for every head) are read as they are."""
    c = pages([300, 40], hkv, 16, BF, 85)
    cu = starts([100, 20])
    for q in (randn(1, hq, 128, dtype=BF, seed=1).expand(120, hq, 128), randn(120, 1, 128, dtype=BF, seed=2).expand(120, hq, 128)):
        for w in (False, True):
            check(c, q.contiguous(), cu, prefill(c, q, cu, w))
    c.kv_len.copy_(ints([5, 40]))
    one = randn(1, hq, 128, dtype=BF, seed=3).expand(2, hq, 128)
    assert torch.equal(decode(c, one), decode(c, one.contiguous()))


def test_pages_interleaved_in_one_buffer_and_by_head():
    """Keys and values side by side in one buffer, and a buffer ordered by head first."""
    both = randn(12, 2, 2, 16, 128, dtype=BF, seed=1)         # [page][k or v][head][slot][128]
    byhead = randn(2, 12, 16, 128, dtype=BF, seed=2)          # [head][page][slot][128]
    table = torch.randperm(12, device="cuda").to(torch.int32)[:10].view(1, 10)
    q = randn(90, 8, 128, dtype=BF, seed=3)
    cu = starts([90])
    for k, v in ((both[:, 0], both[:, 1]), (byhead.transpose(0, 1), byhead.transpose(0, 1)), (both[:, 0], byhead.transpose(0, 1))):
        c = mq.moqae_paged_bind(k, v, table, ints([155]))
        for w in (False, True):
            check(c, q, cu, prefill(c, q, cu, w))


def test_prompt_then_steps_as_a_model_runs_them():
    """A prompt in two pieces and generated tokens through append, prefill attention and decode attention; the rows
    are the same as those of one pass over the whole sequence, and decode agrees with a prefill of one token."""
    hq, hkv, total = 8, 2, 400
    cuts = [0, 250, 390, 391, 392, 400]
    qkv = randn(total, hq + 2 * hkv, 128, dtype=BF, seed=1)
    w = [randn(128, dtype=BF, seed=s) for s in (2, 3)]
    table = mq.rope_table(1000, 128)
    rope = mq.make_rope(table, 128, q_weight=w[0], k_weight=w[1])
    k = torch.full((30, hkv, 16, 128), float("nan"), dtype=BF, device="cuda")
    c = mq.moqae_paged_bind(k, k.clone(), torch.randperm(30, device="cuda").to(torch.int32)[:26].view(1, 26).contiguous(), ints([0]))
    pos = torch.arange(total, dtype=torch.int32, device="cuda")
    qr, _ = R.norm_rope(qkv[:, :hq], w[0], table, 128, False, 1e-6, pos)
    ws = torch.zeros(mq.moqae_paged_decode_attn_workspace(c, hq), dtype=torch.uint8, device="cuda")
    for a, b in zip(cuts, cuts[1:]):
        x = qkv[a:b]
        q = torch.empty(b - a, hq, 128, dtype=BF, device="cuda")
        mq.moqae_paged_append(c, x[:, hq:hq + hkv], x[:, hq + hkv:], pos[a:b].contiguous(), seq=torch.zeros(b - a, dtype=torch.int32, device="cuda"),
                              rope=rope, q=x[:, :hq], q_out=q)
        c.kv_len.fill_(b)
        out = torch.empty_like(q)
        mq.moqae_paged_prefill_attn(c, q, ints([0, b - a]), out)
        kk, vv = (R.gather(p, c.block_table[0], b) for p in (c.k_pages, c.v_pages))
        assert torch.equal(vv, qkv[:b, hq + hkv:])
        want, tol = R.attention(q, kk, vv, a, split_weights=False)
        R.close(out, want, tol)
        assert (q.double() - qr[a:b]).abs().max() < 0.05
        if b - a == 1:
            one = torch.empty_like(q)
            mq.moqae_paged_decode_attn(c, q, one, ws)
            want, tol = R.attention(q, kk, vv, a)
            R.close(one, want, tol)


def test_paged_and_quantised_cache_agree_on_16_bit_chunks():
    """The same rotated keys and values in pages and in a quantised cache whose chunks are all 16-bit."""
    T, hq, hkv = 64 * 5 + 11, 8, 2
    k, v = randn(1, T, hkv, 128, dtype=FP, seed=1), randn(1, T, hkv, 128, dtype=FP, seed=2)
    q = randn(1, hq, 128, dtype=FP, seed=3)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    rope = mq.make_rope(mq.rope_table(T, 128), 128)
    mq.moqae_norm_rope(rope, None, k[0], pos)
    cfg = mq.make_config(n_layers=1, n_q_heads=hq, n_kv_heads=hkv, chunk=64, dtype=0, d_in=64, max_tokens=T, batch=1)
    quant = mq.moqae_cache_bind(cfg, [0, 0, 0, 5], zero_pools=True)
    mq.moqae_quantize_kv(cfg, k, v, T, 0, quant, forced_map=torch.full((1, 5), 3, dtype=torch.uint8, device="cuda"))
    a = torch.empty(1, hq, 128, dtype=torch.float32, device="cuda")
    mq.moqae_decode_attn(cfg, q, 0, quant, a, torch.zeros(mq.moqae_decode_attn_workspace(cfg), dtype=torch.uint8, device="cuda"))
    kp = torch.empty(6, hkv, 64, 128, dtype=FP, device="cuda")
    c = mq.moqae_paged_bind(kp, torch.empty_like(kp), torch.arange(6, dtype=torch.int32, device="cuda").view(1, 6), ints([T]))
    mq.moqae_paged_append(c, k[0], v[0], pos, seq=torch.zeros(T, dtype=torch.int32, device="cuda"))
    b = torch.empty(1, hq, 128, dtype=FP, device="cuda")
    mq.moqae_paged_decode_attn(c, q, b, torch.zeros(mq.moqae_paged_decode_attn_workspace(c, hq), dtype=torch.uint8, device="cuda"))
    assert (a - b.float()).abs().max() <= 2e-3                # the tolerance of the quantised cache's attention
