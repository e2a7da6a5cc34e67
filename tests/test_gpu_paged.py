"""The operators of the paged 16-bit cache on the GPU against their definitions in 64 bits."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def randn(*shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def pages(lengths, hkv, page, dtype, seed, order="hsd", spare=2, fill=None):
    """A cache whose sequences have these lengths, in pages of no order; rows behind a sequence's end, spare pages
    and spare table entries hold NaN and nonsense."""
    need = [(n + page - 1) // page for n in lengths]
    n_pages = sum(need) + spare
    shape = (n_pages, hkv, page, 128) if order == "hsd" else (n_pages, page, hkv, 128)
    k, v = randn(*shape, dtype=dtype, seed=seed), randn(*shape, dtype=dtype, seed=seed + 1)
    if order == "shd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lengths), max(need + [0]) + 1), -(1 << 30), dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor([free.pop() for _ in range(n)], dtype=torch.int32)
        if lengths[b] % page:
            last = int(table[b, n - 1])
            k[last, :, lengths[b] % page:] = float("nan")
            v[last, :, lengths[b] % page:] = float("nan")
    for p in free:
        k[p], v[p] = float("inf"), float("nan")
    return mq.moqae_paged_bind(k, v, table.cuda(), ints(lengths))


# ---- norm + rotation ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rot, interleaved", [(128, False), (128, True), (64, False), (64, True), (16, False), (16, True), (112, False), (112, True), (0, False)])
@pytest.mark.parametrize("norm", [False, True])
def test_norm_rope(dtype, rot, interleaved, norm):
    n, hq, hkv = 37, 5, 3
    qkv = randn(n, hq + 2 * hkv, 128, dtype=dtype, seed=1, scale=3.0)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]                 # slices of a wider row
    w = [randn(128, dtype=dtype, seed=s) for s in (2, 3)] if norm else [None, None]
    table = mq.rope_table(5000, rot) if rot else None
    rope = mq.make_rope(table, rot, interleaved=interleaved, q_weight=w[0], k_weight=w[1], eps=1e-5)
    pos = torch.randint(0, 5000, (n,), device="cuda", dtype=torch.int32)
    pos[[3, 36]] = -1                                        # padding tokens
    out = [torch.full((n, h, 128), 7.0, dtype=dtype, device="cuda") for h in (hq, hkv)]
    before = qkv.clone()
    mq.moqae_norm_rope(rope, q, k, pos, *out)
    assert torch.equal(qkv, before)
    real = pos >= 0
    for x, o, weight in zip((q, k), out, w):
        want, tol = R.norm_rope(x[real], weight, table, rot, interleaved, 1e-5, pos[real])
        R.close(o[real], want, tol)
        assert (o[~real] == 7.0).all()
        if not norm and rot < 128:
            assert torch.equal(o[real][..., rot:], x[real][..., rot:])      # channels that are not touched keep their bits
    mq.moqae_norm_rope(rope, q, k, pos)                      # in place
    assert torch.equal(q[real], out[0][real]) and torch.equal(k[real], out[1][real])
    assert torch.equal(qkv[~real], before[~real]) and torch.equal(qkv[:, hq + hkv:], before[:, hq + hkv:])


@pytest.mark.parametrize("n, hq, hkv", [(1, 1, 0), (1, 0, 1), (1, 32, 8), (3, 40, 40), (600, 8, 2), (5000, 9, 1)])
def test_norm_rope_sizes(n, hq, hkv):
    q, k = (randn(n, h, 128, dtype=BF, seed=h, scale=0.01) if h else None for h in (hq, hkv))
    w = randn(128, dtype=BF, seed=5)
    table = mq.rope_table(131072, 128)
    rope = mq.make_rope(table, 128, q_weight=w, eps=1e-6)    # keys without a norm
    pos = torch.arange(131072 - n, 131072, device="cuda", dtype=torch.int32)
    a, b = (None if x is None else torch.empty_like(x) for x in (q, k))
    mq.moqae_norm_rope(rope, q, k, pos, a, b)
    for x, o, weight in ((q, a, w), (k, b, None)):
        if x is not None:
            R.close(o, *R.norm_rope(x, weight, table, 128, False, 1e-6, pos))


def test_norm_rope_position_past_the_table_and_no_tokens():
    q = randn(4, 2, 128, dtype=BF, seed=1)
    table = mq.rope_table(100, 128)
    rope, status = mq.make_rope(table, 128), ints([0, 0, 0, 0])
    out = torch.full_like(q, 7.0)
    pos = ints([5, 100, 99, 1 << 30])
    mq.moqae_norm_rope(rope, q, None, pos, out, None, status)
    R.close(out[[0, 2]], *R.norm_rope(q[[0, 2]], None, table, 128, False, 1e-6, pos[[0, 2]]))
    assert (out[[1, 3]] == 7.0).all()
    assert status.tolist()[:3] in ([mq.ERR_INVALID_ARG, 1, 100], [mq.ERR_INVALID_ARG, 3, 1 << 30])
    mq.moqae_norm_rope(rope, q[:0], None, pos[:0], out[:0])
    assert mq.make_rope(None, 0).view.rot_dim == 0


def test_norm_of_extreme_rows():
    """Rows of zeros stay zero; rows whose squares pass the range of 16 bits (but not of float32) are normalised."""
    q = torch.zeros(3, 1, 128, dtype=BF, device="cuda")
    q[1] = 2.0 ** 60
    q[2] = 2.0 ** -60
    w = torch.ones(128, dtype=BF, device="cuda")
    out = torch.empty_like(q)
    mq.moqae_norm_rope(mq.make_rope(None, 0, q_weight=w, eps=1e-6), q, None, ints([0, 1, 2]), out, None)
    R.close(out, *R.norm_rope(q, w, None, 0, False, 1e-6, ints([0, 1, 2])))


# ---- append ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype, page, order", [(BF, 16, "hsd"), (FP, 16, "shd"), (BF, 64, "shd"), (FP, 128, "hsd"), (BF, 256, "hsd"), (FP, 32, "hsd")])
@pytest.mark.parametrize("with_rope", [False, True])
def test_append(dtype, page, order, with_rope):
    hq, hkv = 6, 3
    lengths = [1, page, 2 * page + 5, 0, 3 * page - 1]
    new = [1, page, 7, 0, 2 * page]
    c = pages(lengths, hkv, page, dtype, 11, order)
    seq = ints([b for b, n in enumerate(new) for _ in range(n)])
    pos = ints([lengths[b] - n + i for b, n in enumerate(new) for i in range(n)])
    n = len(pos)
    pos[4], seq[6] = -1, 5                                    # a padding token, a sequence that does not exist
    order_of = torch.randperm(n, device="cuda")
    pos, seq = pos[order_of], seq[order_of]
    qkv = randn(n, hq + 2 * hkv, 128, dtype=dtype, seed=3)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    w = randn(128, dtype=dtype, seed=4)
    table = mq.rope_table(1000, 128)
    rope = mq.make_rope(table, 128, interleaved=True, q_weight=w, k_weight=w) if with_rope else None
    out = torch.full((n, hq, 128), 7.0, dtype=dtype, device="cuda")
    k0, v0 = c.k_pages.clone(), c.v_pages.clone()
    mq.moqae_paged_append(c, k, v, pos, seq=seq, rope=rope, q=q, q_out=out)
    good = (pos >= 0) & (seq < 5)
    assert int(good.sum()) == n - 2 and (out[~good] == 7.0).all()
    page_of = c.block_table[seq[good].long(), (pos[good] // page).long()].long()
    at = (pos[good] % page).long()
    if with_rope:
        R.close(c.k_pages[page_of, :, at], *R.norm_rope(k[good], w, table, 128, True, 1e-6, pos[good]))
        R.close(out[good], *R.norm_rope(q[good], w, table, 128, True, 1e-6, pos[good]))
    else:
        assert torch.equal(c.k_pages[page_of, :, at], k[good]) and torch.equal(out[good], q[good])
    assert torch.equal(c.v_pages[page_of, :, at], v[good])
    same = torch.ones(c.k_pages.shape[0], page, dtype=torch.bool, device="cuda")    # every other row is as it was
    same[page_of, at] = False
    for now, then in ((c.k_pages, k0), (c.v_pages, v0)):
        a, b = (x.transpose(1, 2)[same].view(torch.int16) for x in (now, then))
        assert torch.equal(a, b)
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE


def test_append_one_token_per_sequence_and_bad_pages():
    c = pages([5, 40, 17], 2, 16, BF, 12)
    k, v = randn(3, 2, 128, dtype=BF, seed=1), randn(3, 2, 128, dtype=BF, seed=2)
    c.block_table[1, 2] = c.k_pages.shape[0]                  # one past the last page
    before = c.k_pages.clone()
    mq.moqae_paged_append(c, k, v, ints([4, 39, 16]))         # sequence t for token t
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE and c.status.tolist()[1:3] == [1, 39]
    for b, p in ((0, 4), (2, 16)):
        row = int(c.block_table[b, p // 16])
        assert torch.equal(c.k_pages[row, :, p % 16], k[b]) and torch.equal(c.v_pages[row, :, p % 16], v[b])
    changed = (c.k_pages.view(torch.int16) != before.view(torch.int16)).any(-1).any(1)
    assert int(changed.sum()) == 2
    c.status.zero_()
    mq.moqae_paged_append(c, k, v, ints([-5, 16 * 4, (1 << 31) - 1]))    # padding, and positions past the table
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE
    mq.moqae_paged_append(c, k[:0], v[:0], ints([]))


# ---- one new token -----------------------------------------------------------------------------

def decode(c, q, **opt):
    ws = torch.zeros(mq.moqae_paged_decode_attn_workspace(c, q.shape[1]), dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(2):                                        # the second call finds the workspace as the first left it
        out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
        mq.moqae_paged_decode_attn(c, q, out, ws, mq.make_attn_options(**opt) if opt else None)
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    return outs[0]


def check_decode(c, q, out, what="", **opt):
    prefix = opt.pop("prefix_len", None)
    for b, n in enumerate(c.kv_len.tolist()):
        k, v = (R.gather(x, c.block_table[b], n) for x in (c.k_pages, c.v_pages))
        want, tol = R.attention(q[b:b + 1], k, v, n - 1, prefix=0 if prefix is None else int(prefix[b]), **opt)
        R.close(out[b:b + 1], want, tol, f"{what} sequence {b} of {n}")


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (8, 8), (8, 2), (6, 2), (10, 2), (8, 1), (7, 1), (40, 40)])
@pytest.mark.parametrize("page, order", [(16, "hsd"), (64, "shd")])
def test_decode_head_layouts(dtype, hq, hkv, page, order):
    lengths = [1, 2, 15, 16, 17, 33, 257, 1000]
    c = pages(lengths, hkv, page, dtype, hq, order)
    q = randn(len(lengths), hq, 128, dtype=dtype, seed=5)
    check_decode(c, q, decode(c, q))
    assert mq.moqae_paged_poll_status(c) == 0


@pytest.mark.parametrize("lengths", [[0], [0, 0, 5, 0], [1], [31], [4000], [131071], [20000, 1, 0, 300] * 3, [5] * 300, [100, 0] * 200])
def test_decode_lengths(lengths):
    c = pages(lengths, 2, 32, BF, 21)
    q = randn(len(lengths), 8, 128, dtype=BF, seed=6)
    out = decode(c, q)
    if 0 in lengths:
        assert (out[[i for i, n in enumerate(lengths) if n == 0]] == 0).all()
    check_decode(c, q, out)


@pytest.mark.parametrize("dtype, hq, hkv", [(BF, 8, 2), (FP, 8, 1)])
@pytest.mark.parametrize("opt", [dict(cap=30.0), dict(cap=0.5), dict(window=1), dict(window=100), dict(window=17, cap=50.0), dict(scale=0.3),
                                 dict(slopes=True), dict(slopes=True, cap=20.0, window=200, prefix=True), dict(prefix=True),
                                 dict(window=64, prefix=True)])
def test_decode_options(dtype, hq, hkv, opt):
    lengths = [3, 64, 65, 500, 2049, 90, 130]
    c = pages(lengths, hkv, 16, dtype, 31)
    q = randn(len(lengths), hq, 128, dtype=dtype, seed=7)
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = 2.0 ** (-torch.arange(1, hq + 1, device="cuda").float())
    if opt.pop("prefix", False):
        opt["prefix_len"] = ints([100, 64, 1, 40, 16, -3, 66])
    prefix = opt.get("prefix_len")
    out = decode(c, q, **opt)
    check = dict(opt)
    if prefix is not None:
        check["prefix_len"] = prefix.clamp(min=0)
    check_decode(c, q, out, **check)


@pytest.mark.parametrize("cap", [1e-4, 0.01, 1.0, 3.0, 500.0, 1e5, 1e20])
def test_decode_caps(cap):
    """Caps far below and far above the scores: an all but uniform and an all but plain softmax."""
    c = pages([700, 33], 2, 16, FP, 35)
    q = randn(2, 8, 128, dtype=FP, seed=9, scale=3.0)
    check_decode(c, q, decode(c, q, cap=cap), cap=cap)


def test_decode_reads_only_what_is_seen():
    """Tokens outside the window may hold NaN, and their pages may have been given back."""
    c = pages([1000], 2, 16, BF, 41)
    q = randn(1, 8, 128, dtype=BF, seed=8)
    want = decode(c, q, window=100, prefix_len=ints([10]))
    hidden = torch.zeros(1000, dtype=torch.bool)
    hidden[10:900] = True
    for p in range(63):
        at = torch.arange(16) + 16 * p
        at = at[at < 1000]
        rows = hidden[at].nonzero().flatten()
        page = int(c.block_table[0, p])
        c.k_pages[page, :, rows] = float("nan")
        c.v_pages[page, :, rows] = float("inf")
        if hidden[at].all():
            c.block_table[0, p] = -1
    assert torch.equal(decode(c, q, window=100, prefix_len=ints([10])), want)
    assert mq.moqae_paged_poll_status(c) == 0


def test_decode_large_scores_and_values():
    """Scores far apart (weights from 1 down to nothing) in rising and falling order, and large values."""
    for sign in (1, -1):
        c = pages([3000], 1, 16, BF, 51)
        ramp = torch.linspace(0, 40.0 * sign, 3008, device="cuda")
        for p in range(188):
            c.k_pages[int(c.block_table[0, p]), 0] = (ramp[16 * p:16 * p + 16, None] / 128 ** 0.5).to(BF).expand(16, 128)
            c.v_pages[int(c.block_table[0, p]), 0] *= 1e4
        q = torch.ones(1, 4, 128, dtype=BF, device="cuda") * torch.tensor([1.0, 4.0, -1.0, 0.0], device="cuda", dtype=BF)[None, :, None]
        c.kv_len[0] = 3000
        check_decode(c, q, decode(c, q))


def test_decode_bad_pages_are_left_out():
    c = pages([100, 60], 2, 16, FP, 61)
    q = randn(2, 4, 128, dtype=FP, seed=9)
    good = decode(c, q)
    c.block_table[0, 2] = c.k_pages.shape[0]
    c.block_table[0, 5] = -1
    out = decode(c, q)
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE and c.status.tolist()[1] == 0 and c.status.tolist()[2] in (2, 5)
    assert torch.equal(out[1], good[1]) and torch.isfinite(out[0].float()).all()
    assert mq.moqae_paged_validate(c) == (mq.ERR_CORRUPT_TABLE, 0, 2)
    c = pages([100, 60], 2, 16, FP, 61)
    c.kv_len[1] = 16 * c.block_table.shape[1] + 1             # longer than its row of the table
    c.kv_len[0] = -4
    out = decode(c, q)
    assert (out[0] == 0).all()
    assert mq.moqae_paged_poll_status(c) == mq.ERR_CORRUPT_TABLE and c.status.tolist()[2] == -1


def test_decode_strided_rows_other_stream_and_graph():
    c = pages([700, 20, 333], 2, 16, BF, 71)
    wide = randn(3, 12, 128, dtype=BF, seed=10)
    q = wide[:, 2:10]
    want = decode(c, q.contiguous())
    big = torch.full((3, 20, 128), 7.0, dtype=BF, device="cuda")
    ws = torch.zeros(mq.moqae_paged_decode_attn_workspace(c, 8), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mq.moqae_paged_decode_attn(c, q, big[:, 4:12], ws)
    stream.synchronize()
    assert torch.equal(big[:, 4:12], want) and (big[:, :4] == 7).all() and (big[:, 12:] == 7).all()
    # a captured call sees the lengths and tables of the time it is replayed
    out = torch.empty(3, 8, 128, dtype=BF, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.moqae_paged_decode_attn(c, q, out, ws)
    for lengths in ([700, 20, 333], [1, 16, 300], [699, 0, 17]):
        c.kv_len.copy_(ints(lengths))
        graph.replay()
        check_decode(c, q, out)


def test_decode_past_32_bit_offsets():
    """A pool of more than 2^32 bytes and 2^31 elements of keys: a sequence in its last pages."""
    n_pages = (1 << 31) // (2 * 64 * 128) + 40
    k = torch.empty(n_pages, 2, 64, 128, dtype=BF, device="cuda")
    v = torch.empty(n_pages, 2, 64, 128, dtype=BF, device="cuda")
    table = torch.arange(n_pages - 8, n_pages, dtype=torch.int32, device="cuda")[None].flip(1).contiguous()
    c = mq.moqae_paged_bind(k, v, table, ints([500]))
    new_k, new_v = randn(500, 2, 128, dtype=BF, seed=1), randn(500, 2, 128, dtype=BF, seed=2)
    mq.moqae_paged_append(c, new_k, new_v, torch.arange(500, dtype=torch.int32, device="cuda"), seq=torch.zeros(500, dtype=torch.int32, device="cuda"))
    q = randn(1, 8, 128, dtype=BF, seed=3)
    want, tol = R.attention(q, new_k, new_v, 499)
    R.close(decode(c, q), want, tol)


def test_refusals_of_the_binding():
    c = pages([20], 2, 16, BF, 81)
    q = randn(1, 8, 128, dtype=BF, seed=1)
    ws = torch.zeros(mq.moqae_paged_decode_attn_workspace(c, 8), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for bad in (q.half(), q.cpu(), q[:, :, :64], q.expand(2, 8, 128), q.transpose(1, 2), q[0]):
        with pytest.raises(mq.MoqaeError):
            mq.moqae_paged_decode_attn(c, bad, out, ws)
    with pytest.raises(mq.MoqaeError) as e:
        mq.moqae_paged_decode_attn(c, q, out, ws[:-16])
    assert e.value.code == mq.ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(mq.MoqaeError):
        mq.moqae_paged_decode_attn(c, q, out, ws, mq.make_attn_options(slopes=torch.zeros(4, device="cuda")))
    with pytest.raises(mq.MoqaeError):
        mq.moqae_paged_append(c, q[:, :2], q[:, :2], ints([0, 1]))
    with pytest.raises(mq.MoqaeError):
        mq.moqae_paged_append(c, q[:, :2], q[:, :2], ints([0]), rope=mq.make_rope(None, 0, k_weight=torch.ones(128, device="cuda", dtype=FP)))
    with pytest.raises(mq.MoqaeError):
        mq.moqae_paged_bind(c.k_pages, c.v_pages[:1], c.block_table, c.kv_len)
    with pytest.raises(mq.MoqaeError):
        mq.moqae_paged_bind(c.k_pages, c.v_pages, c.block_table.long(), c.kv_len)
