"""Paged 4-bit cache on the GPU: append and read against the quantiser in 64 bits, one-token and several-token attention
against the definition over the stored bytes."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .paged_reference import F32, close, norm_rope

pytestmark = pytest.mark.gpu
DTYPES = (torch.bfloat16, torch.float16)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def make_cache(gen, lens, hkv, page, dtype, *, heads_first=False, spread=1.0, max_pages=None, fill=True):
    """A cache of random keys and values; pages in no order, unused bytes 0xff (scales and zeros are NaN there)."""
    need = [(n + page - 1) // page for n in lens]
    n_pages, width = sum(need) + 2, max_pages or max(1, max(need, default=1))
    shape = (hkv, n_pages) if heads_first else (n_pages, hkv)
    pages = torch.full((*shape, page * 160), 255, dtype=torch.uint8, device="cuda")
    if heads_first:
        pages = pages.transpose(0, 1)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), width), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cache = mq.moqae_paged4_bind(pages, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), dtype)
    for b, n in enumerate(lens if fill else []):
        if not n:
            continue
        m = (n + 15) // 16 * 16
        k, v = (randn(gen, m // 16, hkv, 16, 128) * spread for _ in range(2))
        tiles = ref.pack(k, v)
        t = torch.arange(n, device="cuda")
        # whole tiles, then the bytes of the tokens that the sequence has in its last one
        full, rest = n // 16, n % 16
        entry = lambda i: (int(table[b, i * 16 // page]), slice(None), slice((i * 16 % page) * 160, (i * 16 % page) * 160 + 2560))  # noqa: E731
        for i in range(full):
            pages[entry(i)] = tiles[i]
        if rest:
            own = torch.zeros(2560, dtype=torch.bool, device="cuda")
            key, key_s, value, value_s = ref.places("cuda")
            for x in (key, key_s, key_s + 1, key_s + 8, key_s + 9, value, value_s, value_s + 1, value_s + 16, value_s + 17):
                own[x[:rest].flatten()] = True
            pages[entry(full)] = torch.where(own, tiles[full], pages[entry(full)])
        del t
    return cache


def stored(cache, b, n):
    return ref.rows_of(cache.pages, cache.block_table[b], n)


def space(size):
    return torch.zeros(size, dtype=torch.uint8, device="cuda")


def options_of(gen, hq, batch, *, scale=None, cap=0.0, window=0, alibi=False, prefix=0):
    slopes = (2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda") / hq)).float() if alibi else None
    lens = torch.randint(-1, prefix + 1, (batch,), generator=gen, device="cuda").to(torch.int32) if prefix else None
    return mq.make_attn_options(scale=scale or 0.0, cap=cap, window=window, slopes=slopes, prefix_len=lens), slopes, lens


def check(cache, q, new, got, slopes, prefix, *, scale=None, cap=0.0, window=0, up=0, what=""):
    """`got` against the definition, sequence by sequence."""
    at = 0
    for b, n in enumerate(new):
        total = int(cache.kv_len[b])
        rows = q[at:at + n]
        f = 0 if prefix is None else min(max(int(prefix[b]), 0), total)
        want, tol = ref.attention(rows, *stored(cache, b, total), total - n, scale=scale, cap=cap, window=window, slopes=slopes, prefix=f, up=up)
        close(got[at:at + n], want, tol, f"{what} sequence {b} of {total}, {n} new")
        at += n


# ---- append and read ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq, hkv, page, order", [(8, 2, 16, "seq"), (3, 3, 64, "mixed"), (5, 1, 256, "mixed"), (0, 4, 32, "seq")])
def test_values_and_plain_keys_are_quantised_exactly(dtype, hq, hkv, page, order):
    gen = generator(hq + page)
    lens = [37, 0, 1, 300]
    cache = make_cache(gen, lens, hkv, page, dtype, heads_first=page == 64, fill=False)
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()
    seq = torch.repeat_interleave(torch.arange(4, dtype=torch.int32), torch.tensor(lens)).cuda()
    if order == "mixed":
        mix = torch.randperm(len(pos), generator=gen, device="cuda")
        pos, seq = pos[mix], seq[mix]
    n = len(pos)
    qkv = randn(gen, n, hq + 2 * hkv, 128) * torch.logspace(-4, 3, n, device="cuda")[:, None, None]
    qkv[5] = 0.125                                                          # groups of one value
    qkv[7, :, 33] = 60000.0
    qkv = qkv.to(dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    before = cache.pages.clone()
    if hq:
        q_out = torch.zeros(n, hq, 128, dtype=dtype, device="cuda")
        mq.moqae_paged4_append(cache, k, v, pos, seq=seq, q=q, q_out=q_out)
        assert (q_out == q).all()
    else:
        mq.moqae_paged4_append(cache, k, v, pos, seq=seq)
    # the whole cache, byte for byte
    key, key_s, value, value_s = ref.places("cuda")
    k_out, v_out = torch.zeros_like(k), torch.zeros_like(v)
    mq.moqae_paged4_read(cache, k_out, v_out, pos, seq=seq)
    for b, total in enumerate(lens):
        mine = seq == b
        at = pos[mine].long()
        kk, vv = (torch.zeros((total + 15) // 16 * 16, hkv, 128, dtype=torch.float64, device="cuda") for _ in range(2))
        kk[at], vv[at] = k[mine].double(), v[mine].double()
        tiles = ref.pack(kk.unflatten(0, (-1, 16)).transpose(1, 2), vv.unflatten(0, (-1, 16)).transpose(1, 2))
        for i in range(tiles.shape[0]):
            p, first = int(cache.block_table[b, i * 16 // page]), (i * 16 % page) * 160
            got, old = cache.pages[p, :, first:first + 2560], before[p, :, first:first + 2560]
            own = torch.zeros(2560, dtype=torch.bool, device="cuda")
            live = min(16, total - 16 * i)
            for x in (key, key_s, key_s + 1, key_s + 8, key_s + 9, value, value_s, value_s + 1, value_s + 16, value_s + 17):
                own[x[:live].flatten()] = True
            assert (got == torch.where(own, tiles[i], old)).all(), f"sequence {b}, tile {i}"
        if total:
            kc, kz, vc, vz, _ = stored(cache, b, total)
            for got, want in ((k_out[mine], (kc + kz)[at]), (v_out[mine], (vc + vz)[at])):
                assert (got == want.float().to(dtype)).all()               # z + s code is exact in float32, or rounded once more there
    assert int(cache.status[0]) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rot, interleaved, norm", [(128, False, True), (64, False, False), (96, False, True), (112, True, True), (128, True, False), (0, False, True), (16, False, False)])
def test_keys_with_norm_and_rotation(dtype, rot, interleaved, norm):
    gen = generator(rot + norm)
    n, hq, hkv, page = 77, 6, 3, 32
    cache = make_cache(gen, [100], hkv, page, dtype, fill=False)
    weight = lambda: (1 + 0.2 * randn(gen, 128)).to(dtype) if norm else None  # noqa: E731
    table = mq.rope_table(100, rot) if rot else None
    rope = mq.make_rope(table, rot, interleaved=interleaved, q_weight=weight(), k_weight=weight(), eps=1e-5)
    q, k, v = (randn(gen, n, h, 128, dtype=dtype) for h in (hq, hkv, hkv))
    pos = (torch.randperm(100, generator=gen, device="cuda")[:n]).to(torch.int32)
    seq = torch.zeros(n, dtype=torch.int32, device="cuda")
    q_out = torch.empty_like(q)
    mq.moqae_paged4_append(cache, k, v, pos, seq=seq, rope=rope, q=q, q_out=q_out)
    want, tol = norm_rope(q, rope.tensors[1], table, rot, interleaved, 1e-5, pos)
    close(q_out, want, tol, "queries")
    want, _ = norm_rope(k, rope.tensors[2], table, rot, interleaved, 1e-5, pos)
    # the row in float32: up to 24 roundings of a pair's size (see norm_rope), here of the row's largest element twice
    e = 48 * F32 * want.abs().amax(-1, keepdim=True)
    kc, kz, _, _, _ = stored(cache, 0, 100)
    rows, z = (kc + kz)[pos.long()].unflatten(-1, (4, 32)), kz[pos.long()].unflatten(-1, (4, 32))[..., 0]
    x, e = want.unflatten(-1, (4, 32)), e
    low, high = x.amin(-1), x.amax(-1)
    page_of = cache.block_table[0].long()[pos.long() // page]
    tiles = cache.pages.unflatten(-1, (page // 16, 2560))[page_of, :, (pos.long() % page) // 16]
    _, s, zs = ref.unpack(tiles)[0]
    s = s.gather(2, (pos.long() % 16)[:, None, None, None].expand(-1, hkv, 1, 4)).squeeze(2)
    line = ref.fp16_line("cuda")
    above = line[(torch.searchsorted(line, z.contiguous(), right=True)).clamp_max(len(line) - 1)]
    below = line[(torch.searchsorted(line, s.contiguous()) - 1).clamp_min(0)]
    assert (z <= low + e).all() and (above > low - e).all()
    span = (high - z) / 15
    assert (s >= span * (1 - 2 * F32) - e).all() and ((below < span * (1 + 2 * F32) + e) | (s == 0)).all()
    # nearest code
    assert ((rows - x).abs() <= (s * (0.5 + 2.0 ** -18) + e)[..., None]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_and_read_leave_padding_and_what_does_not_exist_alone(dtype):
    gen = generator(3)
    cache = make_cache(gen, [40, 20], 2, 16, dtype)
    before = cache.pages.clone()
    k, v = randn(gen, 4, 2, 128, dtype=dtype), randn(gen, 4, 2, 128, dtype=dtype)
    pos = torch.tensor([-1, 48, 3, 5], dtype=torch.int32, device="cuda")           # padding; no such page; no such sequence; negative sequence
    seq = torch.tensor([0, 0, 2, -1], dtype=torch.int32, device="cuda")
    mq.moqae_paged4_append(cache, k, v, pos, seq=seq)
    assert (cache.pages == before).all() and cache.status[0].item() == mq.ERR_CORRUPT_TABLE
    assert mq.moqae_paged_poll_status(cache) == mq.ERR_CORRUPT_TABLE
    cache.status.zero_()
    k_out, v_out = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    mq.moqae_paged4_read(cache, k_out, v_out, pos, seq=seq)
    assert (k_out == 7).all() and (v_out == 7).all() and cache.status[0].item() == mq.ERR_CORRUPT_TABLE
    # one side alone, into rows of a wider buffer
    wide = torch.zeros(3, 6, 128, dtype=dtype, device="cuda")
    p2, s2 = torch.tensor([39, 0, 19], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    mq.moqae_paged4_read(cache, None, wide[:, 2:4], p2, seq=s2)
    for i, (b, p) in enumerate(((0, 39), (1, 0), (1, 19))):
        _, _, vc, vz, _ = stored(cache, b, p + 1)
        assert (wide[i, 2:4] == (vc + vz)[p].float().to(dtype)).all()
    assert (wide[:, :2] == 0).all() and (wide[:, 4:] == 0).all()


# ---- one new token -----------------------------------------------------------------------------

CASES = [
    dict(lens=[1], hq=8, hkv=8, page=16), dict(lens=[0, 1, 2, 15, 16, 17, 0], hq=4, hkv=2, page=16),
    dict(lens=[31, 33, 500, 64], hq=8, hkv=1, page=32), dict(lens=[700, 3, 2049], hq=6, hkv=2, page=256),
    dict(lens=[5000], hq=32, hkv=8, page=64), dict(lens=[130] * 9, hq=7, hkv=1, page=128), dict(lens=[9, 4000, 20, 1], hq=5, hkv=1, page=16),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shaping", [dict(), dict(cap=30.0), dict(window=16), dict(window=100, prefix=40), dict(cap=5.0, alibi=True, prefix=70, scale=0.3)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c["lens"][:3])))
def test_decode(dtype, case, shaping):
    gen = generator(len(case["lens"]) + case["hq"])
    lens, hq, hkv = case["lens"], case["hq"], case["hkv"]
    cache = make_cache(gen, lens, hkv, case["page"], dtype, heads_first=hq == 6)
    opt, slopes, prefix = options_of(gen, hq, len(lens), **shaping)
    q = randn(gen, len(lens), hq + 2, 128, dtype=dtype)[:, 1:hq + 1]
    out = torch.full((len(lens), hq, 128), 9.0, dtype=dtype, device="cuda")
    work = space(mq.moqae_paged4_decode_attn_workspace(cache, hq))
    for _ in range(2):                                   # the second call finds the counters as the first left them
        mq.moqae_paged4_decode_attn(cache, q, out, work, opt)
    rest = {k: v for k, v in shaping.items() if k in ("scale", "cap", "window")}
    for b, n in enumerate(lens):
        if n == 0:
            assert (out[b] == 0).all()
    keep = [b for b, n in enumerate(lens) if n]
    at = torch.tensor(keep, device="cuda", dtype=torch.long)
    for b in keep:
        want, tol = ref.attention(q[b:b + 1], *stored(cache, b, lens[b]), lens[b] - 1, slopes=slopes,
                                  prefix=0 if prefix is None else min(max(int(prefix[b]), 0), lens[b]), **rest)
        close(out[b:b + 1], want, tol, f"sequence {b}")
    assert cache.status[0].item() == 0 and (work[:1 << 20] == 0).all() and len(at) == len(keep)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spread, q_scale", [(1000.0, 1e-3), (1e-3, 1e3), (30.0, 1.0), (1.0, 1e-6)])
def test_decode_of_large_and_small_values(dtype, spread, q_scale):
    gen = generator(11)
    cache = make_cache(gen, [900, 17], 2, 16, dtype, spread=spread)
    q = (randn(gen, 2, 8, 128) * q_scale).to(dtype)
    out = torch.empty_like(q)
    mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 8)))
    # scales: a fifteenth of at most 10 spreads; below 1 the weights' steps count from the code 15 on
    up = max(0, (int(spread * 10 / 15)).bit_length())
    check(cache, q, [1, 1], out, None, None, up=up)


@pytest.mark.parametrize("dtype", DTYPES)
def test_scales_that_grow_along_the_sequence(dtype):
    """Value scales pass 1, 2, 4, .. on the way, so the room above the weights shrinks while sums are under way."""
    gen = generator(12)
    n = 640
    cache = make_cache(gen, [n], 1, 64, dtype, fill=False)
    k = randn(gen, n, 1, 128, dtype=dtype)
    v = (randn(gen, n, 1, 128) * torch.logspace(-3, 3.8, n, base=10.0, device="cuda")[:, None, None]).to(dtype)
    mq.moqae_paged4_append(cache, k, v, torch.arange(n, dtype=torch.int32, device="cuda"), seq=torch.zeros(n, dtype=torch.int32, device="cuda"))
    q = randn(gen, 1, 4, 128, dtype=dtype)
    out = torch.empty_like(q)
    mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 4)))
    check(cache, q, [1], out, None, None, up=13)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_small_weights_behind_one_large_score(dtype):
    """8000 tokens of weight 2^-26 beside one: together 1.2e-4 of the result, which shows where their values are large."""
    n = 8001
    gen = generator(13)
    cache = make_cache(gen, [n], 1, 256, dtype, fill=False)
    k, v = torch.zeros(n, 1, 128, device="cuda"), torch.full((n, 1, 128), 1000.0, device="cuda")
    k[0, 0, 0], v[0] = 16.0, 0.0
    mq.moqae_paged4_append(cache, k.to(dtype), v.to(dtype), torch.arange(n, dtype=torch.int32, device="cuda"), seq=torch.zeros(n, dtype=torch.int32, device="cuda"))
    q = torch.zeros(1, 1, 128, device="cuda")
    q[0, 0, 0] = 1.0
    scale = 26 * 0.6931471805599453 / 16
    out = torch.empty(1, 1, 128, dtype=dtype, device="cuda")
    mq.moqae_paged4_decode_attn(cache, q.to(dtype), out, space(mq.moqae_paged4_decode_attn_workspace(cache, 1)), mq.make_attn_options(scale=scale))
    want = 8000 * 2.0 ** -26 * 1000 / (1 + 8000 * 2.0 ** -26)
    assert ((out.double() - want).abs() <= want * 2.0 ** -6).all(), out[0, 0, 0]


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_mean_of_a_long_context_keeps_its_bits(dtype):
    """40000 tokens of nearly equal weight: the result is 200 times smaller than a value, and the sums of its parts may not hide it.  Rounding
    p, p s and the middle of a range, at random: 2^-11 / sqrt(12) (rms 1.4e-4 x 2) of parts at most 7.5 steps of a fifteenth of 4 to 5 deviations,
    times the sqrt(3) of three of them: below 1.2e-3 of a value's deviation, to which the result's rounding is added."""
    n = 40000
    gen = generator(17)
    cache = make_cache(gen, [n], 1, 256, dtype, fill=False)
    k, v = randn(gen, n, 1, 128, dtype=dtype), randn(gen, n, 1, 128, dtype=dtype)
    mq.moqae_paged4_append(cache, k, v, torch.arange(n, dtype=torch.int32, device="cuda"), seq=torch.zeros(n, dtype=torch.int32, device="cuda"))
    q = (0.1 * randn(gen, 3, 8, 128)).to(dtype)
    work = space(mq.moqae_paged4_prefill_attn_workspace(cache, 8, 3))
    want, _ = ref.attention(q, *stored(cache, 0, n), n - 3)
    out, one = torch.empty_like(q), torch.empty_like(q[:1])
    mq.moqae_paged4_prefill_attn(cache, q, torch.tensor([0, 3], dtype=torch.int32, device="cuda"), out, work)
    mq.moqae_paged4_decode_attn(cache, q[2:], one, work)
    u = torch.finfo(dtype).eps / 2
    for got, right in ((out, want), (one, want[2:])):
        assert ((got.double() - right).norm() / right.norm()) <= 1.2e-3 + u


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_token_is_its_value(dtype):
    gen = generator(14)
    cache = make_cache(gen, [1, 1], 3, 16, dtype)
    q = randn(gen, 2, 24, 128, dtype=dtype)
    out = torch.empty_like(q)
    mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 24)))
    check(cache, q, [1, 1], out, None, None)


def test_bad_pages_and_lengths_are_read_as_nothing():
    gen = generator(15)
    cache = make_cache(gen, [100, 50], 2, 16, torch.bfloat16)
    q = randn(gen, 2, 4, 128, dtype=torch.bfloat16)
    out, work = torch.empty_like(q), space(mq.moqae_paged4_decode_attn_workspace(cache, 4))
    mq.moqae_paged4_decode_attn(cache, q, out, work)
    good = out[1].clone()
    held = cache.block_table[0, 2].item()
    for bad in (-1, cache.pages.shape[0], 1 << 30):
        cache.status.zero_()
        cache.block_table[0, 2] = bad
        mq.moqae_paged4_decode_attn(cache, q, out, work)
        assert cache.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, 0, 2] and (out[1] == good).all() and torch.isfinite(out.float()).all()
        assert mq.moqae_paged_validate(cache) == (mq.ERR_CORRUPT_TABLE, 0, 2)
        want, tol = ref.attention(q[:1], *stored(make_zero_page(cache, 0, 2, held), 0, 100), 99)
        close(out[:1], want, tol, "a page of zeros")
    cache.block_table[0, 2] = held
    assert mq.moqae_paged_validate(cache) == (mq.OK, -1, -1)
    cache.status.zero_()
    cache.kv_len[0] = 16 * cache.block_table.shape[1] + 1
    mq.moqae_paged4_decode_attn(cache, q, out, work)
    assert cache.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, 0, -1] and (out[0] == 0).all() and (out[1] == good).all()


def make_zero_page(cache, b, entry, page):
    """The cache as the kernels see it: that page all zeros."""
    pages, table = cache.pages.clone(), cache.block_table.clone()
    pages[page] = 0
    table[b, entry] = page
    return mq.moqae_paged4_bind(pages, table, cache.kv_len, torch.bfloat16)


def test_pages_past_32_bits_of_bytes():
    gen = generator(16)
    n_pages, hkv, page = 220000, 4, 16                    # 2.3 GB
    pages = torch.empty(n_pages, hkv, page * 160, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, 5], [n_pages - 2, n_pages - 3]], dtype=torch.int32, device="cuda")
    cache = mq.moqae_paged4_bind(pages, table, torch.tensor([20, 32], dtype=torch.int32, device="cuda"), torch.bfloat16)
    n = 52
    k, v = randn(gen, n, hkv, 128, dtype=torch.bfloat16), randn(gen, n, hkv, 128, dtype=torch.bfloat16)
    pos = torch.cat([torch.arange(20), torch.arange(32)]).to(torch.int32).cuda()
    seq = torch.cat([torch.zeros(20), torch.ones(32)]).to(torch.int32).cuda()
    mq.moqae_paged4_append(cache, k, v, pos, seq=seq)
    q = randn(gen, 2, 8, 128, dtype=torch.bfloat16)
    out = torch.empty_like(q)
    mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 8)))
    check(cache, q, [1, 1], out, None, None)
    v_out = torch.empty_like(v)
    mq.moqae_paged4_read(cache, None, v_out, pos, seq=seq)
    _, _, vc, vz, _ = stored(cache, 1, 32)
    assert (v_out[20:] == (vc + vz).float().bfloat16()).all()


# ---- several new tokens ------------------------------------------------------------------------

PREFILLS = [
    dict(new=[1], past=[0], hq=8, hkv=8, page=16), dict(new=[3, 0, 1, 8, 5], past=[100, 7, 0, 33, 900], hq=32, hkv=8, page=16),
    dict(new=[130], past=[0], hq=4, hkv=1, page=64), dict(new=[64, 200, 17], past=[300, 0, 1], hq=6, hkv=2, page=128),
    dict(new=[257, 1], past=[40, 2000], hq=7, hkv=1, page=32), dict(new=[700], past=[0], hq=2, hkv=2, page=256),
    dict(new=[129, 128, 127], past=[0, 1, 129], hq=8, hkv=1, page=16),
    # more new tokens than the sequence has: the first ones stand before it and see nothing
    dict(new=[10, 140, 3], past=[-4, -5, -3], hq=4, hkv=2, page=16),
    # few rows and many side by side: 24 tokens of a group of four are 96 rows, 25 are 100
    dict(new=[1, 24, 25, 0, 300, 1, 23], past=[700, 100, 90, 5, 0, 0, 3], hq=8, hkv=2, page=32),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shaping", [dict(), dict(cap=30.0), dict(window=50), dict(window=40, prefix=30), dict(cap=5.0, alibi=True, prefix=70, scale=0.3), dict(alibi=True)])
@pytest.mark.parametrize("case", PREFILLS, ids=lambda c: "-".join(map(str, c["new"])))
def test_prefill(dtype, case, shaping):
    new, past, hq, hkv = case["new"], case["past"], case["hq"], case["hkv"]
    gen = generator(sum(new) + hq)
    lens = [a + b for a, b in zip(new, past)]
    cache = make_cache(gen, lens, hkv, case["page"], dtype, heads_first=hq == 6)
    opt, slopes, prefix = options_of(gen, hq, len(new), **shaping)
    n = sum(new)
    q = randn(gen, n + 3, hq + 2, 128, dtype=dtype)[:, 1:hq + 1]
    out = torch.full((n + 3, hq, 128), 9.0, dtype=dtype, device="cuda")
    cu = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    size, least = (mq.moqae_paged4_prefill_attn_workspace(cache, hq, n + 3, least=x) for x in (False, True))
    work = space(size)
    for _ in range(2):
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, work, opt)
    # without room for expanded blocks, and with room for some sequences, the same bits
    for part in (least, least + (size - least) // 2):
        small, again = space(part), torch.full_like(out, 9.0)
        mq.moqae_paged4_prefill_attn(cache, q, cu, again, small, opt)
        assert (again == out).all() and (small[:1 << 20] == 0).all(), part
    assert (out[n:] == 9).all()                           # rows behind the last sequence
    rest = {k: v for k, v in shaping.items() if k in ("scale", "cap", "window")}
    check(cache, q[:n], new, out[:n], slopes, prefix, **rest)
    assert cache.status[0].item() == 0 and (work[:1 << 20] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_then_steps(dtype):
    """As a model runs it: plan, append, attend; one workspace, pages shared out by the pool."""
    gen = generator(21)
    batch, hq, hkv, page = 3, 8, 2, 32
    pool = mq.make_page_pool(40)
    pages = torch.empty(40, hkv, page * 160, dtype=torch.uint8, device="cuda")
    cache = mq.moqae_paged4_bind(pages, torch.full((batch, 12), -1, dtype=torch.int32, device="cuda"),
                                 torch.zeros(batch, dtype=torch.int32, device="cuda"), dtype)
    rope = mq.make_rope(mq.rope_table(400, 128), 128)
    work = space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, 384))
    for new in ([200, 1, 77], [1, 1, 1], [0, 5, 1], [1, -4, -78], [3, 2, 90], [1, 1, 1]):
        n = sum(max(0, x) for x in new)
        rows = n + 2
        n_new = torch.tensor(new, dtype=torch.int32, device="cuda")
        cu = torch.empty(batch + 1, dtype=torch.int32, device="cuda")
        pos, seq = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
        mq.moqae_paged_plan(cache, pool, n_new, cu, pos, seq)
        q, k, v = (randn(gen, rows, h, 128, dtype=dtype) for h in (hq, hkv, hkv))
        mq.moqae_paged4_append(cache, k, v, pos, seq=seq, rope=rope, q=q)
        out = torch.zeros_like(q)
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, work)
        grown = [max(0, x) for x in new]
        check(cache, q[:n], grown, out[:n], None, None, what=str(new))
        if all(x == 1 for x in new):
            one = torch.empty(batch, hq, 128, dtype=dtype, device="cuda")
            mq.moqae_paged4_decode_attn(cache, q[:n], one, work)
            check(cache, q[:n], grown, one, None, None, what="one token")
        assert (out[n:] == 0).all()
    assert cache.status[0].item() == 0
    used = sum((int(x) + page - 1) // page for x in cache.kv_len)
    assert int(pool.state[1]) == 40 - used
    live = [int(cache.block_table[b, i]) for b in range(batch) for i in range((int(cache.kv_len[b]) + page - 1) // page)]
    free = [int(pool.ring[(int(pool.state[0]) + i) % 40]) for i in range(int(pool.state[1]))]
    assert sorted(live + free) == list(range(40))


def test_readme_example():
    """The example of the 4-bit cache, run as it stands in the README."""
    import os
    import re
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        block = re.search(r"\n((?: {4}.*\n)*? {4}.*make_page_pool.*\n(?: {4}.*\n)*)", f.read()).group(1)
    gen = generator(41)
    new, n_q_heads, n_kv_heads, page_size, n_pages, n_tokens = [300, 5, 77], 8, 2, 16, 40, 384
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    block_table, kv_len = torch.full((3, 20), -1, dtype=torch.int32, device="cuda"), ints(0, 0, 0)
    n_new, one_each, cu_q = ints(*new), ints(1, 1, 1), torch.zeros(4, dtype=torch.int32, device="cuda")
    positions, seq = (torch.zeros(n_tokens, dtype=torch.int32, device="cuda") for _ in range(2))
    positions1, seq1 = ints(0, 0, 0), ints(0, 0, 0)
    rope = mq.make_rope(mq.rope_table(400, 128), 128)
    q, k, v = (randn(gen, n_tokens, h, 128, dtype=torch.bfloat16) for h in (n_q_heads, n_kv_heads, n_kv_heads))
    q1, k1, v1 = (randn(gen, 3, h, 128, dtype=torch.bfloat16) for h in (n_q_heads, n_kv_heads, n_kv_heads))
    out, out1, k_back, v_back = torch.full_like(q, 7.0), torch.full_like(q1, 7.0), torch.zeros_like(k1), torch.zeros_like(v1)
    names = dict(globals(), **locals())
    exec("".join(line[4:] + "\n" for line in block.splitlines()), names)
    cache = names["cache4"]
    assert mq.moqae_paged_poll_status(cache) == 0 and kv_len.tolist() == [n + 1 for n in new] and (out[382:] == 7).all()
    check(cache, q1, [1, 1, 1], out1, None, None)
    kv_len.copy_(n_new)
    check(cache, q[:382], new, out[:382], None, None)
    for b, n in enumerate(new):
        kc, kz, vc, vz, _ = stored(cache, b, n + 1)
        assert (k_back[b] == (kc + kz)[n].float().bfloat16()).all() and (v_back[b] == (vc + vz)[n].float().bfloat16()).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_views_of_pages(dtype):
    """One page of one head out of a larger buffer, and a cache without pages."""
    gen = generator(42)
    buffer = torch.zeros(3, 5, 16 * 160 + 32, dtype=torch.uint8, device="cuda")
    pages = buffer[1:2, 2:3, 32:]
    cache = mq.moqae_paged4_bind(pages, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([9], dtype=torch.int32, device="cuda"), dtype)
    k, v = randn(gen, 9, 1, 128, dtype=dtype), randn(gen, 9, 1, 128, dtype=dtype)
    mq.moqae_paged4_append(cache, k, v, torch.arange(9, dtype=torch.int32, device="cuda"), seq=torch.zeros(9, dtype=torch.int32, device="cuda"))
    q = randn(gen, 1, 3, 128, dtype=dtype)
    out = torch.empty_like(q)
    mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 3)))
    check(cache, q, [1], out, None, None)
    pages.zero_()
    assert (buffer == 0).all()                            # nothing outside of the view was written
    none = mq.moqae_paged4_bind(torch.empty(0, 2, 2560, dtype=torch.uint8, device="cuda"), torch.zeros(2, 4, dtype=torch.int32, device="cuda"),
                                torch.tensor([0, 5], dtype=torch.int32, device="cuda"), dtype)
    q = randn(gen, 2, 4, 128, dtype=dtype)
    out, work = torch.full_like(q, 3.0), space(mq.moqae_paged4_prefill_attn_workspace(none, 4, 300))
    mq.moqae_paged4_decode_attn(none, q, out, work)       # five tokens without a page: zeros
    assert (out == 0).all() and none.status.tolist()[:3] == [mq.ERR_CORRUPT_TABLE, 1, 0]
    q = randn(gen, 300, 4, 128, dtype=dtype)
    out = torch.full_like(q, 3.0)
    mq.moqae_paged4_prefill_attn(none, q, torch.tensor([0, 0, 300], dtype=torch.int32, device="cuda"), out, work)
    assert (out == 0).all()


def test_tensors_that_do_not_fit_are_refused():
    gen = generator(43)
    cache = make_cache(gen, [40, 20], 2, 16, torch.bfloat16)
    b = torch.bfloat16
    q, k, work = randn(gen, 2, 4, 128, dtype=b), randn(gen, 2, 2, 128, dtype=b), space(mq.moqae_paged4_prefill_attn_workspace(cache, 4, 2))
    pos, cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    other = mq.make_rope(None, 0, k_weight=torch.ones(128, dtype=torch.float16, device="cuda"))
    pool = mq.make_page_pool(8)
    before, lens = cache.pages.clone(), cache.kv_len.clone()
    refused = [
        lambda: mq.moqae_paged4_append(cache, k.half(), k, pos), lambda: mq.moqae_paged4_append(cache, k, k[:1], pos),
        lambda: mq.moqae_paged4_append(cache, k, k, pos.long()), lambda: mq.moqae_paged4_append(cache, k, k, pos, rope=other),
        lambda: mq.moqae_paged4_append(cache, q, k, pos), lambda: mq.moqae_paged4_append(cache, k.cpu(), k, pos),
        lambda: mq.moqae_paged4_read(cache, None, None, pos), lambda: mq.moqae_paged4_read(cache, k, k.float(), pos),
        lambda: mq.moqae_paged4_decode_attn(cache, q[:1], q[:1], work), lambda: mq.moqae_paged4_decode_attn(cache, q, q, work[1:]),
        lambda: mq.moqae_paged4_decode_attn(cache, q, q, work[:1 << 20]), lambda: mq.moqae_paged4_decode_attn(cache, q, q, None),
        lambda: mq.moqae_paged4_prefill_attn(cache, q, cu[:2], q, work), lambda: mq.moqae_paged4_prefill_attn(cache, q, cu, q, None),
        lambda: mq.moqae_paged4_prefill_attn(cache, q[..., ::2], cu, q, work), lambda: mq.moqae_paged4_prefill_attn(cache, q[:, :3], cu, q, work),
        lambda: mq.moqae_paged_plan(cache, pool, pos.long(), cu, pos, pos), lambda: mq.moqae_paged_plan(cache, pool, pos, cu[:2], pos, pos),
        lambda: mq.moqae_paged_plan(cache, pool, pos, cu, pos, pos[:1]), lambda: mq.moqae_paged_plan(cache, mq.PagePool(pool.ring, pool.state[:3]), pos, cu, pos, pos),
        lambda: mq.moqae_paged4_bind(cache.pages[:, :, :100], cache.block_table, cache.kv_len, b),
        lambda: mq.moqae_paged4_bind(cache.pages, cache.block_table, cache.kv_len, torch.float32),
        lambda: mq.moqae_paged4_bind(cache.pages, cache.block_table, cache.kv_len[:1], b),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(mq.MoqaeError):
            call()
            raise AssertionError(i)
    torch.cuda.synchronize()
    assert (cache.pages == before).all() and (cache.kv_len == lens).all() and cache.status[0].item() == 0


def test_sequences_that_share_rows_are_refused():
    gen = generator(22)
    cache = make_cache(gen, [40, 40], 1, 16, torch.float16)
    q = randn(gen, 8, 4, 128, dtype=torch.float16)
    out, work = torch.full_like(q, 3.0), space(mq.moqae_paged4_prefill_attn_workspace(cache, 4, 8))
    cu = torch.tensor([0, 8, 0], dtype=torch.int32, device="cuda")         # the second ends before it starts: no tokens
    mq.moqae_paged4_prefill_attn(cache, q, cu, out, work)
    check(cache, q, [8], out, None, None)
    cu = torch.tensor([0, 1 << 20, 1 << 20], dtype=torch.int32, device="cuda")
    mq.moqae_paged4_prefill_attn(cache, q, cu, out, work)
    check(cache, q, [8], out, None, None)
    assert cache.status[0].item() == 0
    # rows 0..7 and again 4..7: no results, whoever takes the sequences
    for n, heads in ((8, 4), (80, 4), (200, 1)):
        cache = make_cache(gen, [400, 400, 400], 1, 16, torch.float16)
        q = randn(gen, n, heads, 128, dtype=torch.float16)
        out, work = torch.full_like(q, 3.0), space(mq.moqae_paged4_prefill_attn_workspace(cache, heads, n))
        mq.moqae_paged4_prefill_attn(cache, q, torch.tensor([0, n, n // 2, n], dtype=torch.int32, device="cuda"), out, work)
        assert cache.status.tolist()[:3] == [mq.ERR_INVALID_ARG, -1, n + n // 2] and (out == 3).all() and (work[:1 << 20] == 0).all()


# ---- streams, graphs ---------------------------------------------------------------------------

def test_streams_and_graphs():
    gen = generator(31)
    lens, hq, hkv = [300, 5, 1000], 8, 2
    cache = make_cache(gen, lens, hkv, 16, torch.bfloat16, max_pages=70)
    q = randn(gen, 3, hq, 128, dtype=torch.bfloat16)
    want, work = torch.empty_like(q), space(mq.moqae_paged4_decode_attn_workspace(cache, hq))
    mq.moqae_paged4_decode_attn(cache, q, want, work)
    torch.cuda.synchronize()
    outs, streams = [torch.zeros_like(q) for _ in range(3)], [torch.cuda.Stream() for _ in range(3)]
    works = [torch.zeros_like(work) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, w in zip(streams, outs, works):
            with torch.cuda.stream(s):
                mq.moqae_paged4_decode_attn(cache, q, o, w)
    torch.cuda.synchronize()
    assert all((o == want).all() for o in outs)
    # a captured step reads lengths and tables of the time it is replayed
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    k, v = (randn(gen, 3, hkv, 128, dtype=torch.bfloat16) for _ in range(2))
    pool = mq.make_page_pool(cache.pages.shape[0])
    pool.ring[:2] = torch.tensor([i for i in range(cache.pages.shape[0]) if i not in cache.block_table.flatten().tolist()][:2], dtype=torch.int32)
    pool.state[:2] = torch.tensor([0, 2], dtype=torch.int32)
    n_new = torch.ones(3, dtype=torch.int32, device="cuda")
    cu, pos, seq = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3, 3))
    with torch.cuda.graph(graph):
        mq.moqae_paged_plan(cache, pool, n_new, cu, pos, seq)
        mq.moqae_paged4_append(cache, k, v, pos, seq=seq)
        mq.moqae_paged4_decode_attn(cache, q, out, work)
    for step in range(3):
        q.copy_(randn(gen, 3, hq, 128, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        assert cache.kv_len.tolist() == [n + step + 1 for n in lens] and cache.status[0].item() == 0
        check(cache, q, [1, 1, 1], out, None, None)


def test_captured_prompts_follow_their_offsets():
    """Two captured calls of different sizes share a workspace; which sequences bring few rows and which many is decided at the replay."""
    gen = generator(32)
    lens, hq, hkv = [400, 300, 900, 31], 8, 2
    cache = make_cache(gen, lens, hkv, 64, torch.float16)
    calls = []
    work = space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, 500))
    for n in (500, 200):
        q, cu = randn(gen, n, hq, 128, dtype=torch.float16), torch.zeros(5, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q)
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, work)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mq.moqae_paged4_prefill_attn(cache, q, cu, out, work)
        calls.append((n, q, cu, out, graph))
    for first, second in (([300, 1, 100, 31], [1, 1, 190, 8]), ([1, 250, 0, 2], [150, 0, 25, 24]), ([0, 0, 499, 1], [50, 50, 50, 31]), ([0, 0, 0, 0], [1, 0, 0, 0])):
        for (n, q, cu, out, graph), new in zip(calls, (first, second)):
            cu.copy_(torch.tensor([0] + new).cumsum(0).to(torch.int32))
            out.fill_(9.0)
        for call in calls:
            call[4].replay()
        torch.cuda.synchronize()
        for (n, q, cu, out, graph), new in zip(calls, (first, second)):
            check(cache, q[:sum(new)], new, out[:sum(new)], None, None, what=str(new))
            assert (out[sum(new):] == 9).all()
    assert cache.status[0].item() == 0 and (work[:1 << 20] == 0).all()
