"""Operators of a paged cache held in 4 bits, as cases to measure.

Beside the quantised cache of whole chunks and the cache of 16-bit pages stands a cache of pages whose keys and
values are held in 4 bits, for sequences of any lengths that grow token by token:

  plan      block tables, query offsets and the sequence and position of every new token, from the
            lengths that sequences have and the tokens that they bring (or give back), pages from a pool
  append    norm and rotation of new tokens, their keys and values quantised into their pages; and the
            cached rows read back as the values they stand for
  decode    attention of one new token per sequence over its 4-bit pages
  prefill   the same for several new tokens per sequence

A row of 128 channels is four groups of 32; a group keeps z, the largest fp16 value not above its smallest
element, s, the smallest fp16 value not below (largest element - z) / 15, and for every element x the whole
number nearest to (x - z) * r (halves to even), r being the float32 value nearest to 1 / s (the package's rule for
chunks, too), which stands for z + s * code.

`run` computes them in plain torch operations in 32 bits, or (own = True) through the package.  Head counts and
contexts are those of the package's workloads (8, 32 and 40 heads of 128 channels, 32 query heads on 8 key
heads, contexts of 4k to 128k tokens).
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
TILE = 16                        # tokens that are stored together
TOKEN_BYTES = 160                # of a token and head: 64 code bytes and 16 of scales and zeros, for keys and for values
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases -------------------------------------------------------------------------------------

def listed():
    return [
        # a serving step: nearly every sequence brings one token, some have ended and leave
        dict(name="plan_step", op="plan", batch=61, new_min=1, new_max=1, past_min=16, past_max=32000, page=16, leave=0.1, start=0.0,
             pad=64, shapes=1),
        # a turn of the batch: prompts enter, others leave, the rest go on
        dict(name="plan_prompts", op="plan", batch=96, new_min=200, new_max=9000, past_min=16, past_max=32000, page=16, leave=0.1,
             start=0.3, pad=1024, shapes=2),
        # one step of a serving batch of odd size
        dict(name="append4_step", op="append", batch=61, new_min=1, new_max=1, past_min=16, past_max=32000, hq=32, hkv=8, dtype="bf16",
             page=16, rot=128, interleaved=False, norm=True, shapes=3),
        # several prompts of different lengths entering the cache together; half of each head rotated
        dict(name="append4_prompts", op="append", batch=7, new_min=200, new_max=9000, past_min=1, past_max=4000, hq=40, hkv=40,
             dtype="fp16", page=64, rot=64, interleaved=False, norm=False, shapes=4),
        # one user, a short conversation: nothing but latency
        dict(name="decode4_one", op="decode", batch=1, len_min=333, len_max=333, hq=8, hkv=8, dtype="fp16", page=16, cap=0.0, window=0,
             alibi=False, prefix_max=0, shapes=5),
        # a serving batch whose lengths differ by three orders of magnitude
        dict(name="decode4_ragged", op="decode", batch=61, len_min=1, len_max=32000, hq=32, hkv=8, dtype="bf16", page=16, cap=0.0,
             window=0, alibi=False, prefix_max=0, shapes=6),
        # four 128k contexts, the package's own large decode workload with every chunk at 4 bits
        dict(name="decode4_128k", op="decode", batch=4, len_min=131001, len_max=131071, hq=32, hkv=8, dtype="bf16", page=64, cap=0.0,
             window=0, alibi=False, prefix_max=0, shapes=7),
        # multi-head model with capped scores and a sliding window over long contexts
        dict(name="decode4_window", op="decode", batch=24, len_min=3000, len_max=32768, hq=40, hkv=40, dtype="fp16", page=32, cap=30.0,
             window=4096, alibi=False, prefix_max=64, shapes=8),
        # a few proposed tokens per sequence checked in one pass
        dict(name="prefill4_few", op="prefill", batch=8, new_min=1, new_max=8, past_min=100, past_max=4096, hq=32, hkv=8, dtype="bf16",
             page=16, cap=0.0, window=0, alibi=False, prefix_max=0, shapes=9),
        # the next 512 tokens of a prompt that is 32k tokens in
        dict(name="prefill4_chunk", op="prefill", batch=1, new_min=512, new_max=512, past_min=32100, past_max=32100, hq=32, hkv=8,
             dtype="bf16", page=64, cap=0.0, window=0, alibi=False, prefix_max=0, shapes=10),
        # prompts of a model with a distance bias and capped scores, each with a prefix seen by all of it
        dict(name="prefill4_biased", op="prefill", batch=5, new_min=300, new_max=4096, past_min=0, past_max=0, hq=40, hkv=40,
             dtype="fp16", page=128, cap=30.0, window=0, alibi=True, prefix_max=200, shapes=11),
        # one long prompt of the grouped-query model
        dict(name="prefill4_long", op="prefill", batch=1, new_min=16300, new_max=16300, past_min=0, past_max=0, hq=32, hkv=8,
             dtype="bf16", page=64, cap=0.0, window=0, alibi=False, prefix_max=0, shapes=12),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(("plan", "append", "decode", "decode", "prefill", "prefill"))
    shapes = rng.randrange(1 << 20)
    if op == "plan":
        batch = _spread(rng, 1, 256)
        return dict(op=op, batch=batch, new_min=1, new_max=rng.choice((1, _spread(rng, 2, max(2, 100000 // batch)))), past_min=1,
                    past_max=_spread(rng, 16, 32000), page=rng.choice((16, 32, 64, 128, 256)), leave=rng.choice((0.0, 0.1, 0.3)),
                    start=rng.choice((0.0, 0.3, 1.0)), pad=rng.choice((1, 8, 256)), shapes=shapes)
    hq, hkv = rng.choice(((8, 8), (8, 2), (32, 32), (32, 8), (40, 40)))
    base = dict(op=op, hq=hq, hkv=hkv, dtype=rng.choice(("bf16", "fp16")), page=rng.choice((16, 32, 64, 128, 256)), shapes=shapes)
    masks = dict(cap=rng.choice((0.0, 0.0, 30.0, 50.0)), window=rng.choice((0, 0, _spread(rng, 100, 8192))),
                 alibi=rng.random() < 0.3, prefix_max=rng.choice((0, 0, _spread(rng, 4, 300))))
    if op == "append":
        batch, step = _spread(rng, 1, 128), rng.random() < 0.5
        most = 1 if step else max(2, 16000 // batch)
        return dict(base, batch=batch, new_min=1, new_max=most, past_min=1, past_max=_spread(rng, 10, 8000 if batch < 32 else 1000),
                    rot=rng.choice((64, 96, 128, 128)), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5)
    if op == "decode":
        batch = _spread(rng, 1, 128)
        longest = min(131072, (4 * 131072 * 8) // (batch * hkv))
        return dict(base, **masks, batch=batch, len_min=1, len_max=_spread(rng, 64, max(64, longest // 2)))
    batch = _spread(rng, 1, 16)
    new = _spread(rng, 1, max(8, 8000 // batch))
    return dict(base, **masks, batch=batch, new_min=max(1, new // 4), new_max=new, past_min=0,
                past_max=rng.choice((0, _spread(rng, 10, 4000))))


def _ints(rng, count, low, high):
    """`count` whole numbers spread over the logarithm of low .. high, the largest first."""
    if high <= low:
        return [low] * count
    return [high] + [_spread(rng, max(1, low), high) if low > 0 or rng.random() > 0.1 else 0 for _ in range(count - 1)]


def _shapes(case):
    """(new tokens, earlier tokens, prefix) of every sequence; new < 0: it leaves."""
    rng = random.Random(case["shapes"])
    batch = case["batch"]
    if case["op"] == "decode":
        total = _ints(rng, batch, case["len_min"], case["len_max"])
        new, past = [1] * batch, [n - 1 for n in total]
    else:
        new = _ints(rng, batch, case["new_min"], case["new_max"])
        past = _ints(rng, batch, case["past_min"], case["past_max"])
    if case["op"] == "plan":
        for b in range(batch):
            if rng.random() < case["start"]:
                past[b] = 0                              # a prompt of its own
            elif rng.random() < case["leave"]:
                new[b] = -past[b]
            else:
                new[b] = 1
    most = case.get("prefix_max", 0)
    prefix = [min(p + n, rng.randint(0, most)) if most else 0 for n, p in zip(new, past)]
    return new, past, prefix


# ---- the stored form -----------------------------------------------------------------------------

def _order():
    """int64 [16, 160]: where in its tile's 2560 bytes token t keeps, in this order, its key codes (64 bytes: eight
    channels of a quarter's group beside those of the other groups), key scales and zeros (16), value codes
    (64: four channels of every group), value scales and zeros (16)."""
    t = torch.arange(TILE)[:, None]
    i = torch.arange(64)[None]
    row = (t & 8) | ((t & 1) << 2) | ((t >> 1) & 3)
    half = torch.arange(16)[None]                        # byte of a scale or zero: which = half // 2
    keys = torch.cat([64 * t + i, 1024 + 16 * t + half], 1)
    values = torch.cat([1280 + (i >> 5) * 512 + 32 * row + (i & 31), 2304 + 32 * (t >> 1) + 4 * (half >> 1) + 2 * (t & 1) + (half & 1)], 1)
    return torch.cat([keys, values], 1)


def _half_down(x):
    """The largest fp16 value not above x, as fp16 (-0 as +0)."""
    h = x.half()
    bits = h.view(torch.int16)
    below = torch.where(h == 0, torch.full_like(bits, -32767), torch.where(h > 0, bits - 1, bits + 1)).view(torch.float16)
    h = torch.where(h.float() > x, below, h)
    return torch.where(h == 0, torch.zeros_like(h), h)


def _half_up(x):
    """The smallest fp16 value not below x >= 0, as fp16."""
    h = x.half()
    return torch.where(h.float() < x, (h.view(torch.int16) + 1).view(torch.float16), h)


def _quantise(x):
    """Rows [..., 128] in float32: codes uint8 [..., 4, 32], scales and zeros fp16 [..., 4]."""
    x = x.unflatten(-1, (4, 32))
    z = _half_down(x.amin(-1))
    span = x.amax(-1) - z.float()
    s = _half_up(span / torch.full_like(span, 15.0))     # (by a plain number torch multiplies with its reciprocal)
    inv = torch.where(s == 0, 0.0, 1.0 / s.float())
    code = torch.round((x - z.float()[..., None]).double().mul_(inv.double()[..., None]))   # (the product as it is: ties are common)
    return code.clamp_(0, 15).to(torch.uint8), s, z


def _token_bytes(k, v):
    """uint8 [..., 160] of key and value rows [..., 128] in float32."""
    out = []
    for x, units in ((k, 4), (v, 8)):
        code, s, z = _quantise(x)
        pair = code.unflatten(-1, (units, -1, 2))                          # [..., group, unit, byte, nibble]
        byte = (pair[..., 0] | (pair[..., 1] << 4)).transpose(-3, -2)      # [..., unit, group, byte]
        out += [byte.flatten(-3), torch.cat([s, z], -1).contiguous().view(torch.uint8)]
    return torch.cat(out, -1)


def _rows(part, units):
    """float32 [..., 128] that 80 bytes of a token stand for."""
    byte = part[..., :64].unflatten(-1, (units, 4, -1)).transpose(-3, -2)  # [..., group, unit, byte]
    code = torch.stack([byte & 15, byte >> 4], -1).flatten(-3)             # [..., group, 32]
    s, z = part[..., 64:].contiguous().view(torch.float16).float().split(4, -1)
    return code.float().mul_(s[..., None]).add_(z[..., None]).flatten(-2)


# ---- inputs ------------------------------------------------------------------------------------

def _rope_table(n, rot):
    """[n][rot] float32: cosines, then sines, of position * 10000^(-2 i / rot), taken in 64 bits."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _randn(gen, *shape, dtype):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda"))
    return out


def _tables(case, gen, total):
    """A block table over pages in no order, and the number of pages."""
    page, batch = case["page"], case["batch"]
    need = [(n + page - 1) // page for n in total]
    n_pages, width = sum(need) + 3, max(1, max(need))
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _pages(case, gen, n_pages):
    """uint8 [n_pages, hkv, page * 160] with normal keys and values; rows behind a sequence's last token hold what
    earlier sequences left there."""
    hkv, tiles = case["hkv"], case["page"] // TILE
    out = torch.empty((n_pages, hkv, case["page"] * TOKEN_BYTES), dtype=torch.uint8, device="cuda")
    back = torch.argsort(_order().flatten()).cuda()
    step = max(1, (1 << 19) // (hkv * case["page"]))
    for at in range(0, n_pages, step):
        part = out[at:at + step]
        k, v = (torch.randn((part.shape[0], hkv, tiles, TILE, HEAD_DIM), generator=gen, device="cuda") for _ in range(2))
        part.copy_(_token_bytes(k, v).flatten(-2).index_select(-1, back).flatten(-2))
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = dict(case=case, order=_order().cuda())
    new, past, prefix = _shapes(case)
    if case["op"] == "plan":
        return _prepare_plan(s, gen, new, past)
    dtype, hq, hkv = DTYPES[case["dtype"]], case["hq"], case["hkv"]
    total = [a + b for a, b in zip(new, past)]
    s["table"], n_pages = _tables(case, gen, total)
    s["pages"], s["kv_len"] = _pages(case, gen, n_pages), torch.tensor(total, dtype=torch.int32, device="cuda")
    n = sum(new)
    cu = [0]
    for a in new:
        cu.append(cu[-1] + a)
    s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    if own:
        from paper_2506_07533_b200 import binding as mq
        s["cache"] = mq.moqae_paged4_bind(s["pages"], s["table"], s["kv_len"], dtype)
    if case["op"] == "append":
        weight = (lambda: (1.0 + 0.1 * torch.randn(HEAD_DIM, generator=gen, device="cuda")).to(dtype)) if case["norm"] else (lambda: None)
        # queries, keys and values of a token leave the projection side by side
        qkv = _randn(gen, n, (hq + 2 * hkv), HEAD_DIM, dtype=dtype)
        s.update(cos_sin=_rope_table(max(total), case["rot"]), q_weight=weight(), k_weight=weight(), eps=1e-6, q=qkv[:, :hq],
                 k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:])
        s["positions"] = torch.cat([torch.arange(p, p + a, dtype=torch.int32, device="cuda") for a, p in zip(new, past)])
        s["seq"] = torch.repeat_interleave(torch.arange(len(new), dtype=torch.int32, device="cuda"), torch.tensor(new, device="cuda"))
        s["q_out"] = torch.empty((n, hq, HEAD_DIM), dtype=dtype, device="cuda")
        s["k_out"], s["v_out"] = (torch.empty((n, hkv, HEAD_DIM), dtype=dtype, device="cuda") for _ in range(2))
        if own:
            s["rope"] = mq.make_rope(s["cos_sin"], case["rot"], interleaved=case["interleaved"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=s["eps"])
        return s
    s["q"] = _randn(gen, n, hq, HEAD_DIM, dtype=dtype)
    s["out"] = torch.empty((n, hq, HEAD_DIM), dtype=dtype, device="cuda")
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda") / hq).float() if case["alibi"] else None
    s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda") if case["prefix_max"] else None
    s["scale"] = 1.0 / math.sqrt(HEAD_DIM)
    s["new"], s["total"] = new, total
    if own:
        s["options"] = mq.make_attn_options(scale=s["scale"], cap=case["cap"], window=case["window"], slopes=s["slopes"],
                                            prefix_len=s["prefix"])
        size = (mq.moqae_paged4_decode_attn_workspace(s["cache"], hq) if case["op"] == "decode" else
                mq.moqae_paged4_prefill_attn_workspace(s["cache"], hq, n))
        s["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return s


def _prepare_plan(s, gen, new, past):
    case = s["case"]
    page, batch, pad = case["page"], case["batch"], case["pad"]
    have = [(p + page - 1) // page for p in past]
    want = [(max(0, p + n) + page - 1) // page for n, p in zip(new, past)]
    width = max(max(have), max(want), 1) + 1
    used, take = sum(have), sum(max(0, w - h) for w, h in zip(want, have))
    n_pages = used + 2 * take + 8
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    s["table"] = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(have):
        s["table"][b, :n] = order[at:at + n]
        at += n
    # the pool is a ring of page numbers: `state` says where the free ones begin and how many they are
    head = int(torch.randint(0, n_pages, (1,), generator=gen, device="cuda"))
    s["ring"] = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    s["ring"][(head + torch.arange(n_pages - used, device="cuda")) % n_pages] = order[used:]
    s["state"] = torch.tensor([head, n_pages - used, 0, 0], dtype=torch.int32, device="cuda")
    s["state_out"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    rows = max(1, (sum(max(0, n) for n in new) + pad - 1) // pad * pad)
    s["past"], s["n_new"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (past, new))
    s["kv_len"], s["cu_q"] = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (batch, batch + 1))
    s["positions"], s["seq"] = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    s["rows"], s["take"], s["give"] = rows, take, sum(max(0, h - w) for w, h in zip(want, have))
    if own:
        from paper_2506_07533_b200 import binding as mq
        pages = torch.empty((n_pages, 1, page * TOKEN_BYTES), dtype=torch.uint8, device="cuda")
        s["cache"] = mq.moqae_paged4_bind(pages, s["table"], s["kv_len"], torch.bfloat16)
        s["pool"] = mq.PagePool(s["ring"], s["state_out"])
    return s


# ---- plain forms -------------------------------------------------------------------------------

def _plan_plain(s):
    page, past, n_new = s["case"]["page"], s["past"].long(), s["n_new"].long()
    batch, width = s["table"].shape
    n_pages, (head, free) = s["ring"].shape[0], s["state"].long()[:2]
    total = (past + n_new).clamp_min(0)
    have, want = (past + page - 1) // page, (total + page - 1) // page
    zero = torch.zeros(1, dtype=torch.long, device="cuda")
    cu_q = torch.cat([zero, n_new.clamp_min(0).cumsum(0)])
    t = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(cu_q[1:].contiguous(), t, right=True)
    live = t < cu_q[-1]
    at = b.clamp_max(batch - 1)
    positions = torch.where(live, past[at] + t - cu_q[at], -1)
    seq = torch.where(live, at, -1)
    give, take = (have - want).clamp_min(0), (want - have).clamp_min(0)
    ring, table = s["ring"].clone(), s["table"].clone()
    # pages that are given back follow the free ones, in the order of sequences and entries
    j, cu = torch.arange(s["give"], device="cuda"), give.cumsum(0)
    b = torch.searchsorted(cu, j, right=True)
    ring[(head + free + j) % n_pages] = table[b, want[b] + j - (cu[b] - give[b])]
    j, cu = torch.arange(s["take"], device="cuda"), take.cumsum(0)
    b = torch.searchsorted(cu, j, right=True)
    table[b, have[b] + j - (cu[b] - take[b])] = ring[(head + j) % n_pages]
    state = torch.stack([(head + take.sum()) % n_pages, free - take.sum() + give.sum()])
    return tuple(x.to(torch.int32) for x in (table, total, cu_q, positions, seq, ring, state))


def _norm_rotate(x, weight, s):
    """Rows [n][heads][128] in float32 after the norm (where there is a weight) and the rotation."""
    case, x = s["case"], x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
    rot = case["rot"]
    cos, sin = s["cos_sin"][s["positions"].long()][:, None].split(rot // 2, -1)
    turned, rest = x[..., :rot], x[..., rot:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = turned.split(rot // 2, -1)
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, rest], -1)


def _append_plain(s):
    dtype, page = DTYPES[s["case"]["dtype"]], s["case"]["page"]
    q, k = (_norm_rotate(s[x], s[x + "_weight"], s) for x in ("q", "k"))
    pos = s["positions"].long()
    entry, slot = s["table"][s["seq"].long(), pos // page].long(), pos % page
    tiles = s["pages"].unflatten(-1, (page // TILE, TILE * TOKEN_BYTES))
    where = (entry[:, None], slice(None), (slot // TILE)[:, None], s["order"][slot % TILE])
    tiles[where] = _token_bytes(k, s["v"].float()).transpose(1, 2)         # [token, byte, head]
    back = tiles[where].transpose(1, 2)
    return q.to(dtype), _rows(back[..., :80], 4).to(dtype), _rows(back[..., 80:], 8).to(dtype)


def _visible(pos, keys, kv_len, window, prefix):
    """Whether a query at `pos` sees the token at `keys`."""
    seen = keys <= pos
    if window:
        seen = seen & (pos - keys < window)
    if prefix is not None:
        seen = seen | (keys < prefix)
    return seen & (keys < kv_len)


def _scores(s, score, distance, slopes):
    case = s["case"]
    score = score * s["scale"]
    if case["cap"] > 0:
        score = case["cap"] * torch.tanh(score / case["cap"])
    if slopes is not None:
        score = score - slopes * distance.abs()
    return score


def _softmax(score, seen):
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    total = weight.sum(-1, keepdim=True)
    return torch.where(total > 0, weight / total.clamp_min(1e-30), 0.0)


def _gather(s, table):
    """Keys and values [..., hkv, tokens, 128] of the pages in `table` [..., pages] in float32."""
    tiles = s["pages"].unflatten(-1, (-1, TILE * TOKEN_BYTES))[table].transpose(-4, -3).flatten(-3, -2)
    part = lambda a, b: tiles.index_select(-1, s["order"][:, a:b].flatten()).unflatten(-1, (TILE, -1)).flatten(-3, -2)  # noqa: E731
    return _rows(part(0, 80), 4), _rows(part(80, 160), 8)


def _decode_plain(s):
    case = s["case"]
    hq, hkv, batch = case["hq"], case["hkv"], case["batch"]
    keys, values = _gather(s, s["table"].clamp_min(0).long())
    at = torch.arange(keys.shape[2], device="cuda")
    length = s["kv_len"][:, None, None, None]
    pos = length - 1
    prefix = None if s["prefix"] is None else s["prefix"][:, None, None, None]
    q = s["q"].float().view(batch, hkv, hq // hkv, HEAD_DIM)
    slopes = None if s["slopes"] is None else s["slopes"].view(1, hkv, hq // hkv, 1)
    score = _scores(s, q @ keys.transpose(-1, -2), pos - at, slopes)
    p = _softmax(score, _visible(pos, at, length, case["window"], prefix))
    return (p @ values).reshape(batch, hq, HEAD_DIM)


def _prefill_plain(s):
    case = s["case"]
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    group, done, out = hq // hkv, 0, []
    for b, (n, total) in enumerate(zip(s["new"], s["total"])):      # sequences share nothing
        keys, values = (x[:, :total] for x in _gather(s, s["table"][b, :(total + page - 1) // page].long()))
        pos = torch.arange(total - n, total, device="cuda")[:, None]
        at = torch.arange(total, device="cuda")
        seen = _visible(pos, at, total, case["window"], None if s["prefix"] is None else s["prefix"][b])
        q = s["q"][done:done + n].float().view(n, hkv, group, HEAD_DIM).permute(1, 2, 0, 3)
        rows = torch.empty((n, hkv, group, HEAD_DIM), device="cuda")
        step = max(1, (1 << 31) // (group * n * total))             # key heads whose scores fit beside each other
        for h in range(0, hkv, step):
            slopes = None if s["slopes"] is None else s["slopes"].view(hkv, group, 1, 1)[h:h + step]
            score = _scores(s, q[h:h + step] @ keys[h:h + step, None].transpose(-1, -2), pos - at, slopes)
            rows[:, h:h + step] = (_softmax(score, seen) @ values[h:h + step, None]).permute(2, 0, 1, 3)
        out.append(rows.view(n, hq, HEAD_DIM))
        done += n
    return torch.cat(out)


def run(s):
    case = s["case"]
    if own:
        from paper_2506_07533_b200 import binding as mq
        if case["op"] == "plan":
            mq.moqae_paged_plan(s["cache"], s["pool"], s["n_new"], s["cu_q"], s["positions"], s["seq"], past_len=s["past"],
                                pool_state=s["state"])
            return s["table"], s["kv_len"], s["cu_q"], s["positions"], s["seq"], s["ring"], s["state_out"][:2]
        if case["op"] == "append":
            mq.moqae_paged4_append(s["cache"], s["k"], s["v"], s["positions"], seq=s["seq"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
            mq.moqae_paged4_read(s["cache"], s["k_out"], s["v_out"], s["positions"], seq=s["seq"])
            return s["q_out"], s["k_out"], s["v_out"]
        if case["op"] == "decode":
            mq.moqae_paged4_decode_attn(s["cache"], s["q"], s["out"], s["workspace"], s["options"])
        else:
            mq.moqae_paged4_prefill_attn(s["cache"], s["q"], s["cu_q"], s["out"], s["workspace"], s["options"])
        return s["out"]
    if case["op"] == "plan":
        return _plan_plain(s)
    if case["op"] == "append":
        return _append_plain(s)
    return (_decode_plain(s) if case["op"] == "decode" else _prefill_plain(s)).to(DTYPES[case["dtype"]])


# ---- what a pass cannot do without -------------------------------------------------------------

def _seen_pairs(n, total, window, prefix):
    """(visible (query, key) pairs, keys that some query sees) of one sequence."""
    pairs, first = 0, total
    for pos in range(total - n, total):
        low = max(0, pos - window + 1) if window else 0
        first = min(first, low)
        head = min(prefix, total)
        pairs += (pos + 1 - low) + (head if head <= low else head - min(head, pos + 1) + low)
    return pairs, total - max(0, first - min(prefix, total))


def work(case):
    new, past, prefix = _shapes(case)
    if case["op"] == "plan":
        page = case["page"]
        n = sum(max(0, x) for x in new)
        moved = sum(abs((max(0, p + x) + page - 1) // page - (p + page - 1) // page) for x, p in zip(new, past))
        rows = (n + case["pad"] - 1) // case["pad"] * case["pad"]
        return dict(bytes=case["batch"] * 16 + 4 + rows * 8 + moved * 8 + 16, flops=8 * case["batch"] + 4 * rows + 4 * moved)
    hq, hkv, row, n = case["hq"], case["hkv"], HEAD_DIM * 2, sum(new)
    if case["op"] == "append":
        made = 2 * hq * row + hkv * (2 * row + TOKEN_BYTES)
        read = hkv * (TOKEN_BYTES + 2 * row)
        return dict(bytes=n * (made + read + 4 * case["rot"] + 16), flops=n * ((hq + hkv) * HEAD_DIM * 7 + hkv * HEAD_DIM * 14))
    pairs = keys = 0
    for a, p, f in zip(new, past, prefix):
        x, y = _seen_pairs(a, a + p, case["window"], f)
        pairs, keys = pairs + x, keys + y
    return dict(bytes=keys * hkv * TOKEN_BYTES + n * hq * 2 * row, flops=4 * pairs * hq * HEAD_DIM)


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_turned(x, weight, s):
    """The norm and the rotation as a product of complex numbers."""
    case, rot = s["case"], s["case"]["rot"]
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / HEAD_DIM + s["eps"]) * weight.double()
    table = s["cos_sin"].double()[s["positions"].long()]
    turn = torch.complex(table[:, :rot // 2], table[:, rot // 2:])[:, None]
    out = y.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_stored(x):
    """What rows [..., 128] in float64 become: zero and scale searched among all finite fp16 values."""
    bits = torch.arange(-32768, 32768, device="cuda").to(torch.int16).view(torch.float16).double()
    line = torch.unique(bits[torch.isfinite(bits)])
    out = torch.empty_like(x)
    for g in range(4):
        part = x[..., 32 * g:32 * g + 32]
        low, high = part.min(-1).values, part.max(-1).values
        z = line[torch.searchsorted(line, low.contiguous(), right=True) - 1]
        s = line[torch.searchsorted(line, ((high - z) / 15).contiguous())]
        r = torch.where(s > 0, (1.0 / torch.where(s > 0, s, 1.0)).float().double(), 0.0)
        code = torch.round((part - z[..., None]) * r[..., None])
        out[..., 32 * g:32 * g + 32] = z[..., None] + s[..., None] * code
    return out


def _exact_rows(s, b, h, which, tokens):
    """Keys (which = 0) or values (1) of tokens of sequence b, head h, in float64, byte by byte."""
    page = s["case"]["page"]
    slot = tokens % page
    tile = s["pages"][s["table"][b].long()[tokens // page], h].view(-1, page // TILE, TILE * TOKEN_BYTES)
    tile = tile[torch.arange(len(tokens), device="cuda"), slot // TILE].long()
    t, c = (slot % TILE)[:, None], torch.arange(HEAD_DIM, device="cuda")[None]
    g = c // 32
    if which == 0:
        at = 64 * t + 16 * (c % 32 // 8) + 4 * g + c % 8 // 2
        scale = 1024 + 16 * t + 2 * g
        zero = scale + 8
    else:
        unit = c % 32 // 4
        row = 8 * (t // 8) + 4 * (t % 2) + t % 8 // 2
        at = 1280 + 512 * (unit // 4) + 32 * row + 8 * (unit % 4) + 2 * g + c % 4 // 2
        scale = 2304 + 32 * (t // 2) + 4 * g + 2 * (t % 2)
        zero = scale + 16
    code = torch.where(c % 2 == 1, tile.gather(1, at) // 16, tile.gather(1, at) % 16)
    half = lambda where: (tile.gather(1, where) + 256 * tile.gather(1, where + 1)).to(torch.int16).view(torch.float16).double()  # noqa: E731
    return half(zero.expand_as(at)) + half(scale.expand_as(at)) * code.double()


def _exact_attention(s):
    """Head by head: sum of exp(score) v over the visible tokens, divided by sum of exp(score)."""
    case = s["case"]
    hq, hkv = case["hq"], case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    done = 0
    for b, (n, total) in enumerate(zip(s["new"], s["total"])):
        where = torch.arange(total, device="cuda")
        i = torch.arange(n, device="cuda")[:, None] + (total - n)
        allowed = where[None] <= i
        if case["window"]:
            allowed &= where[None] > i - case["window"]
        if s["prefix"] is not None:
            allowed |= where[None] < s["prefix"][b]
        for h in range(hkv):
            k, v = _exact_rows(s, b, h, 0, where), _exact_rows(s, b, h, 1, where)
            for g in range(hq // hkv):
                head = h * (hq // hkv) + g
                e = (s["q"][done:done + n, head].double() @ k.T).mul_(s["scale"])
                if case["cap"] > 0:
                    e = e.div_(case["cap"]).tanh_().mul_(case["cap"])
                if s["slopes"] is not None:
                    e -= s["slopes"][head].double() * (i - where[None]).abs()
                e = e.masked_fill_(~allowed, -math.inf)
                top = e.max(1, keepdim=True).values
                e = e.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
                norm = e.sum(1, keepdim=True)
                out[done:done + n, head] = (e @ v) / norm.masked_fill(norm == 0, 1.0)
        done += n
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return None                                      # whole numbers
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_turned(s["q"], s["q_weight"], s), _exact_stored(_exact_turned(s["k"], s["k_weight"], s)), _exact_stored(s["v"].double())
    return _exact_attention(s)
