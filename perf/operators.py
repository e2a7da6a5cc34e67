"""The paged 16-bit cache and its operators, as cases to measure.

Four operators work on one cache of 16-bit pages that stands beside the quantised one:

  norm_rope      RMS norm of every query and key head and the position rotation, one pass
  paged_append   the same for new tokens, their keys and values put into their pages
  paged_decode   attention of one new token per sequence over its pages
  paged_prefill  causal attention of several new tokens per sequence over its pages, with a
                 tanh cap, a distance bias, a window or a prefix that every token sees

`run` computes them in plain torch operations in 32 bits, or (own = True) through the package.
Head counts and contexts are those of the package's workloads (8, 32 and 40 heads of 128 channels,
32 query heads on 8 key heads, contexts of 4k to 128k tokens).
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases -------------------------------------------------------------------------------------

def listed():
    return [
        # one generated token of a grouped-query model: latency of the smallest call
        dict(name="rope_step", op="norm_rope", tokens=1, hq=32, hkv=8, dtype="bf16", rot=128, interleaved=False,
             norm=True, max_pos=131072),
        # a whole 32k prompt before it is quantised; multi-head, pairs next to each other, no norm
        dict(name="rope_prompt", op="norm_rope", tokens=32719, hq=32, hkv=32, dtype="fp16", rot=128, interleaved=True,
             norm=False, max_pos=32768),
        # one step of a serving batch of odd size
        dict(name="append_step", op="paged_append", batch=61, new_min=1, new_max=1, past_min=16, past_max=32000, hq=32,
             hkv=8, dtype="bf16", page=16, order="hsd", rot=128, interleaved=False, norm=True, shapes=1),
        # several prompts of different lengths entering the cache together; half of each head rotated
        dict(name="append_prompts", op="paged_append", batch=7, new_min=200, new_max=9000, past_min=1, past_max=4000,
             hq=40, hkv=40, dtype="fp16", page=64, order="shd", rot=64, interleaved=False, norm=False, shapes=2),
        # one user, a short conversation: nothing but latency
        dict(name="decode_one", op="paged_decode", batch=1, len_min=333, len_max=333, hq=8, hkv=8, dtype="fp16", page=16,
             order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=3),
        # a serving batch whose lengths differ by three orders of magnitude
        dict(name="decode_ragged", op="paged_decode", batch=61, len_min=1, len_max=32000, hq=32, hkv=8, dtype="bf16",
             page=16, order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=4),
        # four 128k contexts, the package's own large decode workload at 16 bits
        dict(name="decode_128k", op="paged_decode", batch=4, len_min=131001, len_max=131071, hq=32, hkv=8, dtype="bf16",
             page=64, order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=5),
        # multi-head model with capped scores and a sliding window over long contexts
        dict(name="decode_window", op="paged_decode", batch=24, len_min=3000, len_max=32768, hq=40, hkv=40, dtype="fp16",
             page=32, order="shd", cap=30.0, window=4096, alibi=False, prefix_max=64, shapes=6),
        # a few proposed tokens per sequence checked in one pass
        dict(name="prefill_few", op="paged_prefill", batch=8, new_min=1, new_max=8, past_min=100, past_max=4096, hq=32,
             hkv=8, dtype="bf16", page=16, order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=7),
        # the next 512 tokens of a prompt that is 32k tokens in
        dict(name="prefill_chunk", op="paged_prefill", batch=1, new_min=512, new_max=512, past_min=32100, past_max=32100,
             hq=32, hkv=8, dtype="bf16", page=64, order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=8),
        # prompts of a model with a distance bias and capped scores, each with a prefix seen by all of it
        dict(name="prefill_biased", op="paged_prefill", batch=5, new_min=300, new_max=4096, past_min=0, past_max=0, hq=40,
             hkv=40, dtype="fp16", page=128, order="shd", cap=30.0, window=0, alibi=True, prefix_max=200, shapes=9),
        # one long prompt of the grouped-query model
        dict(name="prefill_long", op="paged_prefill", batch=1, new_min=16300, new_max=16300, past_min=0, past_max=0, hq=32,
             hkv=8, dtype="bf16", page=64, order="hsd", cap=0.0, window=0, alibi=False, prefix_max=0, shapes=10),
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(("norm_rope", "paged_append", "paged_decode", "paged_decode", "paged_prefill", "paged_prefill"))
    hq, hkv = rng.choice(((8, 8), (8, 2), (32, 32), (32, 8), (40, 40)))
    base = dict(op=op, hq=hq, hkv=hkv, dtype=rng.choice(("bf16", "fp16")))
    rope = dict(rot=rng.choice((64, 96, 128, 128)), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5)
    pages = dict(page=rng.choice((16, 32, 64, 128)), order=rng.choice(("hsd", "shd")), shapes=rng.randrange(1 << 20))
    masks = dict(cap=rng.choice((0.0, 0.0, 30.0, 50.0)), window=rng.choice((0, 0, _spread(rng, 100, 8192))),
                 alibi=rng.random() < 0.3, prefix_max=rng.choice((0, 0, _spread(rng, 4, 300))))
    if op == "norm_rope":
        return dict(base, **rope, tokens=_spread(rng, 1, 16000), max_pos=rng.choice((4096, 32768, 131072)))
    if op == "paged_append":
        batch, step = _spread(rng, 1, 128), rng.random() < 0.5
        most = 1 if step else max(2, 16000 // batch)
        return dict(base, **rope, **pages, batch=batch, new_min=1, new_max=most, past_min=1, past_max=_spread(rng, 10, 8000 if batch < 32 else 1000))
    if op == "paged_decode":
        batch = _spread(rng, 1, 128)
        longest = min(131072, (4 * 131072 * 8) // (batch * hkv))
        return dict(base, **pages, **masks, batch=batch, len_min=1, len_max=_spread(rng, 64, max(64, longest // 2)))
    batch = _spread(rng, 1, 16)
    new = _spread(rng, 1, max(8, 8000 // batch))
    return dict(base, **pages, **masks, batch=batch, new_min=max(1, new // 4), new_max=new, past_min=0,
                past_max=rng.choice((0, _spread(rng, 10, 4000))))


def _ints(rng, count, low, high):
    """`count` whole numbers spread over the logarithm of low .. high, the largest first."""
    if high <= low:
        return [low] * count
    return [high] + [_spread(rng, max(1, low), high) if low > 0 or rng.random() > 0.1 else 0 for _ in range(count - 1)]


def _shapes(case):
    """(new tokens, earlier tokens, prefix) of every sequence."""
    rng = random.Random(case["shapes"])
    batch = case["batch"]
    if case["op"] == "paged_decode":
        total = _ints(rng, batch, case["len_min"], case["len_max"])
        new, past = [1] * batch, [n - 1 for n in total]
    else:
        new = _ints(rng, batch, case["new_min"], case["new_max"])
        past = _ints(rng, batch, case["past_min"], case["past_max"])
    most = case.get("prefix_max", 0)
    prefix = [min(p + n, rng.randint(0, most)) if most else 0 for n, p in zip(new, past)]
    return new, past, prefix


# ---- inputs ------------------------------------------------------------------------------------

def _rope_table(n, rot):
    """[n][rot] float32: cosines, then sines, of position * 10000^(-2 i / rot), taken in 64 bits."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _randn(gen, *shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda") * scale)
    return out


def _rope_state(case, gen, n_positions):
    dtype = DTYPES[case["dtype"]]
    weight = (lambda: (1.0 + 0.1 * torch.randn(HEAD_DIM, generator=gen, device="cuda")).to(dtype)) if case["norm"] else (lambda: None)
    return dict(cos_sin=_rope_table(n_positions, case["rot"]), q_weight=weight(), k_weight=weight(), eps=1e-6)


def _pages(case, gen, total):
    """Key and value pages, a block table over them in no order, the lengths. The rows behind a sequence's
    last token hold what earlier sequences left there."""
    page, hkv, batch = case["page"], case["hkv"], case["batch"]
    need = [(n + page - 1) // page for n in total]
    n_pages, width = sum(need) + 3, max(need)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (n_pages, hkv, page, HEAD_DIM) if case["order"] == "hsd" else (n_pages, page, hkv, HEAD_DIM)
    k = _randn(gen, *shape, dtype=DTYPES[case["dtype"]])
    v = _randn(gen, *shape, dtype=DTYPES[case["dtype"]])
    if case["order"] == "shd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return k, v, table, torch.tensor(total, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype, hq, hkv = DTYPES[case["dtype"]], case["hq"], case["hkv"]
    s = dict(case=case)
    if case["op"] == "norm_rope":
        n = case["tokens"]
        # queries, keys and values of a token leave the projection side by side
        qkv = _randn(gen, n, (hq + 2 * hkv), HEAD_DIM, dtype=dtype, scale=1.0 if case["norm"] is False else 1.7)
        s.update(_rope_state(case, gen, case["max_pos"]), q=qkv[:, :hq], k=qkv[:, hq:hq + hkv])
        first = int(torch.randint(0, case["max_pos"] - n + 1, (1,), generator=gen, device="cuda"))
        s["positions"] = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        s["q_out"], s["k_out"] = torch.empty((n, hq, HEAD_DIM), dtype=dtype, device="cuda"), torch.empty((n, hkv, HEAD_DIM), dtype=dtype, device="cuda")
        if own:
            from paper_2506_07533_b200 import binding as mq
            s["rope"] = mq.make_rope(s["cos_sin"], case["rot"], interleaved=case["interleaved"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=s["eps"])
        return s
    new, past, prefix = _shapes(case)
    total = [a + b for a, b in zip(new, past)]
    s["k_pages"], s["v_pages"], s["table"], s["kv_len"] = _pages(case, gen, total)
    n = sum(new)
    cu = [0]
    for a in new:
        cu.append(cu[-1] + a)
    s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    if case["op"] == "paged_append":
        qkv = _randn(gen, n, (hq + 2 * hkv), HEAD_DIM, dtype=dtype)
        s.update(_rope_state(case, gen, max(total)), q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:])
        s["positions"] = torch.cat([torch.arange(p, p + a, dtype=torch.int32, device="cuda") for a, p in zip(new, past)])
        s["seq"] = torch.repeat_interleave(torch.arange(len(new), dtype=torch.int32, device="cuda"), torch.tensor(new, device="cuda"))
        s["q_out"] = torch.empty((n, hq, HEAD_DIM), dtype=dtype, device="cuda")
        if own:
            from paper_2506_07533_b200 import binding as mq
            s["rope"] = mq.make_rope(s["cos_sin"], case["rot"], interleaved=case["interleaved"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=s["eps"])
            s["cache"] = mq.moqae_paged_bind(s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
        return s
    s["q"] = _randn(gen, n, hq, HEAD_DIM, dtype=dtype)
    s["out"] = torch.empty((n, hq, HEAD_DIM), dtype=dtype, device="cuda")
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda") / hq).float() if case["alibi"] else None
    s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda") if case["prefix_max"] else None
    s["scale"] = 1.0 / math.sqrt(HEAD_DIM)
    s["new"], s["total"] = new, total
    if own:
        from paper_2506_07533_b200 import binding as mq
        s["cache"] = mq.moqae_paged_bind(s["k_pages"], s["v_pages"], s["table"], s["kv_len"])
        s["options"] = mq.make_attn_options(scale=s["scale"], cap=case["cap"], window=case["window"], slopes=s["slopes"],
                                            prefix_len=s["prefix"])
        size = (mq.moqae_paged_decode_attn_workspace(s["cache"], hq) if case["op"] == "paged_decode" else
                mq.moqae_paged_prefill_attn_workspace(s["cache"], hq, n))
        s["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms -------------------------------------------------------------------------------

def _norm_rotate(x, weight, s, positions):
    """Rows [n][heads][128] in float32 after the norm (where there is a weight) and the rotation."""
    case, x = s["case"], x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"]) * weight.float()
    rot = case["rot"]
    cos, sin = s["cos_sin"][positions.long()][:, None].split(rot // 2, -1)
    turned, rest = x[..., :rot], x[..., rot:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = turned.split(rot // 2, -1)
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, rest], -1)


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


def _decode_plain(s):
    case = s["case"]
    hq, hkv, batch = case["hq"], case["hkv"], case["batch"]
    group, table = hq // hkv, s["table"].clamp_min(0).long()
    keys = s["k_pages"][table].permute(0, 2, 1, 3, 4).reshape(batch, hkv, -1, HEAD_DIM).float()
    values = s["v_pages"][table].permute(0, 2, 1, 3, 4).reshape(batch, hkv, -1, HEAD_DIM).float()
    at = torch.arange(keys.shape[2], device="cuda")
    length = s["kv_len"][:, None, None, None]
    pos = length - 1
    prefix = None if s["prefix"] is None else s["prefix"][:, None, None, None]
    q = s["q"].float().view(batch, hkv, group, HEAD_DIM)
    slopes = None if s["slopes"] is None else s["slopes"].view(1, hkv, group, 1)
    score = _scores(s, q @ keys.transpose(-1, -2), pos - at, slopes)
    p = _softmax(score, _visible(pos, at, length, case["window"], prefix))
    return (p @ values).reshape(batch, hq, HEAD_DIM)


def _prefill_plain(s):
    case = s["case"]
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    group, done, out = hq // hkv, 0, []
    for b, (n, total) in enumerate(zip(s["new"], s["total"])):      # sequences share nothing
        table = s["table"][b, :(total + page - 1) // page].long()
        keys = s["k_pages"][table].transpose(0, 1).reshape(hkv, -1, HEAD_DIM)[:, :total].float()
        values = s["v_pages"][table].transpose(0, 1).reshape(hkv, -1, HEAD_DIM)[:, :total].float()
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
        if case["op"] == "norm_rope":
            mq.moqae_norm_rope(s["rope"], s["q"], s["k"], s["positions"], s["q_out"], s["k_out"])
            return s["q_out"], s["k_out"]
        if case["op"] == "paged_append":
            mq.moqae_paged_append(s["cache"], s["k"], s["v"], s["positions"], seq=s["seq"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
            return s["q_out"], s["k_pages"], s["v_pages"]
        if case["op"] == "paged_decode":
            mq.moqae_paged_decode_attn(s["cache"], s["q"], s["out"], s["workspace"], s["options"])
        else:
            mq.moqae_paged_prefill_attn(s["cache"], s["q"], s["cu_q"], s["out"], s["workspace"], s["options"])
        return s["out"]
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "norm_rope":
        return tuple(_norm_rotate(s[x], s[x + "_weight"], s, s["positions"]).to(dtype) for x in ("q", "k"))
    if case["op"] == "paged_append":
        q, k = (_norm_rotate(s[x], s[x + "_weight"], s, s["positions"]).to(dtype) for x in ("q", "k"))
        pos = s["positions"].long()
        page, slot = s["table"][s["seq"].long(), pos // case["page"]].long(), pos % case["page"]
        s["k_pages"][page, :, slot] = k
        s["v_pages"][page, :, slot] = s["v"]
        return q, s["k_pages"], s["v_pages"]
    return (_decode_plain(s) if case["op"] == "paged_decode" else _prefill_plain(s)).to(dtype)


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
    hq, hkv, row = case["hq"], case["hkv"], HEAD_DIM * 2
    if case["op"] == "norm_rope":
        n = case["tokens"]
        return dict(bytes=n * (2 * (hq + hkv) * row + 4 * case["rot"] + 4), flops=n * (hq + hkv) * HEAD_DIM * 7)
    new, past, prefix = _shapes(case)
    n = sum(new)
    if case["op"] == "paged_append":
        return dict(bytes=n * (2 * (hq + 2 * hkv) * row + 4 * case["rot"] + 12), flops=n * (hq + hkv) * HEAD_DIM * 7)
    pairs = keys = 0
    for a, p, f in zip(new, past, prefix):
        x, y = _seen_pairs(a, a + p, case["window"], f)
        pairs, keys = pairs + x, keys + y
    return dict(bytes=keys * hkv * 2 * row + n * hq * 2 * row, flops=4 * pairs * hq * HEAD_DIM)


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_rows(x, weight, s, positions):
    """The norm and the rotation as a product of complex numbers."""
    case, rot = s["case"], s["case"]["rot"]
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / HEAD_DIM + s["eps"]) * weight.double()
    table = s["cos_sin"].double()[positions.long()]
    turn = torch.complex(table[:, :rot // 2], table[:, rot // 2:])[:, None]
    out = y.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_attention(s):
    """Query by query position, head by head: sum of exp(score) v over the visible tokens, divided by sum of exp(score)."""
    case = s["case"]
    hq, hkv, page = case["hq"], case["hkv"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    done = 0
    for b, (n, total) in enumerate(zip(s["new"], s["total"])):
        where = torch.arange(total, device="cuda")
        pages, slots = s["table"][b].long()[where // page], where % page
        i = torch.arange(n, device="cuda")[:, None] + (total - n)
        allowed = where[None] <= i
        if case["window"]:
            allowed &= where[None] > i - case["window"]
        if s["prefix"] is not None:
            allowed |= where[None] < s["prefix"][b]
        for h in range(hkv):
            k, v = s["k_pages"][pages, h, slots].double(), s["v_pages"][pages, h, slots].double()
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
    s = prepare(case, seed)
    if case["op"] == "norm_rope":
        return tuple(_exact_rows(s[x], s[x + "_weight"], s, s["positions"]) for x in ("q", "k"))
    if case["op"] == "paged_append":
        k, v = s["k_pages"].double(), s["v_pages"].double()
        k_new = _exact_rows(s["k"], s["k_weight"], s, s["positions"])
        pos = s["positions"].long()
        page = s["table"].long()[s["seq"].long(), torch.div(pos, case["page"], rounding_mode="floor")]
        k[page, :, pos - pos // case["page"] * case["page"]] = k_new
        v[page, :, pos - pos // case["page"] * case["page"]] = s["v"].double()
        return _exact_rows(s["q"], s["q_weight"], s, s["positions"]), k, v
    return _exact_attention(s)
