"""Paged 4-bit cache on the GPU: queries far from one, whichever kernel takes them.  The scale brings the scores back to ordinary size, so the result
shows how many bits the queries kept."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .paged_reference import close
from .test_gpu_paged4 import generator, make_cache, options_of, randn, space, stored

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def key_rounding(q, cache, b, total, scale):
    """Several tokens: every element z + s code of a key is rounded to fp16, by at most half a step, which moves a score by at most that
    share of the sum of its products' sizes; e to that power is a weight's error, above and below the line, of the mass at most."""
    kc, kz, vc, vz, _ = stored(cache, b, total)
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    group = q.shape[1] // kc.shape[1]
    for h in range(q.shape[1]):
        k = (kc + kz)[:, h // group].abs()
        e = ref.FP16 * scale * (q[:, h].double().abs() @ k.T).amax(1, keepdim=True)
        out[:, h] = 2 * torch.expm1(e) * (vc + vz)[:, h // group].abs().amax()
    return out


@pytest.mark.parametrize("dtype, spread, size", [(BF, 1.0, 1e-6), (BF, 1.0, 3e-8), (BF, 1.0, 1e-30), (BF, 1.0, 2.0 ** -3), (BF, 1.0, 1e6), (BF, 1.0, 1e11),
                                                 (BF, 1000.0, 1e-3), (BF, 1e-3, 1e3), (FP, 1.0, 1e-6), (FP, 1.0, 1e4), (FP, 1000.0, 1e-3), (FP, 1e-3, 1e3)])
@pytest.mark.parametrize("shaping", [dict(), dict(cap=5.0), dict(alibi=True, prefix=70), dict(cap=30.0, alibi=True, window=150)], ids=lambda s: "-".join(s) or "plain")
@pytest.mark.parametrize("new", [1, 9, 300])
def test_small_and_large_queries(dtype, spread, size, shaping, new):
    """Queries and keys of such sizes; one token, a few (the streaming kernel), many (the large tiles)."""
    gen = generator(new)
    total, hq = 333 + new, 4
    cache = make_cache(gen, [total], 2, 16, dtype, spread=spread)
    scale = 0.0883883 / (size * spread)
    q = (randn(gen, new, hq, 128) * size).to(dtype)
    q[0, 1] = 0                                              # a row of nothing beside the others
    q[-1, 2, 64:] = q[-1, 2, 64:] * 2.0 ** -6                # and one whose elements lie far apart
    opt, slopes, prefix = options_of(gen, hq, 1, scale=scale, **shaping)
    out = torch.empty_like(q)
    if new == 1:
        mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, hq)), opt)
    else:
        cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)), opt)
    rest = {k: v for k, v in shaping.items() if k in ("cap", "window")}
    up = max(0, (int(spread * 10 / 15)).bit_length())
    real = float(opt.view.scale)                             # as float32
    want, tol = ref.attention(q, *stored(cache, 0, total), total - new, scale=real, slopes=slopes,
                              prefix=0 if prefix is None else min(max(int(prefix[0]), 0), total), up=up, **rest)
    close(out, want, tol + (key_rounding(q, cache, 0, total, real) if new * hq // 2 > 96 else 0.0))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_sizes_may_differ_from_row_to_row(dtype):
    """Rows of ordinary size, 2^-24 of it and (bf16) 2^24 times it side by side in one tile: each has the result that it has among its like."""
    gen = generator(7)
    new, total, hq = 200, 900, 2
    cache = make_cache(gen, [total], 1, 32, dtype)
    q, cu = randn(gen, new, hq, 128), torch.tensor([0, new], dtype=torch.int32, device="cuda")
    powers = [0, -24, 24] if dtype == BF else [0, -6, 3]
    mix = torch.tensor([powers[i % 3] for i in range(new * hq)], device="cuda").view(new, hq, 1)
    q = (torch.ldexp(q, mix)).to(dtype)
    work, out = space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)), torch.empty_like(q)
    work, out = space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)), torch.empty_like(q)
    for scale in (0.0883883 * 2.0 ** -p for p in powers):
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, work, mq.make_attn_options(scale=scale))
        real = float(mq.make_attn_options(scale=scale).view.scale)
        pick = mix[..., 0] == -round(torch.log2(torch.tensor(scale / 0.0883883)).item())
        want, tol = ref.attention(q, *stored(cache, 0, total), total - new, scale=real)
        tol = tol + key_rounding(q, cache, 0, total, real)
        close(out[pick], want[pick], tol[pick])
        assert torch.isfinite(out.float()).all()
