"""Paged 4-bit cache on the GPU: scores so large that float32 tells them apart by many units only.  A row then is the value of its largest score, or
where several cannot be told apart a mean of their values, but never more than that and never no number."""
import math

import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .paged_reference import close
from .test_gpu_paged4 import DTYPES, generator, make_cache, options_of, randn, space, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size, spread, scale", [(1e4, 1e3, None), (1e4, 5e3, None), (12000.0, 6000.0, 1.0), (1.0, 1.0, 1e9), (1e-3, 1.0, 1e20)])
@pytest.mark.parametrize("shaping", [dict(), dict(alibi=True), dict(window=40, prefix=30), dict(alibi=True, prefix=30)], ids=lambda s: "-".join(s) or "plain")
@pytest.mark.parametrize("new", [1, 5, 300])
def test_scores_of_any_size(dtype, size, spread, scale, shaping, new):
    gen = generator(new)
    total, hq = 600, 4
    cache = make_cache(gen, [total], 2, 32, dtype, spread=spread)
    q = (randn(gen, new, hq, 128) * size).to(dtype)
    q[-1, 0] = 0.0                                           # a row of ordinary scores beside them
    opt, slopes, prefix = options_of(gen, hq, 1, scale=scale, **shaping)
    out = torch.empty_like(q)
    if new == 1:
        mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, hq)), opt)
    else:
        cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)), opt)
    assert torch.isfinite(out.float()).all()
    kc, kz, vc, vz, _ = stored(cache, 0, total)
    real = 1 / math.sqrt(128) if scale is None else float(opt.view.scale)
    pos, j = torch.arange(total - new, total, device="cuda")[:, None], torch.arange(total, device="cuda")[None]
    see = (j <= pos) if not shaping.get("window") else (j <= pos) & (j > pos - shaping["window"])
    see = see | (j < (0 if prefix is None else min(max(int(prefix[0]), 0), total)))
    told = 0
    u = torch.finfo(dtype).eps / 2
    for h in range(hq):
        k, v, qq = (kc + kz)[:, h // 2], (vc + vz)[:, h // 2], q[:, h].double()
        # between its smallest and largest value; value, middle of its range, weight and result are each rounded to fp16 or the result's type
        top = torch.where(see[..., None], v[None].abs(), 0.0).amax(1)
        assert (out[:, h].double().abs() <= top * (1 + u) * (1 + 8 * ref.FP16) + 1e-6).all(), h
        x = qq @ k.T * real
        if slopes is not None:
            x = x - slopes[h].double() * (pos - j).abs()
        # Scores as the kernels have them: keys rounded to fp16 (several tokens), float32 sums of 160 products, truncated at worst, queries to 2^-24 of the largest
        err = ((ref.FP16 + 400 * 2 * 2.0 ** -24) * real * (qq.abs() @ k.abs().T)).amax(1) + 8
        best = x.masked_fill(~see, -math.inf).sort(-1, descending=True)
        alone = best.values[:, 0] - best.values[:, 1] > 2 * err + 60
        want = v[best.indices[:, 0]]
        off = (out[:, h].double() - want).abs() - (u + 4 * ref.FP16) * want.abs() - 2 * ref.FP16 * v.abs().amax() - 1e-6
        assert off[alone].numel() == 0 or off[alone].max() <= 0
        told += int(alone.sum())
    if new == 300 and spread > 1.0 or scale == 1e9:
        assert told > 0                                      # (the sizes leave some rows that can be told)
    assert cache.status[0].item() == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [1, 5, 300])
def test_a_query_that_is_no_number_shows_and_stays_alone(dtype, new):
    """One row of NaN, in a sequence whose reference moves many times: its result is NaN, all others are right."""
    gen = generator(new)
    total, hq, at = 700, 4, new // 2
    cache = make_cache(gen, [total], 2, 16, dtype, spread=3.0)
    q = randn(gen, new, hq, 128, dtype=dtype)
    q[at, 2, 5] = float("nan")
    out = torch.zeros_like(q)
    if new == 1:
        mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, hq)))
    else:
        cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)))
    assert torch.isnan(out[at, 2].float()).all()
    clean, got = q.clone(), out.clone()
    clean[at, 2] = 1.0
    want, tol = ref.attention(clean, *stored(cache, 0, total), total - new, up=5)
    got[at, 2] = want[at, 2].to(dtype)
    close(got, want, tol)
