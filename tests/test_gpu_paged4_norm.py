"""Paged 4-bit cache on the GPU: how far results are off as a whole, beside the bounds of single values: a small error that all values share would pass those."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .test_gpu_paged4 import DTYPES, generator, make_cache, options_of, randn, space, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shaping", [dict(), dict(cap=5.0, alibi=True), dict(window=300)], ids=lambda s: "-".join(s) or "plain")
@pytest.mark.parametrize("new", [1, 7, 333])
def test_error_of_the_norm(dtype, shaping, new):
    """Roundings to fp16 are at most 2^-11, 2^-11 / sqrt(3) rms.  One token and few: of a token's part p (z + s code) = p mid + p s (code - 7.5), the weight
    (whole part), p s (which meets a code or 15 - code: up to a range, 2.4 deviations rms for one of 4 to 5) and the middle (up to one deviation) are each rounded:
    sqrt(1 + 2.4^2 + 1) = 2.8 of these.  Many: weight, value, and the score by its key's elements, at random over 128 channels: sqrt(3) of them.
    The result's own rounding is at most u.  Roundings add up at random over the tokens, as the values do."""
    gen = generator(new)
    total, hq = 2000, 8
    cache = make_cache(gen, [total], 2, 64, dtype)
    q = randn(gen, new, hq, 128, dtype=dtype)
    opt, slopes, _ = options_of(gen, hq, 1, **shaping)
    out = torch.empty_like(q)
    if new == 1:
        mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, hq)), opt)
    else:
        cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, hq, new)), opt)
    want, _ = ref.attention(q, *stored(cache, 0, total), total - new, slopes=slopes, **{k: v for k, v in shaping.items() if k in ("cap", "window")})
    u, parts = torch.finfo(dtype).eps / 2, 2.8 if new * 4 <= 96 else 3 ** 0.5
    error = (out.double() - want).norm() / want.norm()
    assert error <= u + parts * 2.0 ** -11 / 3 ** 0.5, float(error)
    # No part that all values share: the error's component along the result itself.  N errors at random leave error / sqrt(N) of it, or by values that are
    # spread like normal ones (fourth moment three times the square of the second) error / sqrt(N / 3); five times that, and 2^-13 for what is not random.
    shared = ((out.double() - want) * want).sum() / want.square().sum()
    assert shared.abs() <= 2.0 ** -13 + 5 * error / (want.numel() / 3) ** 0.5, float(shared)
