"""Many tokens of small weight behind one of large weight: what 16-bit weights make of them."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests import paged_reference as R
from tests.test_gpu_paged import BF, FP, ints, randn

pytestmark = pytest.mark.gpu


def sink(dtype, n, hkv, hq, batch, bits, seed=5):
    """Sequences (all in the same pages) whose first token outweighs each of the others by 2^bits, with a value of zero; the
    others' values lie around 100, so that the result is what their small weights add up to."""
    k, v = randn(n // 16, hkv, 16, 128, dtype=dtype, seed=seed, scale=0.02), randn(n // 16, hkv, 16, 128, dtype=dtype, seed=seed + 1) + 100
    q = torch.ones(batch, hq, 128, dtype=dtype, device="cuda")
    k[0, :, 0] = bits * 0.6931472 / 128 ** 0.5               # q.k / sqrt(128) = bits * ln 2
    v[0, :, 0] = 0
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").expand(batch, -1).contiguous()
    return mq.moqae_paged_bind(k, v, table, ints([n] * batch)), q


def rows_of(c, n):
    return R.gather(c.k_pages, c.block_table[0], n), R.gather(c.v_pages, c.block_table[0], n)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("group", [1, 4, 8])
@pytest.mark.parametrize("bits", [12, 20, 26])
def test_decode_keeps_small_weights(dtype, group, bits):
    """More (sequence, head) pairs than warps, so that a warp meets the large score and the small ones in one piece."""
    n, hkv, batch = 8000, 32, 64
    c, q = sink(dtype, n, hkv, hkv * group, batch, bits)
    out = torch.empty_like(q)
    ws = torch.zeros(mq.moqae_paged_decode_attn_workspace(c, hkv * group), dtype=torch.uint8, device="cuda")
    mq.moqae_paged_decode_attn(c, q, out, ws)
    k, v = rows_of(c, n)
    want, tol = R.attention(q[:1], k, v, n - 1)
    if dtype is FP:                                          # a weight is off by at most 2^-35 of the largest
        tol = tol + 2.0 ** -35 * v.double().abs().sum(0).repeat_interleave(group, 0)
    for b in (0, 1, 30, 63):
        R.close(out[b:b + 1], want, tol, f"sequence {b}")


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("opt", [dict(), dict(cap=30.0), dict(slopes=True), dict(cap=30.0, slopes=True)])
@pytest.mark.parametrize("bits", [12, 20, 26])
def test_prefill_keeps_small_weights(dtype, opt, bits):
    """A token that outweighs everything before it, seen by all rows.  Blocks are walked from the last to the first, so the large score comes
    first; without a workspace one CTA walks them all."""
    n, new, hkv, hq = 8000, 40, 2, 8
    c, q = sink(dtype, n, hkv, hq, 1, bits)
    q = q.expand(new, hq, 128).contiguous()
    c.k_pages[-1, :, 15] = 0                                  # the large score moves to the last block: to the token before the new ones
    at = n - new - 1
    page, slot = int(c.block_table[0, at // 16]), at % 16
    c.k_pages[page, :, slot], c.v_pages[page, :, slot] = c.k_pages[0, :, 0], 0
    c.k_pages[0, :, 0], c.v_pages[0, :, 0] = 0, 100
    opt = dict(opt)
    if opt.pop("slopes", False):
        opt["slopes"] = torch.full((hq,), 1e-4, device="cuda")
    out = torch.full_like(q, 7.0)
    mq.moqae_paged_prefill_attn(c, q, ints([0, new]), out, None, mq.make_attn_options(**opt))
    k, v = rows_of(c, n)
    want, tol = R.attention(q, k, v, n - new, split_weights=False, **opt)
    # The bound of the definition's file allows 2^-24 of a weight of one.  The reference lies 4 below a score that the row
    # sees, rounded up: that score's weight is at least 2^3, half a step of the smallest ones is 2^-25, so they are off by 2^-28 of it.
    if dtype is FP:
        used = v.double().abs().sum(0).repeat_interleave(hq // hkv, 0)
        tol = tol - 2 * R.SUBNORMAL[FP] * seen_sum(v, n, new, hq) + 2.0 ** -28 * used
    R.close(out, want, tol)


def seen_sum(v, n, new, hq):
    """sum of |v| over the tokens that each of the last `new` queries sees, [new, hq, 128]"""
    total = v.double().abs().cumsum(0)[n - new:]
    return total.repeat_interleave(hq // v.shape[1], 1)
