"""The operators of the paged 16-bit cache in 64 bits, written from their definitions, and how far the
kernels' 16-bit outputs may be from them.

Roundings: a 16-bit result is off by at most half a step, u = finfo(dtype).eps / 2 relative (fp16 also 2^-25
absolute where it is subnormal); a float32 operation by 2^-24 relative.
"""
import math

import torch

F32 = 2.0 ** -24
SUBNORMAL = {torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}


def norm_rope(x, weight, cos_sin, rot, interleaved, eps, positions):
    """Rows [n, heads, 128] in float64 and the largest error of a kernel's row elements."""
    y = x.double()
    if weight is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    out, size = y.clone(), y.abs().clone()
    if rot:
        c, s = cos_sin.double()[positions.long()][:, None].split(rot // 2, -1)
        i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        out[..., i], out[..., j] = y[..., i] * c - y[..., j] * s, y[..., i] * s + y[..., j] * c
        size[..., i] = size[..., j] = y[..., i].abs() + y[..., j].abs()
    # float32: the sum of 128 squares (8 + 3 additions deep, relative error halved by the root), root, division,
    # three products, and two roundings of the rotation: below 24 float32 roundings of the pair's size
    u = torch.finfo(x.dtype).eps / 2
    return out, u * out.abs() * (1 + u) + 24 * F32 * size + SUBNORMAL[x.dtype]


def gather(pages, table_row, n):
    """Rows [n, heads, 128] of one sequence."""
    at = torch.arange(n, device=pages.device)
    return pages[table_row.long()[at // pages.shape[2]], :, at % pages.shape[2]]


def attention(q, k, v, first, *, scale=None, cap=0.0, window=0, slopes=None, prefix=0, split_weights=True):
    """One sequence: q [n, hq, 128] at positions first .. first + n - 1 over k, v [total, hkv, 128].  The
    result in float64, and the largest error of the kernels' result.  split_weights: the kernel keeps its
    weights as two 16-bit halves (else they are rounded to 16 bits)."""
    n, hq, _ = q.shape
    total, hkv, _ = k.shape
    scale = 1 / math.sqrt(128) if scale is None else scale
    dtype = q.dtype
    u = torch.finfo(dtype).eps / 2
    pos = torch.arange(first, first + n, device=q.device)[:, None]
    j = torch.arange(total, device=q.device)[None]
    seen = j <= pos
    if window:
        seen = seen & (j > pos - window)
    seen = seen | (j < prefix)
    out = torch.zeros(n, hq, 128, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    if not n or not total:
        return out, tol
    for h in range(hq):
        kk, vv, qq = k[:, h // (hq // hkv)].double(), v[:, h // (hq // hkv)].double(), q[:, h].double()
        # rows that no query may use can hold anything
        used = seen.any(0)
        kk, vv = torch.where(used[:, None], kk, 0.0), torch.where(used[:, None], vv, 0.0)
        x = qq @ kk.T * scale
        # products are exact; the float32 sum of 128 of them in a tensor core: 128 roundings at most, of 2^-23 each
        # because the hardware may truncate
        err = 128 * 2 * F32 * (qq.abs() @ kk.abs().T) * scale
        if cap > 0:
            x = cap * torch.tanh(x / cap)
            # up to the cap a polynomial of relative error 6e-7 (10 F32) with about ten roundings; beyond, the
            # exponential (argument off by 4 roundings, |2 z| <= 40 where it matters), 1 + e, the reciprocal, the
            # difference: a few roundings of the cap, of which the score is then at least three quarters
            err = err + 128 * F32 * x.abs()
        if slopes is not None:
            bias = slopes[h].double() * (pos - j).abs()
            x = x - bias
            err = err + 4 * F32 * bias
        err = err + 6 * F32 * x.abs() + 8 * F32          # times log2(e), minus the reference, the exponential itself
        err = torch.where(seen, err, 0.0).amax(1, keepdim=True)
        x = x.masked_fill(~seen, -math.inf)
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
        norm = p.sum(1, keepdim=True)
        p = torch.where(norm > 0, p / norm.clamp_min(1e-300), 0.0)
        out[:, h] = p @ vv
        mass = p @ vv.abs()
        # every weight off by e^err in the sum and in the norm; sums of total / 16 steps in float32 (truncated at worst)
        weight = 2 * torch.expm1(err) + (2 * F32) * (total / 16 + 160)
        # rounding of the weights: halves hi + lo are off by u * u; one half by u, and in fp16 by 2^-25 of a
        # reference weight that is at least a half
        weight = weight + (u * u if split_weights else u)
        # one half: the norm may add the rounded weights p (1 + e), |e| <= u, of any part of the tokens, which moves the
        # result by -o times the sum of their p e: at most u |o| more (and u u (mass + |o|) from 1 / (1 + that sum))
        norm_off = 0.0 if split_weights else u * out[:, h].abs() + 2 * u * u * (mass + out[:, h].abs())
        low = 0.0 if split_weights else 2 * SUBNORMAL[dtype] * torch.where(seen, 1.0, 0.0).double() @ vv.abs()
        tol[:, h] = weight * mass + low + norm_off + u * out[:, h].abs() * (1 + u) + SUBNORMAL[dtype] + 1e-30
    return out, tol


def close(got, want, tol, what=""):
    off = (got.double() - want).abs() - tol
    assert torch.isfinite(got.double()).all(), f"{what}: not finite"
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {int((off > 0).sum())} values off, worst {(got.double() - want).abs().max():.3g}, allowed there {tol.flatten()[off.argmax()]:.3g}"
