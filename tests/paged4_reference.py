"""The operators of the paged 4-bit cache in 64 bits, written from their definitions, and how far the kernels' results
may be from them (roundings counted as in paged_reference)."""
import math

import torch

from .paged_reference import F32, SUBNORMAL

FP16 = 2.0 ** -11                # half a step of fp16, relative


def fp16_line(device):
    """All finite fp16 values in order, float64."""
    bits = torch.arange(-32768, 32768, device=device).to(torch.int16).view(torch.float16).double()
    return torch.unique(bits[torch.isfinite(bits)]) + 0.0       # (one zero, of positive sign)


def quantise(x):
    """Rows [..., 128] (float64): codes int64 [..., 4, 32], scales and zeros float64 [..., 4]."""
    line, x = fp16_line(x.device), x.double().unflatten(-1, (4, 32))
    z = line[torch.searchsorted(line, x.amin(-1).contiguous(), right=True) - 1]
    span = (x.amax(-1) - z).float() / torch.full_like(z, 15.0).float()          # a float32 quotient
    s = line[torch.searchsorted(line, span.double().contiguous())]
    r = torch.where(s > 0, 1.0 / torch.where(s > 0, s, 1.0), 0.0).float().double()
    return torch.round((x - z[..., None]) * r[..., None]).long(), s, z


def places(device):
    """Byte of a tile: key codes [16, 128], key scales [16, 4], value codes, value scales; zeros lie 8 and 16 further."""
    t, c, g = torch.arange(16, device=device)[:, None], torch.arange(128, device=device)[None], torch.arange(4, device=device)[None]
    key = 64 * t + 16 * ((c % 32) // 8) + 4 * (c // 32) + (c % 8) // 2
    u, r = (c % 32) // 4, 8 * (t // 8) + 4 * (t % 2) + (t % 8) // 2
    value = 1280 + 512 * (u // 4) + 32 * r + 8 * (u % 4) + 2 * (c // 32) + (c % 4) // 2
    return key, 1024 + 16 * t + 2 * g, value, 2304 + 32 * (t // 2) + 4 * g + 2 * (t % 2)


def pack(k, v):
    """Tiles uint8 [..., 2560] of keys and values [..., 16, 128]."""
    key, key_s, value, value_s = places(k.device)
    tiles = torch.zeros(*k.shape[:-2], 2560, dtype=torch.int64, device=k.device)
    for x, at, scale, further in ((k, key, key_s, 8), (v, value, value_s, 16)):
        code, s, z = quantise(x)
        code = code.flatten(-2) << (4 * (torch.arange(128, device=k.device) % 2))
        tiles.scatter_add_(-1, at.flatten().expand(*k.shape[:-2], -1), code.flatten(-2))
        for part, first in ((s, scale), (z, scale + further)):
            bits = part.half().view(torch.int16).long() & 0xffff
            tiles.scatter_add_(-1, first.flatten().expand(*k.shape[:-2], -1), (bits & 255).flatten(-2))
            tiles.scatter_add_(-1, (first + 1).flatten().expand(*k.shape[:-2], -1), (bits >> 8).flatten(-2))
    return tiles.to(torch.uint8)


def unpack(tiles):
    """((codes, scales, zeros) of keys, of values): [..., 16, 4, 32] and [..., 16, 4] of tiles uint8 [..., 2560]."""
    key, key_s, value, value_s = places(tiles.device)
    out, tiles = [], tiles.long()
    for at, scale, further in ((key, key_s, 8), (value, value_s, 16)):
        byte = tiles[..., at]
        code = torch.where(torch.arange(128, device=tiles.device) % 2 == 1, byte >> 4, byte & 15).unflatten(-1, (4, 32))
        half = lambda w: (tiles[..., w] | (tiles[..., w + 1] << 8)).to(torch.int16).view(torch.float16).double()  # noqa: E731
        out.append((code, half(scale), half(scale + further)))
    return out


def rows_of(pages, table_row, n):
    """scale * code and zero of keys, the same of values, and scales of values, [n, heads, 128] each in float64, of one sequence."""
    page = pages.shape[2] // 160
    at = torch.arange(n, device=pages.device)
    tiles = pages.unflatten(-1, (page // 16, 2560))[table_row.long()[at // page], :, (at % page) // 16]
    slot = (at % 16)[:, None]
    out = []
    heads = torch.arange(pages.shape[1], device=pages.device)[None]
    for code, s, z in unpack(tiles):
        i = torch.arange(n, device=pages.device)[:, None]
        code, s, z = code[i, heads, slot], s[i, heads, slot], z[i, heads, slot]
        out += [(code * s[..., None]).flatten(-2), z.repeat_interleave(32, -1)]
    return out + [s.repeat_interleave(32, -1)]


def attention(q, kc, kz, vc, vz, vs, first, *, scale=None, cap=0.0, window=0, slopes=None, prefix=0, up=0):
    """One sequence: q [n, hq, 128] at positions first .. first + n - 1 over keys kc + kz, values vc + vz [total, hkv, 128] of scales vs.  The
    result in float64, and the largest error of the kernels' result.  2^up (up >= 0): not below any value scale."""
    n, hq, _ = q.shape
    total, hkv, _ = kc.shape
    scale = 1 / math.sqrt(128) if scale is None else scale
    u = torch.finfo(q.dtype).eps / 2
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
        kv = h // (hq // hkv)
        used, qq = seen.any(0)[:, None], q[:, h].double()
        a, b, c, d, s = (torch.where(used, x[:, kv], 0.0) for x in (kc, kz, vc, vz, vs))
        x = qq @ (a + b).T * scale
        # Float32 sums in a tensor core: 128 products and 32 for the zeros, 2^-23 each as the hardware may truncate, and a
        # dozen roundings beside them.  Queries in fp16: off by half a step of 2^-24 at most where the largest element is 8 or more,
        # 16 times that in the odd channels, so by 2^-24 of the largest.  The sum of a group as two halves: 2^-22.
        size = qq.abs() @ (a.abs() + b.abs()).T
        err = (180 * 2 * F32 * size + 2 * F32 * qq.abs().amax(1, keepdim=True) * a.abs().sum(1)[None] + 4 * F32 * (qq.abs() @ b.abs().T)) * scale
        if cap > 0:
            x = cap * torch.tanh(x / cap)
            err = err + 128 * F32 * x.abs()
        if slopes is not None:
            bias = slopes[h].double() * (pos - j).abs()
            x = x - bias
            err = err + 4 * F32 * bias
        err = err + 6 * F32 * x.abs() + 8 * F32
        err = torch.where(seen, err, 0.0).amax(1, keepdim=True)
        x = x.masked_fill(~seen, -math.inf)
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
        norm = p.sum(1, keepdim=True)
        p = torch.where(norm > 0, p / norm.clamp_min(1e-300), 0.0)
        out[:, h] = p @ (c + d)
        mass, codes, mid = p @ (c + d).abs(), p @ (15 * s), p @ (d + 7.5 * s).abs()
        # Every weight off by e^err above and below the line; the weight in fp16 above and below the line; its product with the scale in
        # fp16, which meets a code or 15 - code, at most 15; z + 7.5 s in fp16; float32 sums of these parts.
        t = (2 * torch.expm1(err) + 2 * FP16 * (1 + FP16)) * mass + FP16 * (1 + 2 * FP16) * (codes + mid)
        t = t + 2 * F32 * (total / 16 + 160) * (2 * codes + mid + mass)
        # The largest weight is 2^(12 - up) or more: small ones are off by 2^-25 of one, as are their products, times a code of 15
        n_seen = seen.sum(1, keepdim=True).double()
        t = t + n_seen * 2.0 ** (up - 37) * ((c + d).abs().amax() + 15)
        tol[:, h] = t + u * out[:, h].abs() * (1 + u) + SUBNORMAL[q.dtype] + 1e-30
    return out, tol
