"""The 4-bit reference against itself and against the chunk quantiser's rule."""
import torch

from . import paged4_reference as ref


def test_every_byte_of_a_tile_has_one_use():
    key, key_s, value, value_s = ref.places("cpu")
    used = torch.zeros(2560, dtype=torch.int64)
    for at in (key, value):                              # two codes a byte
        used.scatter_add_(0, at.flatten(), torch.ones(at.numel(), dtype=torch.int64))
    for at in (key_s, key_s + 8, value_s, value_s + 16):
        for byte in (0, 1):
            used.scatter_add_(0, (at + byte).flatten(), torch.full((at.numel(),), 2))
    assert (used == 2).all()


def test_pack_and_unpack():
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn(3, 16, 128, generator=gen, dtype=torch.float64) for _ in range(2))
    k[0, 3, 32:64] = 0.25                                # a group of one value
    k[1, 5] *= 1e4
    v[2, 7] *= 1e-6
    for x, (code, s, z) in zip((k, v), ref.unpack(ref.pack(k, v))):
        want = ref.quantise(x)
        assert (code == want[0]).all() and (s == want[1]).all() and (z == want[2]).all()
        assert code.min() >= 0 and code.max() <= 15
        back = (z[..., None] + s[..., None] * code).flatten(-2)
        # nearest code: half a step, and what the float32 inverse is off
        assert ((back - x).abs() <= s.repeat_interleave(32, -1) * (0.5 + 2 ** -19)).all()


def test_the_rule_is_that_of_the_chunks():
    import numpy as np
    from oracle import moqae_oracle as O
    gen = torch.Generator().manual_seed(2)
    v = (torch.randn(32, 128, generator=gen) * torch.logspace(-3, 3, 32)[:, None]).half()
    tile = O.quantize_tile(v.float().numpy(), v.float().numpy(), 4)     # values: per token over 32 channels
    code, s, z = ref.quantise(v.double())
    assert (tile["v_codes"] == code.flatten(-2).numpy()).all()
    assert (tile["v_scale"].astype(np.float64).T == s.numpy()).all() and (tile["v_zero"].astype(np.float64).T == z.numpy()).all()
