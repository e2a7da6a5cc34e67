"""Paged 4-bit cache on the GPU: scales so small that float32 loses the scores beside them."""
import pytest
import torch

from paper_2506_07533_b200 import binding as mq

from . import paged4_reference as ref
from .paged_reference import close
from .test_gpu_paged4 import generator, make_cache, space, stored

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new", [1, 5])
def test_nothing_to_say_under_a_tiny_scale(dtype, new):
    """Rows of zeros, and of the smallest numbers, with a scale that float32 loses beside them: all tokens count alike."""
    gen = generator(8)
    cache = make_cache(gen, [37], 1, 16, dtype)
    for scale in (1e-12, 1e-20, 1e-38):
        q = torch.zeros(new, 3, 128, dtype=dtype, device="cuda")
        q[:, 1] = 2.0 ** -24
        q[:, 2] = 1.0
        out, opt = torch.empty_like(q), mq.make_attn_options(scale=scale)
        if new == 1:
            mq.moqae_paged4_decode_attn(cache, q, out, space(mq.moqae_paged4_decode_attn_workspace(cache, 3)), opt)
        else:
            cu = torch.tensor([0, new], dtype=torch.int32, device="cuda")
            mq.moqae_paged4_prefill_attn(cache, q, cu, out, space(mq.moqae_paged4_prefill_attn_workspace(cache, 3, new)), opt)
        want, tol = ref.attention(q, *stored(cache, 0, 37), 37 - new, scale=scale)
        close(out, want, tol, str(scale))
