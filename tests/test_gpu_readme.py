"""The README's example of the paged cache, run as it stands there."""
import os
import re

import pytest
import torch

from paper_2506_07533_b200 import binding as mq
from tests import paged_reference as R
from tests.test_gpu_paged import BF, ints, randn

pytestmark = pytest.mark.gpu


def example():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        block = re.search(r"\n((?: {4}.*\n)*? {4}.*moqae_paged_append.*\n(?: {4}.*\n)*)", f.read()).group(1)
    return "".join(line[4:] + "\n" for line in block.splitlines())


def test_readme_example():
    new, hq, hkv = [300, 5, 77], 8, 2
    cu_q = ints([0, 300, 305, 382])
    n_tokens, n_q_heads = 382, hq
    wq, wk = randn(128, dtype=BF, seed=1), randn(128, dtype=BF, seed=2)
    k_pages, v_pages = (torch.full((40, hkv, 16, 128), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    free, kv_len = torch.randperm(40, device="cuda").to(torch.int32), ints([0, 0, 0])
    block_table = torch.full((3, 19), -1, dtype=torch.int32, device="cuda")
    block_table[0], block_table[1, :1], block_table[2, :5] = free[:19], free[19:20], free[20:25]
    positions = torch.cat([torch.arange(n, dtype=torch.int32, device="cuda") for n in new])
    seq = torch.repeat_interleave(ints([0, 1, 2]), torch.tensor(new, device="cuda"))
    q, k, v = (randn(n_tokens, h, 128, dtype=BF, seed=s) for h, s in ((hq, 3), (hkv, 4), (hkv, 5)))
    q1, k1, v1 = (randn(3, h, 128, dtype=BF, seed=s) for h, s in ((hq, 6), (hkv, 7), (hkv, 8)))
    positions1 = ints(new)
    out, out1 = torch.full_like(q, 7.0), torch.full_like(q1, 7.0)
    names = dict(locals())
    exec(example(), names)
    assert mq.moqae_paged_poll_status(names["cache"]) == 0
    assert kv_len.tolist() == [n + 1 for n in new]
    at = cu_q.tolist()
    for b, n in enumerate(new):
        kk, vv = (R.gather(x, block_table[b], n + 1) for x in (k_pages, v_pages))
        assert torch.equal(vv, torch.cat([v[at[b]:at[b + 1]], v1[b:b + 1]]))
        R.close(out[at[b]:at[b + 1]], *R.attention(q[at[b]:at[b + 1]], kk[:n], vv[:n], 0, window=4096, split_weights=False))
        R.close(out1[b:b + 1], *R.attention(q1[b:b + 1], kk, vv, n, window=4096))
