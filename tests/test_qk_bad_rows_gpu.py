"""Rows of queries that hold an infinity or NaN."""
import math

import pytest
import torch

from layer_common import BF16, F32
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rotary", [(64, 64), (64, 32), (36, 18)])
def test_what_an_infinity_leaves(cuda_device, d, rotary, interleaved, dt):
    g = torch.Generator().manual_seed(0)
    x, up = (torch.randn(1, 2, 9, d, generator=g).to(dt).to(cuda_device) for _ in range(2))
    how = dict(inv_freq=slim.rotary_frequencies(rotary), interleaved=interleaved)
    ref = slim.qk_norm_forward(x, None, **how)[0]
    refg = slim.qk_norm_backward(x, None, None, None, up, None, **how)[0]
    bad = x.clone()
    bad[0, 0, 3, 1], bad[0, 0, 4, d - 1], bad[0, 1, 5, 2] = math.inf, -math.inf, math.nan
    got = slim.qk_norm_forward(bad, None, **how)[0]
    half = rotary // 2
    pair = lambda e: {e} if e >= rotary else {e, e ^ 1} if interleaved else {e, (e + half) % rotary}
    for row, e in ((3, 1), (4, d - 1)):
        nan = sorted(pair(e))
        rest = [i for i in range(d) if i not in nan]
        assert got[0, 0, row, nan].isnan().all() and (got[0, 0, row, rest] == 0).all()
    assert got[0, 1, 5].isnan().all()
    grad = slim.qk_norm_backward(bad, None, None, None, up, None, **how)[0]
    for h, row in ((0, 3), (0, 4), (1, 5)):
        assert grad[0, h, row].isnan().all()
        got[0, h, row], grad[0, h, row] = ref[0, h, row], refg[0, h, row]
    assert torch.equal(got, ref) and torch.equal(grad, refg)
