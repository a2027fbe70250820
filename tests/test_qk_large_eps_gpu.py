"""Rows whose squares pass fp32's range beside an eps of their size."""
import pytest
import torch

from layer_common import F32, qk64, rel
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e33, 1e36, 1e38])
@pytest.mark.parametrize("d", [64, 36])
def test_eps_counts_beside_large_rows(cuda_device, d, eps):
    """Sizes of 2e18 to 1e19: squares of 4e36 and more, their sums past 1e38.  The norm is off
    by (d + 40) 2^-24 as anywhere, its gradient by two such, together below 1e-5."""
    g = torch.Generator().manual_seed(0)
    x, up = (torch.randn(1, 2, 40, d, generator=g).to(cuda_device) for _ in range(2))
    x = x * torch.logspace(18.4, 19.0, 40, device=cuda_device).view(1, 1, 40, 1)
    eps = float(torch.tensor(eps, dtype=F32))
    x64 = x.double().requires_grad_()
    want = qk64(x64, None, None, None, False, eps, 1.0)
    wanted, = torch.autograd.grad((want * up.double()).sum(), x64)
    assert rel(slim.qk_norm_forward(x, None, eps=eps)[0], want.detach()) <= 1e-5
    assert rel(slim.qk_norm_backward(x, None, None, None, up, None, eps=eps)[0], wanted) <= 1e-5
