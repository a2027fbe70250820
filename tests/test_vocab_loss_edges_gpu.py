"""The vocabulary loss where small differences, long sums or few rows decide.
The 64-bit references and the bounds of test_vocab_loss_gpu.py are used where
they apply; the others are derived at each test."""
import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,V", [(200, 300, 700), (200, 512, 700), (257, 520, 300), (200, 1024, 700),
                                   (130, 2048, 2500), (200, 4096, 700)])
def test_rows_that_are_sure_of_their_target(cuda_device, dt, N, D, V):
    """A target 30 above the rest: 1 - p is about V e^-30, and g = p - 1 is what
    rounding leaves of the difference of two equal logits.  The log-sum is the
    logit (to fp32), so the exponent is off by the rounding of 30 log2 e in fp32,
    2^-24 of it or so, and p by 2^-23 |lse| and the exponential's 2^-21."""
    g = torch.Generator().manual_seed(D)
    x = (0.5 + torch.rand(N, D, generator=g)).to(dt).to(cuda_device)
    w = torch.randn(V, D, generator=g) * 0.3 / D ** 0.5
    w[0] = (0.5 + torch.rand(D, generator=g)) * 30.0 / D
    w = w.to(dt).to(cuda_device)
    t = torch.zeros(N, dtype=torch.long, device=cuda_device)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    z = x.double() @ w.double().T
    assert (z[:, 0] - z[:, 1:].amax(1)).min() > 20
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, torch.ones(1, device=cuda_device))
    rest = (z[:, 1:] - z[:, :1]).exp().sum(1).max().item()
    bound = 2.0 ** -23 * lse.abs().max().item() + 2.0 ** -21 + 1.01 * rest
    assert dw[0].abs().max().item() <= N * bound * 1.5 * (1 + 2.0 ** -7)
    # dx = g_0 w_0, and as little of the other words
    most = bound * w[0].abs().max().item() + rest * w.abs().max().item()
    assert dx.abs().max().item() <= most * (1 + 2.0 ** -7)
