"""The vocabulary loss where small differences, long sums or few rows decide.
The 64-bit references and the bounds of test_vocab_loss_gpu.py are used where
they apply; the others are derived at each test."""
import pytest
import torch

from paper_2012_11346_gb300 import slim
from test_vocab_loss_gpu import U_G, U_OUT, check, make, ref64

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


def test_a_million_terms_of_one_sign(cuda_device):
    """dw of a bf16 problem over 2^20 rows that all push the same way.  The tensor
    core cuts the end off what it adds to a long sum, always downwards, so such
    sums are cut into parts that are joined in fp32.  What may be missing is 2^-12
    of the result, an eighth of the unit it is rounded to: that shows in the mean
    over 10^5 elements, from which the results' own rounding (2^-9 / sqrt 3 each)
    vanishes to below 1e-5; 2e-5 is left to it.  26 tiles of words, so that the
    work alone gives no reason to split the sums."""
    g = torch.Generator(device=cuda_device).manual_seed(11)
    N, D, V = 1 << 20, 16, 26 * 256
    x = (0.5 + torch.rand(N, D, generator=g, device=cuda_device)).to(BF16)
    w = (0.5 * torch.randn(V, D, generator=g, device=cuda_device)).to(BF16)
    t = torch.zeros(N, dtype=torch.long, device=cuda_device)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, torch.ones(1, device=cuda_device))
    ref = torch.zeros(V, D, dtype=torch.float64, device=cuda_device)
    for a in range(0, N, 1 << 15):
        rows = x[a:a + (1 << 15)].double()
        ref += torch.softmax(rows @ w.double().T, 1).T @ rows
    off = ((dw.double()[1:] - ref[1:]) / ref[1:]).mean().item()
    assert -(2.0 ** -12 + 2e-5) <= off <= 2e-5
    # the last row of dx, against the definition
    p = torch.softmax(x[-1:].double() @ w.double().T, 1)
    p[0, 0] -= 1
    last = p @ w.double()
    assert (dx[-1:].double() - last).norm() <= 5e-3 * last.norm()


# every row count that takes the few-row kernels, and the first that does not
FEW = [(BF16, n) for n in (1, 2, 3, 4, 5)] + [(F32, n) for n in (1, 2, 3, 4, 5, 6, 7, 8, 9)]


@pytest.mark.parametrize("D,V", [(64, 500), (37, 90), (1000, 33)])
@pytest.mark.parametrize("dt,N", FEW)
def test_few_rows_with_an_ignored_one(cuda_device, dt, N, D, V):
    """What an ignored row and its upstream gradient hold goes nowhere."""
    for gone in range(N):
        x, w, t, c = make(cuda_device, N, D, V, dt, it=torch.int32, ignored=0.0, seed=gone)
        t[gone] = -100
        clean = check(x, w, t, c)
        for bad in (float("nan"), float("inf"), torch.finfo(dt).min):
            y, d = x.clone(), c.clone()
            y[gone], d[gone] = bad, bad
            loss, lse, total = slim.vocab_loss_forward(y, w, t)
            dx, dw = slim.vocab_loss_backward(y, w, t, lse, d)
            for a, b in zip((loss, total, dx, dw), (clean[0], clean[2], clean[3], clean[4])):
                assert torch.equal(a, b)
            assert (dx[gone] == 0).all()


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("dt,N", FEW)
def test_few_rows_all_ignored(cuda_device, dt, N, mean):
    x, w, t, c = make(cuda_device, N, 64, 300, dt, ignored=2.0)
    loss, lse, total = slim.vocab_loss_forward(x, w, t)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c[:1] if mean else c, count=total[1:] if mean else None)
    assert (loss == 0).all() and (total == 0).all() and (dx == 0).all() and (dw == 0).all()
    assert ((lse.double() - torch.logsumexp(x.double() @ w.double().T, 1)).abs() <= 1e-4).all()


@pytest.mark.parametrize("dt,N", FEW)
@pytest.mark.parametrize("bad", [-1, 500, 1 << 31])
def test_few_rows_with_a_target_out_of_range(cuda_device, dt, N, bad):
    x, w, t, c = make(cuda_device, N, 64, 500, dt, ignored=0.0)
    at = N // 2
    t[at] = bad
    loss, lse, total = slim.vocab_loss_forward(x, w, t)
    assert torch.isnan(loss).tolist() == [i == at for i in range(N)] and total[1].item() == N
    assert torch.isnan(total[0]) and torch.isfinite(lse).all()
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    assert torch.isnan(dx).all(1).tolist() == [i == at for i in range(N)]
    assert torch.isfinite(dx[torch.arange(N, device=cuda_device) != at]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("big", [30.0, 80.0])
@pytest.mark.parametrize("N,D", [(140, 128), (140, 700), (3, 128)])
def test_gradients_at_large_logits(cuda_device, dt, N, D, big):
    """Logits of several hundred: the elementwise bounds of test_vocab_loss_gpu.py.
    Errors of the exponents are no longer small there: p is off by a factor of
    exp(4 dz + ...)."""
    x, w, t, c = make(cuda_device, N, D, 600, dt)
    x = (x.float() * big).to(dt)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    r = ref64(x, w, t, c)
    soft = torch.expm1(4 * r["dz"] + 2.0 ** -20 * (1 + r["lse"].abs()))[:, None]
    ge = soft * r["pc"] + U_G[dt] * (r["g"].abs() + soft * r["pc"])
    x64, w64 = x.double().abs(), w.double().abs()
    for got, ref, err, mag, n in ((dx, r["dx"], ge @ w64, r["g"].abs() @ w64, w.shape[0]),
                                  (dw, r["dw"], ge.T @ x64, r["g"].abs().T @ x64, N)):
        bound = err + (n + 8) * 2.0 ** -23 * mag + U_OUT[dt] * (ref.abs() + err) + 1e-37
        assert ((got.double() - ref).abs() <= bound).all()
