"""Vocabulary loss and its gradients, against the definition in 64 bits.

Tolerances, derived from the arithmetic.  With A_iv = sum_d |x_id w_vd|, a logit
is off by at most dz = (D + 8) 2^-23 max A (each of the D additions of the
tensor core may cut off a unit in the last place of a 24-bit sum; three-piece
operands drop products below 2^-22).  A loss or log-sum is then off by at most
2 dz + 2^-20 (1 + |lse|), the last for the exponential and logarithm.  A
gradient element sums g_iv = c_i (p_iv - onehot): g is off by its logits' and
log-sum's errors, c p (4 dz + 2^-20 (1 + |lse|)), and by its own rounding
(2^-8 |g| to bf16, 2^-22 |g| to three pieces); the sum adds one unit per term
of sum |g w|, and the result is rounded to its type.  Beside these worst cases
the 2-norm of the error is held to 1e-5 (fp32) or 5e-3 (bf16: two roundings of
2^-8 / sqrt 3 in the root mean square, 3.2e-3) of the result's."""
import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
REL = {F32: 1e-5, BF16: 5e-3}
U_OUT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
U_G = {F32: 2.0 ** -22, BF16: 2.0 ** -8}


def make(dev, N, D, V, dt, it=torch.int64, ignored=0.1, seed=0, lean=6.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(V, D, generator=g) / D ** 0.5
    t = (torch.rand(N, generator=g) ** 2 * V).long().clamp(0, V - 1)
    x = 1.5 * torch.randn(N, D, generator=g) + lean * torch.rand(N, 1, generator=g) * w[t]
    t[torch.rand(N, generator=g) < ignored] = -100
    c = 0.5 + torch.rand(N, generator=g)
    return x.to(dt).to(dev), w.to(dt).to(dev), t.to(it).to(dev), c.to(dev)


def ref64(x, w, t, c):
    x, w, t = x.double(), w.double(), t.long()
    live = t != -100
    z = x @ w.T
    lse = torch.logsumexp(z, 1)
    at = torch.where(live, t, 0)[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0.0)
    p = (z - lse[:, None]).exp()
    g = p.scatter_add(1, at, -torch.ones_like(lse)[:, None])
    cc = torch.where(live, c.double(), 0.0)[:, None]
    g = g * cc
    size = float((x.abs() @ w.abs().T).max()) if z.numel() else 0.0
    return dict(loss=loss, lse=lse, dx=g @ w, dw=g.T @ x, g=g, pc=p * cc.abs(), live=live,
                dz=(x.shape[1] + 8) * 2.0 ** -23 * size)


def rel(a, b):
    return float((a.double() - b).norm() / b.norm().clamp(min=1e-300))


def check(x, w, t, c, piece=None, mean=False):
    dt = x.dtype
    loss, lse, total = slim.vocab_loss_forward(x, w, t)
    count = (t != -100).sum().item()
    if mean:
        c = torch.full_like(c, 0.75)
        r = ref64(x, w, t, c / max(count, 1))
        dx, dw = slim.vocab_loss_backward(x, w, t, lse, c[:1].contiguous(), count=total[1:],
                                          piece=piece)
    else:
        r = ref64(x, w, t, c)
        dx, dw = slim.vocab_loss_backward(x, w, t, lse, c, piece=piece)
    tol = 2 * r["dz"] + 2.0 ** -20 * (1 + r["lse"].abs())
    assert ((loss.double() - r["loss"]).abs() <= tol).all()
    assert ((lse.double() - r["lse"]).abs() <= tol).all()
    assert (loss[~r["live"]] == 0).all() and total[1].item() == count
    assert abs(total[0].item() - r["loss"].sum().item()) <= tol.sum().item() + 1e-6 * r["loss"].sum().item()
    assert dx.dtype == dt and dw.dtype == dt
    soft = 4 * r["dz"] + 2.0 ** -20 * (1 + r["lse"].abs())[:, None]
    ge = soft * r["pc"] + U_G[dt] * (r["g"].abs() + soft * r["pc"])
    x64, w64 = x.double().abs(), w.double().abs()
    for got, ref, err, mag, n in ((dx, r["dx"], ge @ w64, r["g"].abs() @ w64, w.shape[0]),
                                  (dw, r["dw"], ge.T @ x64, r["g"].abs().T @ x64, x.shape[0])):
        bound = err + (n + 8) * 2.0 ** -23 * mag + U_OUT[dt] * (ref.abs() + err) + 1e-37
        assert ((got.double() - ref).abs() <= bound).all()
        if ref.numel() >= 1000 and ref.norm() > 0:
            assert rel(got, ref) <= REL[dt]
    if r["loss"].numel() >= 100 and count:
        assert rel(loss, r["loss"]) <= 1e-5 and rel(lse, r["lse"]) <= 1e-5
    return loss, lse, total, dx, dw


SHAPES = [(1, 1, 1), (1, 8, 1), (1, 64, 2), (2, 3, 700), (3, 5, 7), (127, 64, 255), (128, 64, 256),
          (129, 72, 257), (130, 200, 513), (300, 520, 1000), (1000, 33, 97), (64, 128, 5000),
          (257, 96, 40001), (2500, 64, 300), (700, 1030, 2049)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,V", SHAPES)
@pytest.mark.parametrize("mean", [False, True])
def test_loss_and_gradients(cuda_device, N, D, V, dt, mean):
    x, w, t, c = make(cuda_device, N, D, V, dt)
    check(x, w, t, c, mean=mean)


FEW = [(1, 512, 5000), (2, 96, 4097), (3, 1000, 333), (4, 4096, 50), (1, 16384, 40), (8, 2048, 65),
       (5, 100, 20001), (8, 37, 1000), (7, 515, 200), (8, 2056, 40), (9, 64, 3000), (6, 8, 3)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,V", FEW)
@pytest.mark.parametrize("mean", [False, True])
def test_few_rows(cuda_device, N, D, V, dt, mean):
    """Up to eight fp32 or four bf16 rows take kernels of their own."""
    x, w, t, c = make(cuda_device, N, D, V, dt, ignored=0.3)
    a, b = check(x, w, t, c, mean=mean), check(x, w, t, c, mean=mean)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_few_rows_ignored_and_bad(cuda_device, dt):
    x, w, t, c = make(cuda_device, 6, 64, 500, dt, ignored=0.0)
    t[2] = -100
    clean = check(x, w, t, c)
    y, d = x.clone(), c.clone()
    y[2], d[2] = float("nan"), float("inf")
    loss, lse, total = slim.vocab_loss_forward(y, w, t)
    dx, dw = slim.vocab_loss_backward(y, w, t, lse, d)
    for a, b in zip((loss, total, dx, dw), (clean[0], clean[2], clean[3], clean[4])):
        assert torch.equal(a, b)
    t[4] = 500
    loss, lse, total = slim.vocab_loss_forward(x, w, t)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    assert torch.isnan(loss).tolist() == [i == 4 for i in range(6)]
    assert torch.isnan(dx[4]).all() and torch.isfinite(dx[:4]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("piece", [1, 256, 300, 768, 1 << 20])
def test_pieces(cuda_device, dt, piece):
    x, w, t, c = make(cuda_device, 333, 136, 1900, dt, it=torch.int32)
    check(x, w, t, c, piece=piece)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,V,piece", [(333, 131, 1900, 256), (333, 132, 1900, 768),
                                         (100, 77, 30000, 8192), (12000, 20, 300, 256),
                                         (9000, 50, 40, None), (20, 1000, 9000, 2048)])
def test_pieces_of_uneven_rows_and_split_sums(cuda_device, N, D, V, piece, dt):
    """Rows that are no whole 16 bytes, several pieces, and reductions long enough
    to be split, together."""
    x, w, t, c = make(cuda_device, N, D, V, dt)
    a, b = check(x, w, t, c, piece=piece, mean=True), check(x, w, t, c, piece=piece, mean=True)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_same_bits_again(cuda_device, dt):
    x, w, t, c = make(cuda_device, 1500, 320, 6000, dt)
    a, b = check(x, w, t, c, piece=2048), check(x, w, t, c, piece=2048)
    for u, v in zip(a, b):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_long_sums_keep_their_digits(cuda_device, dt):
    """Same-signed sums over many rows and words: dw over 30000 rows that all
    push one way, dx over 12000 words.  A sum that loses a unit at every step of
    the tensor core would be off by thousands of units here."""
    g = torch.Generator().manual_seed(5)
    N, D, V = 30000, 64, 12000
    x = (1.0 + torch.rand(N, D, generator=g)).to(dt).to(cuda_device)
    w = (0.02 * torch.rand(V, D, generator=g)).to(dt).to(cuda_device)
    t = torch.full((N,), V - 1, device=cuda_device)
    c = torch.ones(N, device=cuda_device)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    r = ref64(x, w, t, c)
    assert rel(dw[:-1], r["dw"][:-1]) <= REL[dt] and rel(dw, r["dw"]) <= REL[dt]


@pytest.mark.parametrize("dt", [F32, BF16])
def test_all_rows_ignored(cuda_device, dt):
    x, w, t, c = make(cuda_device, 200, 48, 300, dt, ignored=2.0)
    loss, lse, total, dx, dw = check(x, w, t, c)
    assert (total == 0).all() and (dx == 0).all() and (dw == 0).all()
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c[:1].contiguous(), count=total[1:])
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), "lowest"])
def test_what_ignored_rows_hold_goes_nowhere(cuda_device, dt, bad):
    x, w, t, c = make(cuda_device, 300, 64, 500, dt, ignored=0.2)
    clean = check(x, w, t, c)
    bad = torch.finfo(dt).min if bad == "lowest" else bad
    gone = t == -100
    y, d = x.clone(), c.clone()
    y[gone] = bad
    d[gone] = float("nan")
    loss, lse, total = slim.vocab_loss_forward(y, w, t)
    dx, dw = slim.vocab_loss_backward(y, w, t, lse, d)
    for a, b in zip((loss, total, dx, dw), (clean[0], clean[2], clean[3], clean[4])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_words_masked_by_the_lowest_value(cuda_device, dt):
    """A word masked through a constant feature (x_0 = 1, w_v0 = lowest) has no
    weight and gets no gradient."""
    x, w, t, c = make(cuda_device, 150, 64, 400, dt)
    x[:, 0], w[:, 0] = 1.0, 0.0
    masked = torch.arange(400, device=cuda_device) % 3 == 1
    live = torch.where(masked[t.clamp(min=0)], t + 1, t).clamp(max=399)
    live = torch.where(t == -100, t, torch.where(masked[live.clamp(min=0)], 0, live))
    v = w.clone()
    v[masked, 0] = torch.finfo(dt).min
    loss, lse, _ = slim.vocab_loss_forward(x, v, live)
    dx, dw = slim.vocab_loss_backward(x, v, live, lse, c)
    keep = (~masked).nonzero()[:, 0]
    new = torch.full((400,), -1, device=cuda_device)
    new[keep] = torch.arange(len(keep), device=cuda_device)
    r = ref64(x, w[keep], torch.where(live == -100, live, new[live.clamp(min=0)]), c)
    assert rel(loss, r["loss"]) <= 1e-5 and rel(lse, r["lse"]) <= 1e-5
    assert rel(dw[keep], r["dw"]) <= REL[dt] and (dw[masked] == 0).all()
    assert rel(dx[:, 1:], r["dx"][:, 1:]) <= REL[dt]


@pytest.mark.parametrize("dt", [F32, BF16])
def test_targets_out_of_range_are_loud(cuda_device, dt):
    x, w, t, c = make(cuda_device, 200, 64, 300, dt, ignored=0.0)
    t[7], t[150] = 300, -1
    loss, lse, total = slim.vocab_loss_forward(x, w, t)
    bad = torch.zeros(200, dtype=torch.bool, device=cuda_device)
    bad[7] = bad[150] = True
    assert torch.isnan(loss[bad]).all() and torch.isfinite(loss[~bad]).all()
    assert torch.isnan(total[0]) and total[1].item() == 200
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_small_losses_keep_their_digits(cuda_device, dt):
    """A target far above the rest: loss = log1p(sum of the others against it),
    down to 1e-9, within the logits' own error (2 dz) relative."""
    D, V = 16, 50
    w = torch.zeros(V, D, device=cuda_device)
    w[:, 0] = torch.linspace(-1, 1, V, device=cuda_device)
    w[0, 1] = 1.0
    x = torch.zeros(20, D, device=cuda_device)
    x[:, 0] = 0.5
    x[:, 1] = torch.linspace(2, 24, 20, device=cuda_device)
    x, w = x.to(dt), w.to(dt)
    t = torch.zeros(20, dtype=torch.long, device=cuda_device)
    loss, lse, _ = slim.vocab_loss_forward(x, w, t)
    z = x.double() @ w.double().T
    d = torch.logsumexp(z[:, 1:], 1) - z[:, 0]
    ref = torch.log1p(d.exp())
    dz = (D + 8) * 2.0 ** -23 * float((x.double().abs() @ w.double().abs().T).max())
    assert ((loss.double() - ref).abs() <= (2 * dz + 2.0 ** -18) * ref).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("big", [30.0, 80.0])
def test_large_logits(cuda_device, dt, big):
    """Logits of several hundred: no overflow, the same bounds."""
    x, w, t, c = make(cuda_device, 140, 128, 600, dt)
    x = (x.float() * big).to(dt)
    check_large = ref64(x, w, t, c)
    loss, lse, _ = slim.vocab_loss_forward(x, w, t)
    tol = 2 * check_large["dz"] + 2.0 ** -20 * (1 + check_large["lse"].abs())
    assert ((loss.double() - check_large["loss"]).abs() <= tol).all()
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()


def test_gradients_against_differences(cuda_device):
    """Central differences of the summed loss along random directions.  The
    truncation error of the quotient is below h^2/6 times the third derivative
    along the unit direction; the losses' rounding enters over 2h."""
    x, w, t, c = make(cuda_device, 90, 40, 120, F32)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    ones = torch.ones_like(c)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, ones)
    g = torch.Generator(device=cuda_device).manual_seed(3)
    h = 0.25  # both error terms stay small against the gradients
    for name, a, grad in (("x", x, dx), ("w", w, dw)):
        step = torch.randn(a.shape, generator=g, device=cuda_device)
        step /= step.norm()
        val = []
        for s in (h, -h):
            b = a + s * step
            loss, _, _ = slim.vocab_loss_forward(b if name == "x" else x, b if name == "w" else w, t)
            val.append(loss.double().sum().item())
        quotient = (val[0] - val[1]) / (2 * h)
        slope = (grad.double() * step.double()).sum().item()
        r = ref64(x, w, t, ones)
        rounding = (2 * r["dz"] + 2.0 ** -20 * (1 + r["lse"].abs())).sum().item() / h
        # |third derivative| of log-sum-exp along u is at most 8 max|u z|^3 per row
        zs = (step @ w.T if name == "x" else x @ step.T).double().abs().amax(1)
        truncation = h * h / 6 * 8 * (zs ** 3).sum().item()
        assert abs(quotient - slope) <= rounding + truncation + 1e-5 * abs(slope)
        assert rounding + truncation < 0.05 * max(abs(slope), grad.double().norm().item())


def test_autograd(cuda_device):
    for red in ("mean", "sum", "none"):
        x, w, t, c = make(cuda_device, 200, 64, 300, F32)
        x.requires_grad_(), w.requires_grad_()
        out = slim.vocab_loss(x.view(4, 50, 64), w, t.view(4, 50), reduction=red)
        (out * c.view(4, 50) if red == "none" else 3.0 * out).sum().backward()
        n = (t != -100).sum()
        cc = {"mean": 3.0 / n, "sum": torch.tensor(3.0, device=cuda_device), "none": c}[red]
        r = ref64(x.detach(), w.detach(), t, cc.expand(200).contiguous())
        assert rel(x.grad, r["dx"]) <= 1e-5 and rel(w.grad, r["dw"]) <= 1e-5


def test_autograd_takes_slices_and_transposes(cuda_device):
    """Rows that begin off a 16-byte boundary and transposed operands: refused by
    the plain calls, copied by the differentiable one."""
    x, w, t, c = make(cuda_device, 201, 33, 120, F32)
    with pytest.raises(slim.SlimError) as e:
        slim.vocab_loss_forward(x[1:], w, t[1:])
    assert e.value.status == 1
    with pytest.raises(RuntimeError):
        slim.vocab_loss_forward(x, w.t().contiguous().t(), t)
    x.requires_grad_(), w.requires_grad_()
    slim.vocab_loss(x[1:], w.t().contiguous().t(), t[1:]).backward()
    n = (t[1:] != -100).sum()
    r = ref64(x.detach()[1:], w.detach(), t[1:], (1.0 / n).expand(200).contiguous())
    assert rel(x.grad[1:], r["dx"]) <= 1e-5 and rel(w.grad, r["dw"]) <= 1e-5
    assert (x.grad[0] == 0).all()


def test_another_stream_and_given_workspace(cuda_device):
    x, w, t, c = make(cuda_device, 500, 64, 3000, BF16)
    base = check(x, w, t, c)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    n = max(slim.vocab_loss_workspace_size(500, 64, 3000, BF16, False),
            slim.vocab_loss_workspace_size(500, 64, 3000, BF16, True))
    ws = torch.full((n,), 255, dtype=torch.uint8, device=cuda_device)
    torch.cuda.synchronize()
    loss, lse, total = slim.vocab_loss_forward(x, w, t, workspace=ws, stream=s)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, c, workspace=ws, stream=s)
    s.synchronize()
    for a, b in zip(base, (loss, lse, total, dx, dw)):
        assert torch.equal(a, b)
    slim.check_device_error(ws)


@pytest.mark.parametrize("N", [3, 300])
def test_error_word_is_cleared(cuda_device, N):
    """Whatever a workspace held, a call leaves its error word clear."""
    x, w, t, c = make(cuda_device, N, 64, 500, F32)
    n = max(slim.vocab_loss_workspace_size(N, 64, 500, F32, b) for b in (False, True))
    ws = torch.full((n,), 255, dtype=torch.uint8, device=cuda_device)
    _, lse, _ = slim.vocab_loss_forward(x, w, t, workspace=ws)
    slim.check_device_error(ws)
    ws.fill_(255)
    slim.vocab_loss_backward(x, w, t, lse, c, workspace=ws)
    slim.check_device_error(ws)


def test_no_rows(cuda_device):
    x, w, t, c = make(cuda_device, 4, 64, 30, BF16)
    loss, lse, total = slim.vocab_loss_forward(x[:0], w, t[:0])
    assert loss.shape == (0,) and (total == 0).all()
    dx, dw = slim.vocab_loss_backward(x[:0], w, t[:0], lse, c[:1].contiguous())
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_refusals(cuda_device):
    x, w, t, c = make(cuda_device, 8, 16, 30, F32)
    _, lse, _ = slim.vocab_loss_forward(x, w, t)
    with pytest.raises(TypeError):
        slim.vocab_loss_forward(x, w.to(BF16), t)
    with pytest.raises(TypeError):
        slim.vocab_loss_forward(x, w, t.float())
    with pytest.raises(ValueError):
        slim.vocab_loss_forward(x, w[:, :8].contiguous(), t)
    with pytest.raises(ValueError):
        slim.vocab_loss_forward(x, w, t[:4])
    with pytest.raises(RuntimeError):
        slim.vocab_loss_forward(x[:, ::2], w[:, ::2], t)
    with pytest.raises(ValueError):
        slim.vocab_loss_backward(x, w, t, lse[:3], c)
    with pytest.raises(ValueError):
        slim.vocab_loss_backward(x, w, t, lse, c[:3])
    with pytest.raises(ValueError):
        slim.vocab_loss_backward(x, w, t, lse, c, count=c)
    with pytest.raises(slim.SlimError) as e:
        slim.vocab_loss_backward(x, w, t, lse, c, piece=0)
    assert e.value.status == 1
    with pytest.raises(slim.SlimError) as e:
        slim.vocab_loss_forward(x, w, t, workspace=torch.empty(256, dtype=torch.uint8, device=cuda_device))
    assert e.value.status == 3
    with pytest.raises(ValueError):
        slim.vocab_loss(x, w, t, reduction="median")
