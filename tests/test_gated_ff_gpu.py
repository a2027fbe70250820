"""The gated feed-forward and its gradients against the formula in 64 bits.

Tolerances, from the arithmetic.  With A = |x| |w|^T a projection is off by at most
dz = (D + 8) 2^-23 A (each of D additions may cut a unit of a 24-bit sum; three-piece
operands drop products below 2^-22).  An activation takes that times 1.2 (its steepest
slope) and adds 2^-20 (1 + g^2) of itself (its exponential's argument is g or g^2, a
product's rounding in it counts by its size); its derivative takes dz (its own slope is
below 1) and adds 2^-19 (1 + g^2); the step of relu' may fall on the other side where
|g| <= dz.  dz_out = dh * (..) is rounded once more (2^-8 to bf16, 2^-22 to three
pieces), the sums add a unit per term, the results are rounded.  Beside these worst
cases the 2-norm of the error is held to 1e-5 (fp32) or 5e-3 (bf16: two roundings of
2^-8 / sqrt 3 in the root mean square, 3.2e-3) of the result's."""
import ctypes

import pytest
import torch

from layer_common import ACTS, BF16, F32, U, ff64, rel
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

REL = {F32: 1e-5, BF16: 5e-3}
U_G = {F32: 2.0 ** -22, BF16: 2.0 ** -8}


def make(dev, N, D, F, dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, D, generator=g) * (0.5 + torch.rand(N, 1, generator=g))
    w = torch.randn(2 * F, D, generator=g) / D ** 0.5
    return x.to(dt).to(dev), w.to(dt).to(dev), torch.randn(N, F, generator=g).to(dt).to(dev)


def check(x, w, dh, act, backward=True):
    dt, u = x.dtype, U[x.dtype]
    F, D = w.shape[0] // 2, w.shape[1]
    x64, w64, d64 = (t.double().reshape(-1, t.shape[-1]) for t in (x, w, dh))
    z = x64 @ w64.T
    err = (D + 8) * 2.0 ** -23 * (x64.abs() @ w64.abs().T)
    g, up, eg, eu = z[:, :F], z[:, F:], err[:, :F], err[:, F:]
    g = g.clone().requires_grad_()
    a = ACTS[act](g)
    da = torch.autograd.grad(a.sum(), g)[0]
    a, g = a.detach(), g.detach()
    ea = 1.2 * eg + 2.0 ** -20 * (1 + g * g) * a.abs()
    want = a * up
    tol = up.abs() * ea + a.abs() * eu + ea * eu
    h, zk = slim.gated_ff_forward(x, w, act, keep=True)
    assert h.dtype == dt and h.shape == (*x.shape[:-1], F)
    h64 = h.double().reshape(-1, F)
    assert ((h64 - want).abs() <= tol + u * (want.abs() + tol) + 1e-37).all()
    if want.numel() >= 1000 and want.norm() > 0:
        assert rel(h64, want) <= REL[dt]
    if not backward:
        return h, None, None
    eda = eg + 2.0 ** -19 * (1 + g * g)
    if act == "relu":
        eda = torch.where(g.abs() <= eg, 1.0, 0.0)
    dz = torch.cat([d64 * up * da, d64 * a], 1)
    ge = torch.cat([d64.abs() * (up.abs() * eda + (da.abs() + eda) * eu), d64.abs() * ea], 1)
    ge = ge + U_G[dt] * (dz.abs() + ge)
    both = [slim.gated_ff_backward(x, w, dh, act)]
    if zk is not None:
        both.append(slim.gated_ff_backward(x, w, dh, act, z=zk))
    for k, (dx, dw) in enumerate(both):
        if k:  # kept projections are rounded to the type once
            ez = u * z.abs()
            more = torch.cat([d64.abs() * (up.abs() * (ez[:, :F] if act != "relu" else 0.0) + da.abs() * ez[:, F:]),
                              d64.abs() * 1.2 * ez[:, :F]], 1)
            ge = ge + 1.01 * more
        for got, ref, e, mag, n in ((dx, dz @ w64, ge @ w64.abs(), dz.abs() @ w64.abs(), 2 * F),
                                    (dw, dz.T @ x64, ge.T @ x64.abs(), dz.abs().T @ x64.abs(), len(x64))):
            assert got.dtype == dt
            got = got.double().reshape(ref.shape)
            bound = e + (n + 8) * 2.0 ** -23 * mag + u * (ref.abs() + e) + 1e-37
            assert ((got - ref).abs() <= bound).all()
            if ref.numel() >= 1000 and ref.norm() > 0:
                assert rel(got, ref) <= REL[dt]
    return h, dx, dw


SHAPES = [(1, 1, 1), (1, 8, 1), (2, 3, 5), (3, 64, 100), (4, 512, 130), (5, 40, 17), (7, 33, 300), (8, 200, 64),
          (9, 64, 64), (12, 7, 9), (127, 64, 128), (128, 72, 129), (129, 64, 16), (256, 128, 127), (257, 200, 533),
          (300, 520, 1040), (257, 400, 533), (1000, 33, 97), (600, 1030, 80), (2500, 64, 24), (513, 96, 1500)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,F", SHAPES)
def test_against_the_formula(cuda_device, N, D, F, dt):
    check(*make(cuda_device, N, D, F, dt), "silu")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,D,F", [(3, 64, 100), (300, 128, 160), (270, 40, 77)])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations(cuda_device, N, D, F, dt, act):
    x, w, dh = make(cuda_device, N, D, F, dt, seed=1)
    check(3 * x, w, dh, act)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N", list(range(1, 12)))
def test_few_rows(cuda_device, N, dt):
    check(*make(cuda_device, N, 264, 1100, dt, seed=N), "gelu_tanh", backward=False)
    check(*make(cuda_device, N, 37, 50, dt, seed=N), "relu")


@pytest.mark.parametrize("dt", [F32, BF16])
def test_long_walks_and_sums(cuda_device, dt):
    """More tile columns than a worker's share, rows held and not, reductions that are split."""
    check(*make(cuda_device, 700, 64, 9000, dt), "silu")
    check(*make(cuda_device, 300, 576, 3500, dt), "silu")
    check(*make(cuda_device, 40000, 72, 40, dt), "silu")


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("N", [2, 20])
def test_gates_at_their_ends(cuda_device, act, dt, N):
    """Far out the activations are g or nothing, and never NaN."""
    size = [-1e30, -1e5, -300.0, -90.0, -40.0, -12.0, -6.0, 0.0, 6.0, 12.0, 40.0, 90.0, 300.0, 1e5, 1e18, -0.0]
    x = torch.zeros(N, 16, device=cuda_device)
    x[:, 0] = 1.0
    w = torch.zeros(2 * 16, 16, device=cuda_device)
    w[:16, 0], w[16:, 0] = torch.tensor(size, device=cuda_device), 1.0
    x, w, dh = x.to(dt), w.to(dt), torch.ones(N, 16, device=cuda_device, dtype=dt)
    h = slim.gated_ff_forward(x, w, act)
    want = ff64(x.double(), w.double(), act)
    want = torch.where(w[:16, 0].double() < -1e4, torch.zeros_like(want), want)  # g^3 leaves even 64 bits no digits
    g = w[:16, 0].double()
    assert h.isfinite().all()
    # 2^-20 (1 + g^2) where an exponential is left, and what fp32 can hold of it
    tol = torch.where(g.abs() < 100, (2.0 ** -20 * (1 + g * g) + U[dt]) * want.abs(), U[dt] * want.abs()) + 1e-36
    assert ((h.double() - want).abs() <= tol).all()
    dx, dw = slim.gated_ff_backward(x, w, dh, act)
    assert dw.isfinite().all() and (dx.isfinite().all() or act != "sigmoid")


@pytest.mark.parametrize("dt", [F32, BF16])
def test_shapes_and_given_outputs(cuda_device, dt):
    x, w, dh = make(cuda_device, 60, 48, 56, dt)
    ref = slim.gated_ff_forward(x, w)
    refg = slim.gated_ff_backward(x, w, dh)
    x3, dh3 = x.view(3, 4, 5, 48), dh.view(3, 4, 5, 56)
    out = torch.full((62, 56), 7.0, dtype=dt, device=cuda_device)
    got = slim.gated_ff_forward(x3, w, out=out[1:61].view(3, 4, 5, 56))
    assert torch.equal(got.view(60, 56), ref) and (out[0] == 7.0).all() and (out[61] == 7.0).all()
    dx, dw = slim.gated_ff_backward(x3, w, dh3)
    assert dx.shape == x3.shape and torch.equal(dx.view(60, 48), refg[0]) and torch.equal(dw, refg[1])
    one = slim.gated_ff_forward(x[0], w)
    assert one.shape == (56,)
    none = slim.gated_ff_forward(x[:0], w)
    assert none.shape == (0, 56)
    dx, dw = slim.gated_ff_backward(x[:0], w, dh[:0])
    assert dx.shape == (0, 48) and (dw == 0).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N", [3, 300])
def test_a_bad_row_stays_its_own(cuda_device, dt, N):
    x, w, dh = make(cuda_device, N, 64, 96, dt)
    ref = slim.gated_ff_forward(x, w)
    x[1, 5] = float("nan")
    h = slim.gated_ff_forward(x, w)
    dx, _ = slim.gated_ff_backward(x, w, dh)
    rows = [i for i in range(N) if i != 1]
    assert h[1].isnan().all() and torch.equal(h[rows], ref[rows])
    assert dx[1].isnan().all() and dx[rows].isfinite().all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N", [4, 700])
def test_same_bits_streams_and_graphs(cuda_device, dt, N):
    x, w, dh = make(cuda_device, N, 136, 200, dt)

    def both(**kw):
        return (slim.gated_ff_forward(x, w, **kw), *slim.gated_ff_backward(x, w, dh, **kw))

    ref = both()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for t in (x, w, dh):
        t.copy_(t.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    assert not torch.equal(got[0], ref[0])


@pytest.mark.parametrize("N", [3, 300])
@pytest.mark.parametrize("backward", [False, True])
def test_a_wait_that_gave_up_is_reported(cuda_device, N, backward):
    """The next call on the workspace launches nothing and returns the error, and the
    call after it runs.  The wait runs out on a barrier that nothing arrives at."""
    x, w, dh = make(cuda_device, N, 64, 80, F32)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=cuda_device)

    def call(**kw):
        return slim.gated_ff_backward(x, w, dh, **kw) if backward else (slim.gated_ff_forward(x, w, **kw),)

    want = call()
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert slim.library().slim_diag_wait_timeout(ws.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    before = slim.launch_count()
    with pytest.raises(slim.SlimError) as e:
        call(workspace=ws)
    assert e.value.status == 5 and slim.launch_count() == before
    got = call(workspace=ws)
    slim.check_device_error(ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_differences(cuda_device):
    """The kernel's gradient against differences of the kernel's forward along a random
    direction: steps of 2^-8 leave curvature of 2^-16 and roundings of 2^-24 * 2^8."""
    x, w, dh = make(cuda_device, 200, 64, 72, F32)
    g = torch.Generator().manual_seed(1)
    for act in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        grads = slim.gated_ff_backward(x, w, dh, act)
        for i, a in enumerate((x, w)):
            v = torch.randn(a.shape, generator=g).to(cuda_device) * a.std() * 2.0 ** -8
            val = []
            for s in (1.0, -1.0):
                args = [b + s * v if j == i else b for j, b in enumerate((x, w))]
                val.append((slim.gated_ff_forward(*args, act).double() * dh.double()).sum().item())
            want = (grads[i].double() * v.double()).sum().item()
            assert abs((val[0] - val[1]) / 2 - want) <= 4e-3 * (grads[i].double().norm() * v.double().norm()).item()


def test_autograd(cuda_device):
    """The differentiable call on rows that lie apart and off their boundary."""
    x, w, dh = make(cuda_device, 100, 40, 48, F32)
    wide = torch.zeros(100, 47, device=cuda_device)
    wide[:, 3:43] = x

    def run(call, cast):
        a, b = cast(wide).requires_grad_(), cast(w).requires_grad_()
        return torch.autograd.grad((call(a[:, 3:43], b, "gelu") * cast(dh)).sum(), (a, b))

    got = run(slim.gated_ff, lambda t: t.detach().clone())
    want = run(ff64, lambda t: t.detach().double())
    for a, b in zip(got, want):
        assert rel(a, b) < 1e-5


def test_offsets_past_32_bits(cuda_device):
    """More than 2^31 values of h and of dz."""
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 40 GB")
    N, D, F = (1 << 17) + 3, 16, (1 << 14) + 16
    x, w, _ = make(cuda_device, N, D, F, BF16)
    h = slim.gated_ff_forward(x, w)
    rows = torch.tensor([0, 5, N // 2, N - 2, N - 1], device=cuda_device)
    want = ff64(x[rows].double(), w.double(), "silu")
    assert rel(h[rows], want) <= REL[BF16]
    dx, dw = slim.gated_ff_backward(x, w, h)
    x64, w64 = x[rows].double().requires_grad_(), w.double()
    ref = torch.autograd.grad((ff64(x64, w64, "silu") * h[rows].double()).sum(), x64)[0]
    assert rel(dx[rows], ref) <= REL[BF16]
    # a few of w's rows, the first and last of either half among them
    f = torch.tensor([0, 77, F - 1], device=cuda_device)
    x64 = x.double()
    w64 = torch.cat([w[f], w[F + f]]).double().requires_grad_()
    ref = torch.autograd.grad((ff64(x64, w64, "silu") * h[:, f].double()).sum(), w64)[0]
    assert rel(torch.cat([dw[f], dw[F + f]]), ref) <= REL[BF16]
