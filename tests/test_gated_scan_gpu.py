"""The gated recurrence and its gradients against the formula in 64 bits, step by step.

Tolerances, from the arithmetic.  exp(g) = 2^(g log2 e) is off by 2^-22 of itself, and
by 1.25 |g| 2^-24 through its argument (the product's rounding 2^-24, the constant's
2^-26); a sigmoid adds a sum, a reciprocal and a product: with |g| <= 8 here a gate is
within 17 * 2^-24.  A step rounds twice, and joining chunks rounds a term's factors at
most once more per step: C = 20 * 2^-24 a step covers them.  With m_t = |a_t| m_(t-1) + |u_t| the size of
what meets in h_t, its error follows e_t = |a_t| e_(t-1) + C m_t.  The same from the
other end for g; a product of two such values takes both errors and C of its size;
the result's rounding adds U."""
import ctypes
import math

import pytest
import torch

from layer_common import BF16, F32, U, gates64, rel, scan64
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

C = 20 * 2.0 ** -24
KINDS = ["value", "log", "sigmoid"]


def make(dev, B, L, D, kind, dt, seed=0, resets=True, packed=True):
    g = torch.Generator().manual_seed(seed)
    gate = 1.5 * torch.randn(B, L, D, generator=g) + 2.0 + 2.0 * torch.rand(D, generator=g)
    border = torch.rand(B, L, 1, generator=g) < (0.02 if resets else -1.0)
    if kind == "value":
        gate = torch.where(border, 0.0, torch.sigmoid(gate)) * torch.where(torch.rand(D, generator=g) < 0.2, -1.0, 1.0)
    elif kind == "log":
        gate = torch.where(border, -math.inf, -torch.nn.functional.softplus(-gate))
    else:
        gate = torch.where(border, -math.inf, gate)
    rows = torch.stack([gate, torch.randn(B, L, D, generator=g)], 2).to(dt).to(dev)
    gate, x = rows[:, :, 0], rows[:, :, 1]
    if not packed:
        gate, x = gate.contiguous(), x.contiguous()
    h0, dlast = (torch.randn(B, D, generator=g).to(dev) for _ in range(2))
    return gate, x, h0, torch.randn(B, L, D, generator=g).to(dt).to(dev), dlast


def along(a, u, start, back=False):
    """All s_t = |a_t| s_(t-1) + u_t, or from the other end s_t = u_t + |a_(t+1)| s_(t+1)."""
    s, out = start, []
    for t in (range(u.shape[1] - 1, -1, -1) if back else range(u.shape[1])):
        s = u[:, t] + (s if back and t == u.shape[1] - 1 else (a[:, t + 1] if back else a[:, t]).abs() * s)
        out.append(s)
    return torch.stack(out[::-1] if back else out, 1)


def check(gate, x, kind, h0, dh, dlast, **kw):
    dt, u = x.dtype, U[x.dtype]
    h, last, kept = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
    dgate, dx, dh0 = slim.gated_scan_backward(gate, x, kept, dh, kind, dlast=dlast)
    B, L, D = x.shape
    g64, x64 = gate.double().requires_grad_(), x.double().requires_grad_()
    s64 = torch.zeros(B, D, dtype=torch.float64, device=x.device) if h0 is None else h0.double()
    s64 = s64.requires_grad_()
    up = torch.zeros_like(s64) if dlast is None else dlast.double()
    wh, wl = scan64(g64, x64, kind, s64)
    wg, wx, w0 = torch.autograd.grad((wh * dh.double()).sum() + (wl * up).sum(), (g64, x64, s64))
    wg = torch.where(gate.isinf(), 0.0, wg)  # exp(-inf) * 0: the limit
    with torch.no_grad():
        a, b = gates64(g64, kind)
        m = along(a, (b * x64).abs(), s64.abs())
        e = along(a, C * m, torch.zeros_like(s64))
        mg = along(a, dh.double().abs(), dh.double()[:, -1].abs() + up.abs(), back=True)
        # the last step's start is its own value
        eg = along(a, C * mg, C * mg[:, -1], back=True)
        before = torch.cat([s64.abs()[:, None], m[:, :-1]], 1)
        ebefore = torch.cat([torch.zeros_like(s64)[:, None], e[:, :-1]], 1)
        if kind == "sigmoid":
            before, factor = before + x64.abs(), (a * b).abs()
        else:
            factor = torch.ones_like(a) if kind == "value" else a.abs()
        tol = {"h": e, "last": e[:, -1], "dx": b * (eg + C * mg), "dh0": a[:, 0].abs() * (eg[:, 0] + C * mg[:, 0]),
               "dgate": factor * (eg * before + mg * ebefore + C * mg * before)}
        for name, got, want in (("h", h, wh), ("last", last, wl), ("dx", dx, wx), ("dh0", dh0, w0), ("dgate", dgate, wg)):
            r = u if name in ("h", "dx", "dgate") else U[F32]
            assert got.dtype == (dt if name in ("h", "dx", "dgate") else F32)
            bad = (got.double() - want).abs() > tol[name] + r * (want.abs() + tol[name]) + 1e-37
            assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[:3].tolist())
    return h, last, kept, dgate, dx, dh0


SHAPES = [(1, 1, 1), (3, 1, 5), (2, 2, 4), (1, 7, 3), (2, 63, 8), (2, 64, 8), (2, 65, 8), (1, 127, 33), (3, 128, 12),
          (2, 200, 130), (1, 1021, 7), (1, 2100, 36), (70, 3, 2), (1, 300, 260), (2, 577, 64)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,L,D", SHAPES)
def test_against_the_formula(cuda_device, B, L, D, kind, dt):
    gate, x, h0, dh, dlast = make(cuda_device, B, L, D, kind, dt)
    check(gate, x, kind, h0, dh, dlast)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("kind", KINDS)
def test_without_states(cuda_device, kind, dt):
    gate, x, _, dh, _ = make(cuda_device, 2, 150, 20, kind, dt, resets=False)
    check(gate, x, kind, None, dh, None)


@pytest.mark.parametrize("L", [4099, 20011])
@pytest.mark.parametrize("kind", KINDS)
def test_long(cuda_device, L, kind):
    gate, x, h0, dh, dlast = make(cuda_device, 1, L, 5, kind, F32, seed=L)
    check(gate, x, kind, h0, dh, dlast)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("kind", KINDS)
def test_layouts_agree(cuda_device, kind, dt):
    """Contiguous, slices of wider rows, odd starts and pitches, written ones among them:
    the same bits, and nothing but the rows is written."""
    B, L, D = 2, 150, 24
    gate, x, h0, dh, dlast = make(cuda_device, B, L, D, kind, dt, packed=False)
    ref = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
    refg = slim.gated_scan_backward(gate, x, ref[2], dh, kind, dlast=dlast)
    for pitch, start in ((D, 1), (D, 4), (D + 1, 0), (D + 4, 4), (3 * D, 8)):
        buf = [torch.full((B * L * pitch + start + 8,), 9.0, dtype=dt, device=cuda_device) for _ in range(4)]
        v = [b[start:start + B * L * pitch].view(B, L, pitch)[..., :D] for b in buf]
        v[0].copy_(gate)
        v[1].copy_(x)
        out = slim.gated_scan_forward(v[0], v[1], kind, h0=h0, keep=True)
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        g = slim.gated_scan_backward(v[0], v[1], out[2], dh, kind, dlast=dlast, dgate=v[2], dx=v[3])
        assert all(torch.equal(a, b) for a, b in zip(g, refg))
        for b in buf[2:]:
            b[start:start + B * L * pitch].view(B, L, pitch)[..., :D] = 9.0
            assert (b == 9.0).all()
    # one row for all steps
    one = gate[:1, 3:4].expand(1, L, D)
    a = slim.gated_scan_forward(one, x[:1], kind, h0=h0[:1])
    b = slim.gated_scan_forward(one.contiguous(), x[:1], kind, h0=h0[:1])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cut", [64, 128, 1, 77])
def test_segments(cuda_device, kind, cut):
    """A sequence in two calls is the sequence in one within the roundings of another
    order; the gradient of the state carries over."""
    gate, x, h0, dh, dlast = make(cuda_device, 2, 200, 40, kind, F32, seed=cut)
    h, last, kept = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
    grads = slim.gated_scan_backward(gate, x, kept, dh, kind, dlast=dlast)
    parts = [t.contiguous() for t in (gate[:, :cut], x[:, :cut], dh[:, :cut], gate[:, cut:], x[:, cut:], dh[:, cut:])]
    h1, s1, k1 = slim.gated_scan_forward(parts[0], parts[1], kind, h0=h0, keep=True)
    h2, s2, k2 = slim.gated_scan_forward(parts[3], parts[4], kind, h0=s1, keep=True)
    g2 = slim.gated_scan_backward(parts[3], parts[4], k2, parts[5], kind, dlast=dlast)
    g1 = slim.gated_scan_backward(parts[0], parts[1], k1, parts[2], kind, dlast=g2[2])
    got = [torch.cat([h1, h2], 1), s2, torch.cat([g1[0], g2[0]], 1), torch.cat([g1[1], g2[1]], 1), g1[2]]
    for a, b in zip(got, (h, last, *grads)):
        assert rel(a, b) < 1e-5


def test_token_by_token(cuda_device):
    """A sequence decoded one token a call, its state updated in place, is the sequence
    in one call within the roundings of another order."""
    gate, x, h0, _, _ = make(cuda_device, 3, 100, 48, "sigmoid", F32, resets=False)
    h, last = slim.gated_scan_forward(gate, x, "sigmoid", h0=h0)
    state = h0.clone()
    for t in range(100):
        ht, s = slim.gated_scan_forward(gate[:, t:t + 1], x[:, t:t + 1], "sigmoid", h0=state, last=state)
        assert s is state and rel(ht[:, 0], h[:, t]) < 1e-5
    assert rel(state, last) < 1e-5


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("L", [3, 64, 300, 3000])
def test_gradients_over_their_inputs(cuda_device, L, dt):
    gate, x, h0, dh, dlast = make(cuda_device, 3, L, 72, "sigmoid", dt)
    kept = slim.gated_scan_forward(gate, x, "sigmoid", h0=h0, keep=True)[2]
    ref = slim.gated_scan_backward(gate, x, kept, dh, "sigmoid", dlast=dlast)
    got = slim.gated_scan_backward(gate, x, kept, dh, "sigmoid", dlast=dlast, dgate=gate, dx=x)
    assert got[0] is gate and got[1] is x and all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("L", [3, 64, 300])
def test_states_in_place(cuda_device, L):
    gate, x, h0, dh, dlast = make(cuda_device, 2, L, 36, "log", F32)
    ref = slim.gated_scan_forward(gate, x, "log", h0=h0, keep=True)
    refg = slim.gated_scan_backward(gate, x, ref[2], dh, "log", dlast=dlast)
    s, d = h0.clone(), dlast.clone()
    out = slim.gated_scan_forward(gate, x, "log", h0=s, last=s, keep=True)
    g = slim.gated_scan_backward(gate, x, out[2], dh, "log", dlast=d, dh0=d)
    assert out[1] is s and g[2] is d
    assert all(torch.equal(a, b) for a, b in zip((*out, *g), (*ref, *refg)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("at", [0, 5, 63, 64, 130])
def test_a_new_start_forgets_everything(cuda_device, kind, at):
    """Behind a gate of zero nothing is left of what came before, infinities and NaN
    included; other channels and sequences do not notice."""
    gate, x, h0, dh, dlast = make(cuda_device, 2, 200, 12, kind, F32, resets=False, packed=False)
    gate[:, at] = 0.0 if kind == "value" else -math.inf
    clean = slim.gated_scan_forward(gate, x, kind, h0=h0)
    x2, h2 = x.clone(), h0.clone()
    if at:
        x2[0, :at, 3], x2[0, :at, 4] = math.inf, math.nan
    h2[0, 3], h2[0, 4] = math.nan, math.inf
    h, last = slim.gated_scan_forward(gate, x2, kind, h0=h2)
    assert torch.equal(last, clean[1]) and torch.equal(h[:, at:], clean[0][:, at:])
    assert torch.equal(h[1], clean[0][1]) and torch.equal(h[0][:, 5:], clean[0][0][:, 5:])
    if at:
        assert h[0, :at, 3].isnan().any() or h[0, :at, 3].isinf().any()
    # from the other end: gradients behind the start do not pass it
    d2 = dh.clone()
    d2[0, at:, 3] = math.nan
    _, _, kept = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
    a = slim.gated_scan_backward(gate, x, kept, dh, kind, dlast=dlast)
    b = slim.gated_scan_backward(gate, x, kept, d2, kind, dlast=dlast)
    assert torch.equal(a[1][:, :at], b[1][:, :at]) and torch.equal(a[0][:, :at], b[0][:, :at])
    assert torch.equal(a[2], b[2])
    if kind != "value":
        assert (a[0][:, at] == 0).all()


@pytest.mark.parametrize("L", [64, 200, 5000])
def test_gates_beyond_one(cuda_device, L):
    """Whose product passes fp32's range: behind a new start nothing is left of it."""
    gate = torch.full((2, L, 6), 100.0, device=cuda_device)
    x = torch.zeros_like(gate)
    x[:, 3, 1] = 1.0
    gate[:, L // 2] = 0.0
    gate[:, L // 2 + 1:] = 0.5
    x[:, L // 2 + 1:] = torch.randn(2, L - L // 2 - 1, 6, generator=torch.Generator().manual_seed(0)).to(cuda_device)
    h, last, kept = slim.gated_scan_forward(gate, x, "value", keep=True)
    # (before it the state's and the gradient's products have none either)
    clean, clean_last = slim.gated_scan_forward(gate[:, L // 2:].contiguous(), x[:, L // 2:].contiguous(), "value")
    assert rel(h[:, L // 2:], clean) <= 1e-6 and rel(last, clean_last) <= 1e-6
    assert not h[:, L // 2 - 1, 1].isfinite().any()
    dh = torch.zeros_like(x)
    dh[:, -1] = 1.0
    _, dx, _ = slim.gated_scan_backward(gate, x, kept, dh, "value")
    k = torch.arange(L - L // 2 - 1, -1, -1, device=cuda_device)  # steps to the last: exact powers of a half
    assert (dx[:, L // 2:] == 0.5 ** k[None, :, None].float()).all()


def test_gates_at_their_ends(cuda_device):
    """Sigmoid gates far out keep either factor's digits; gates of one add up exactly."""
    g = torch.tensor([-200.0, -90.0, -20.0, 0.0, 20.0, 80.0, 200.0, math.inf], device=cuda_device).view(1, 1, 8)
    x, h0 = torch.full_like(g, 3.0), torch.full((1, 8), 2.0, device=cuda_device)
    _, last = slim.gated_scan_forward(g, x, "sigmoid", h0=h0)
    want = 2 * torch.sigmoid(g.double()) + 3 * torch.sigmoid(-g.double())
    assert ((last.double() - want[0]).abs() <= 2.0 ** -21 * want[0]).all()
    up = torch.zeros_like(g)
    kept = h0[:, None].contiguous()
    _, dx, dh0 = slim.gated_scan_backward(g, x, kept, up, "sigmoid", dlast=torch.ones_like(h0))
    for got, w in ((dx[0], torch.sigmoid(-g.double())[0]), (dh0, torch.sigmoid(g.double())[0])):
        # 2^(g log2 e): its argument's rounding counts by its size
        far = torch.where(g.isinf(), 0.0, g.double().abs())[0]
        assert ((got.double() - w).abs() <= (7 * 2.0 ** -24 + 1.25 * far * 2.0 ** -24) * w + 1e-37).all()
    ones = torch.ones(1, 1000, 3, device=cuda_device)
    h, last = slim.gated_scan_forward(ones, ones, "value")
    assert torch.equal(h[0, :, 1], torch.arange(1, 1001, device=cuda_device).float())


def test_nothing_to_do(cuda_device):
    z = torch.zeros(2, 0, 6, device=cuda_device)
    h0 = torch.randn(2, 6, device=cuda_device)
    h, last, kept = slim.gated_scan_forward(z, z, "log", h0=h0, keep=True)
    assert h.shape == z.shape and torch.equal(last, h0) and kept.shape == (2, 0, 6)
    dg, dx, dh0 = slim.gated_scan_backward(z, z, kept, z, "log", dlast=h0)
    assert torch.equal(dh0, h0) and dg.shape == z.shape
    assert (slim.gated_scan_forward(z, z, "log")[1] == 0).all()
    n = torch.zeros(0, 5, 6, device=cuda_device)
    assert slim.gated_scan_forward(n, n)[0].shape == n.shape


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,L,D", [(3, 600, 40), (2, 1024, 33), (40, 640, 70), (700, 150, 20), (5, 2049, 100)])
def test_tiles_of_a_cluster_and_of_the_whole_gpu(cuda_device, B, L, D, dt):
    """Sequences whose tiles are one cluster (with blocks to spare, and full) and such that
    look back through the workspace, with too many tiles or too many sequences."""
    gate, x, h0, dh, dlast = make(cuda_device, B, L, D, "sigmoid", dt, seed=L)
    check(gate, x, "sigmoid", h0, dh, dlast)


def test_a_sequence_does_not_depend_on_its_neighbours(cuda_device):
    """Alone (a cluster's tiles) and among many (tiles that look back): the same bits."""
    gate, x, h0, dh, dlast = make(cuda_device, 300, 500, 24, "log", F32)
    out = slim.gated_scan_forward(gate, x, "log", h0=h0, keep=True)
    grads = slim.gated_scan_backward(gate, x, out[2], dh, "log", dlast=dlast)
    assert slim.gated_scan_workspace_size(300, 500, 24, F32) and not slim.gated_scan_workspace_size(1, 500, 24, F32)
    for b in (0, 7, 299):
        one = [t[b:b + 1].contiguous() for t in (gate, x, h0, dh, dlast)]
        a = slim.gated_scan_forward(one[0], one[1], "log", h0=one[2], keep=True)
        g = slim.gated_scan_backward(one[0], one[1], a[2], one[3], "log", dlast=one[4])
        assert all(torch.equal(p[0], q[b]) for p, q in zip((*a, *g), (*out, *grads)))


@pytest.mark.parametrize("B,L,D,kind,dt", [(8, 4096, 512, "value", F32), (2, 4097, 1000, "sigmoid", BF16),
                                           (1, 30000, 512, "log", BF16), (1, 9001, 77, "log", F32)])
def test_the_same_bits_beside_other_work(cuda_device, B, L, D, kind, dt):
    """Warps that are held up do not read what others have moved on to: the same bits every
    time, alone and with products on another stream, and those of the same sequence cut
    into pieces within the roundings of another order."""
    gate, x, h0, dh, dlast = make(cuda_device, B, L, D, kind, dt)
    other, side = torch.randn(4096, 4096, device=cuda_device).to(BF16), torch.cuda.Stream()

    def both():
        a = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
        return a + slim.gated_scan_backward(gate, x, a[2], dh, kind, dlast=dlast)

    ref = both()
    torch.cuda.synchronize()
    for i in range(20):
        if i % 2:
            with torch.cuda.stream(side):
                for _ in range(3):
                    other @ other
        out = both()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, ref)), i
    # pieces of up to 512 steps are clusters of a few tiles each
    s, pieces = h0, []
    for a in range(0, L, 512):
        g, u = gate[:, a:a + 512].contiguous(), x[:, a:a + 512].contiguous()
        h, s, kept = slim.gated_scan_forward(g, u, kind, h0=s, keep=True)
        pieces.append((g, u, h, kept))
    assert rel(torch.cat([p[2] for p in pieces], 1), ref[0]) < (1e-5 if dt == F32 else 4e-3) and rel(s, ref[1]) < 1e-5
    d, grads = dlast, []
    for i, (g, u, _, kept) in reversed(list(enumerate(pieces))):
        dg, du, d = slim.gated_scan_backward(g, u, kept, dh[:, 512 * i:512 * i + 512].contiguous(), kind, dlast=d)
        grads.append((dg, du))
    for k in range(2):
        assert rel(torch.cat([g[k] for g in reversed(grads)], 1), ref[3 + k]) < (1e-5 if dt == F32 else 4e-3)
    assert rel(d, ref[5]) < 1e-5


def test_two_calls_at_once(cuda_device):
    """Two streams whose tiles share the GPU, each with a workspace of its own."""
    sets = [make(cuda_device, 2, 9000, 96, "sigmoid", BF16, seed=i) for i in range(2)]
    ref = [slim.gated_scan_forward(s[0], s[1], "sigmoid", h0=s[2], keep=True) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, stream in zip(sets, streams):
            a = slim.gated_scan_forward(s[0], s[1], "sigmoid", h0=s[2], keep=True, stream=stream)
            got.append(a + slim.gated_scan_backward(s[0], s[1], a[2], s[3], "sigmoid", dlast=s[4], stream=stream))
        torch.cuda.synchronize()
        for s, r, a in zip(sets, ref, got):
            assert all(torch.equal(p, q) for p, q in zip(a, r))
            g = slim.gated_scan_backward(s[0], s[1], r[2], s[3], "sigmoid", dlast=s[4])
            assert all(torch.equal(p, q) for p, q in zip(a[3:], g))


@pytest.mark.parametrize("L", [5, 300, 5000])
@pytest.mark.parametrize("backward", [False, True])
def test_a_wait_that_gave_up_is_reported(cuda_device, backward, L):
    """The next call on the workspace launches nothing and says so; the one after it runs.
    The wait runs out on a barrier that nothing arrives at."""
    gate, x, h0, dh, dlast = make(cuda_device, 1, L, 16, "log", F32)
    ref = slim.gated_scan_forward(gate, x, "log", h0=h0, keep=True)
    ws = torch.full((1 << 21,), 255, dtype=torch.uint8, device=cuda_device)

    def call():
        if backward:
            return slim.gated_scan_backward(gate, x, ref[2], dh, "log", dlast=dlast, workspace=ws)
        return slim.gated_scan_forward(gate, x, "log", h0=h0, workspace=ws)

    want = call()  # whatever the workspace held
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert slim.library().slim_diag_wait_timeout(ws.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    before = slim.launch_count()
    with pytest.raises(slim.SlimError) as e:
        call()
    assert e.value.status == 5 and slim.launch_count() == before
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    if slim.gated_scan_workspace_size(1, L, 16, F32):  # (else the call has not touched it)
        slim.check_device_error(ws)


def test_same_bits_streams_and_graphs(cuda_device):
    gate, x, h0, dh, dlast = make(cuda_device, 2, 1500, 64, "sigmoid", BF16)

    def both(**kw):
        a = slim.gated_scan_forward(gate, x, "sigmoid", h0=h0, keep=True, **kw)
        return a + slim.gated_scan_backward(gate, x, a[2], dh, "sigmoid", dlast=dlast, **kw)

    ref = both()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for t in (gate, x, dh):
        t.copy_(t.flip(1))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    assert not torch.equal(got[0], ref[0])


def test_differences(cuda_device):
    """The kernel's gradient against differences of the kernel's forward along a random
    direction: steps of 2^-8 leave curvature of 2^-16 and roundings of 2^-24 * 2^8."""
    for kind in KINDS:
        gate, x, h0, dh, dlast = make(cuda_device, 1, 150, 8, kind, F32, resets=False, packed=False)
        _, _, kept = slim.gated_scan_forward(gate, x, kind, h0=h0, keep=True)
        grads = slim.gated_scan_backward(gate, x, kept, dh, kind, dlast=dlast)
        g = torch.Generator().manual_seed(1)
        for i, a in enumerate((gate, x, h0)):
            v = torch.randn(a.shape, generator=g).to(cuda_device) * 2.0 ** -8 * (0.1 if i == 0 else 1.0)
            val = []
            for s in (1.0, -1.0):
                args = [a + s * v if j == i else b for j, b in enumerate((gate, x, h0))]
                h, last = slim.gated_scan_forward(args[0], args[1], kind, h0=args[2])
                val.append((h.double() * dh.double()).sum().item() + (last.double() * dlast.double()).sum().item())
            want = (grads[i].double() * v.double()).sum().item()
            size = (grads[i].double().norm() * v.double().norm()).item()
            assert abs((val[0] - val[1]) / 2 - want) <= 4e-3 * size


def test_autograd(cuda_device):
    """The differentiable call, from a transposed projection, against autograd on the formula."""
    gate, x, h0, dh, dlast = make(cuda_device, 2, 90, 10, "log", F32, resets=False)

    def run(call, cast):
        a, b, c = (cast(t).requires_grad_() for t in (gate, x, h0))
        h, last = call(a, b.transpose(1, 2).contiguous().transpose(1, 2), "log", c)
        return torch.autograd.grad((h * cast(dh)).sum() + (last * cast(dlast)).sum(), (a, b, c))

    got = run(slim.gated_scan, lambda t: t.detach().clone())
    want = run(scan64, lambda t: t.detach().double())
    for a, b in zip(got, want):
        assert rel(a, b) < 1e-5
    a = x.detach().clone().requires_grad_()
    slim.gated_scan(gate, a, "log")[0].sum().backward()
    assert a.grad is not None
