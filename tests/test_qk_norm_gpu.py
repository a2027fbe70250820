"""Norms of queries and keys with the rotation by position, and their gradients,
against the formula in 64 bits.

Tolerances, from the arithmetic.  A row's sum of squares is a sum of d positive
terms, off by at most (d + 4) 2^-24 of itself; the norm's reciprocal square root by
half of that and 2^-22 of its own; weight, scale and the products add four roundings
of 2^-24.  cos and sin are off by at most 2^-23, and by what 53 bits leave of the
frequency at that position, 2^-51 |angle|.  So a value before its rounding is off by
at most E = (d + 40) 2^-24 + 2^-51 |angle| of the sizes of its pair, and the rounding
adds U.  A gradient r (g - n mean(g n)) is off by E of r |g|, and by 2 E of r |n|
mean |g n| (the mean's sum, and n in it and before it).  The weights' gradients sum R
rows: R 2^-24 + E of the sum of their sizes."""
import ctypes

import pytest
import torch

from layer_common import BF16, F32, U, angles64, partner, qk64, rel
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


def make(dev, B, Hq, Hk, L, d, dt, seed=0, packed=True, zeros=True):
    g = torch.Generator().manual_seed(seed)
    H = Hq + 2 * Hk
    rows = torch.randn(B, L, H, d, generator=g) * (0.1 + 3 * torch.rand(H, 1, generator=g))
    if zeros and L > 2:
        rows[:, L // 2] = 0.0  # a padded token
    rows = rows.to(dt).to(dev)
    q, k = rows[:, :, :Hq].transpose(1, 2), rows[:, :, Hq:Hq + Hk].transpose(1, 2)
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(dev) for _ in range(2)]
    up = [torch.randn(B, h, L, d, generator=g).to(dt).to(dev) for h in (Hq, Hk)]
    return q, k, w, up


def bounds(x, w, up, pos, freq, inter, eps, scale):
    """Per value: how far y and dx may be off before their rounding; per weight: dw."""
    B, H, L, d = x.shape
    x, w = x.double(), (torch.ones(d, device=x.device) if w is None else w).double()
    n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    E = torch.full((B, 1, L, 1), (d + 40) * 2.0 ** -24, dtype=torch.float64, device=x.device)
    pairs = 0 if freq is None else len(freq)
    if pairs:
        E = E + 2.0 ** -51 * angles64(pos, freq, B, L, x.device).abs().amax(-1, keepdim=True)
    y = E * partner(scale * n * w, pairs, inter)
    dz = abs(scale) * partner(up.double(), pairs, inter)
    r = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    g = dz * w.abs()
    dx = r * E * (g + 2 * n.abs() * (g * n.abs()).mean(-1, keepdim=True))
    R = B * H * L
    dw = ((R * 2.0 ** -24 + E) * dz * n.abs()).sum((0, 1, 2))
    return y, dx, dw


def check(q, k, w, up, pos=None, freq=None, inter=False, eps=1e-6, scale=1.0, **kw):
    how = dict(positions=pos, inv_freq=freq, interleaved=inter, eps=eps, scale=scale)
    out = slim.qk_norm_forward(q, k, *w, **how)
    grads = slim.qk_norm_backward(q, k, *w, *up, **how)
    for i, x in enumerate((q, k)):
        if x is None:
            assert out[i] is None and grads[i] is None
            continue
        x64 = x.double().requires_grad_()
        w64 = None if w[i] is None else w[i].double().requires_grad_()
        want = qk64(x64, w64, pos, freq, inter, eps, scale)
        wanted = torch.autograd.grad((want * up[i].double()).sum(), [x64] + ([] if w64 is None else [w64]))
        ey, edx, edw = bounds(x, w[i], up[i], pos, freq, inter, eps, scale)
        u, want = U[x.dtype], want.detach()
        assert out[i].dtype == grads[i].dtype == x.dtype and out[i].is_contiguous()
        assert ((out[i].double() - want).abs() <= ey + u * (want.abs() + ey) + 1e-37).all()
        assert ((grads[i].double() - wanted[0]).abs() <= edx + u * (wanted[0].abs() + edx) + 1e-37).all()
        if w64 is not None:
            assert grads[2 + i].dtype == F32
            assert ((grads[2 + i].double() - wanted[1]).abs() <= edw + 1e-37).all()
        else:
            assert grads[2 + i] is None
    return out, grads


SHAPES = [  # B, Hq, Hk, L, d, rotary
    (1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 2, 2), (2, 3, 1, 5, 7, 4), (1, 2, 2, 3, 8, 8), (3, 4, 2, 17, 16, 16),
    (2, 2, 1, 33, 36, 18), (2, 8, 8, 65, 64, 64), (1, 6, 2, 129, 64, 32), (8, 8, 8, 1, 64, 64),
    (1, 3, 3, 100, 96, 96), (1, 5, 1, 40, 128, 128), (1, 2, 1, 20, 250, 250), (2, 1, 1, 19, 256, 128),
    (1, 40, 7, 50, 32, 8), (1, 4096, 1, 2, 8, 8), (1, 1, 1, 3001, 24, 24)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hk,L,d,rotary", SHAPES)
@pytest.mark.parametrize("inter", [False, True])
def test_against_the_formula(cuda_device, B, Hq, Hk, L, d, rotary, dt, inter):
    q, k, w, up = make(cuda_device, B, Hq, Hk, L, d, dt)
    check(q, k, w, up, freq=slim.rotary_frequencies(rotary), inter=inter, scale=d ** -0.25)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("it", [torch.int32, torch.int64])
def test_positions(cuda_device, dt, it):
    """Any place: counted back from zero, far out, and where 32 bits of angle have nothing left."""
    q, k, w, up = make(cuda_device, 2, 2, 2, 40, 64, dt)
    pos = torch.arange(80).view(2, 40) * 53687091 - 2 ** 31 + 11
    freq = slim.rotary_frequencies(64)
    check(q, k, w, up, pos=pos.to(it).to(cuda_device), freq=freq)
    if it == torch.int64:
        check(q, k, w, up, pos=(pos * 1000).to(cuda_device), freq=freq)


def test_frequencies(cuda_device):
    """Given ones, zero and negative and faster than a turn among them, as numbers or a CPU tensor."""
    q, k, w, up = make(cuda_device, 1, 2, 2, 30, 16, F32)
    freq = [0.0, -1.0, 6.5, 100.25, -1e-9, 3.14159265358979, 2.0, 1e-300]
    a, _ = check(q, k, w, up, freq=freq)
    b = slim.qk_norm_forward(q, k, *w, inv_freq=torch.tensor(freq, dtype=torch.float64))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dt", [F32, BF16])
def test_without_weights_keys_or_rotation(cuda_device, dt):
    q, k, w, up = make(cuda_device, 2, 3, 2, 21, 48, dt)
    check(q, k, [None, None], up)
    check(q, k, [None, w[1]], up, freq=slim.rotary_frequencies(48))
    check(q, None, [w[0], None], [up[0], None], freq=slim.rotary_frequencies(16))
    dq, dk, a, b = slim.qk_norm_backward(q, k, *w, *up, weights=False)
    full = slim.qk_norm_backward(q, k, *w, *up)
    assert a is None and b is None and torch.equal(dq, full[0]) and torch.equal(dk, full[1])


@pytest.mark.parametrize("dt", [F32, BF16])
def test_layouts_agree(cuda_device, dt):
    """Contiguous, slices of a projection, odd starts and odd pitches: the same bits."""
    q, k, w, up = make(cuda_device, 2, 3, 2, 37, 64, dt)
    how = dict(inv_freq=slim.rotary_frequencies(64), scale=0.5)
    ref = slim.qk_norm_forward(q, k, *w, **how)
    refg = slim.qk_norm_backward(q, k, *w, *up, **how)

    def moved(t, pitch, start):
        B, H, L, d = t.shape
        buf = torch.zeros(B * L * H * pitch + start + 8, dtype=dt, device=t.device)
        view = buf[start:start + B * L * H * pitch].view(B, L, H, pitch)[..., :d].transpose(1, 2)
        view.copy_(t)
        return view

    for pitch, start in ((64, 1), (64, 4), (67, 0), (68, 8), (72, 3)):
        q2, k2, dq2, dk2 = (moved(t, pitch, start) for t in (q, k, *up))
        oq, ok_ = (moved(torch.zeros_like(t), pitch, start) for t in ref)
        got = slim.qk_norm_forward(q2, k2, *w, q_out=oq, k_out=ok_, **how)
        assert got[0] is oq and torch.equal(oq, ref[0]) and torch.equal(ok_, ref[1])
        g = slim.qk_norm_backward(q2, k2, *w, dq2, dk2, dq=oq, dk=ok_, **how)
        assert all(torch.equal(a, b) for a, b in zip(g[:2], refg[:2]))
        # rows meet in the weights' sums in an order that goes by the vectors' width: either
        # order is off by at most (rows - 1) 2^-24 of the sum of the terms' sizes, |up n| scale
        # with |n| <= sqrt(d) and two of up's features in a turned one
        for a, b, u in zip(g[2:], refg[2:], up):
            size = 2 * 0.5 * 8 * u.double().abs().sum((0, 1, 2))
            size = size + size.roll(32)
            assert ((a - b).abs() <= 2 * 2 * 3 * 37 * 2.0 ** -24 * size).all()
    # read through a stride of zero: one token's rows for every batch and head
    one = q[:1, :1].expand(2, 3, 37, 64)
    assert torch.equal(slim.qk_norm_forward(one, None, w[0], **how)[0],
                       slim.qk_norm_forward(one.contiguous(), None, w[0], **how)[0])


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d,rotary", [(64, 64), (36, 18)])
def test_in_place(cuda_device, dt, d, rotary):
    q, k, w, up = make(cuda_device, 2, 3, 2, 37, d, dt)
    how = dict(inv_freq=slim.rotary_frequencies(rotary), interleaved=True)
    ref = slim.qk_norm_forward(q, k, *w, **how)
    refg = slim.qk_norm_backward(q, k, *w, *up, **how)
    g = slim.qk_norm_backward(q, k, *w, *up, dq=up[0], dk=up[1], **how)
    assert g[0] is up[0] and all(torch.equal(a, b) for a, b in zip(g, refg))
    slim.qk_norm_forward(q, k, *w, q_out=q, k_out=k, **how)
    assert torch.equal(q, ref[0]) and torch.equal(k, ref[1])


def test_only_the_rows_are_written(cuda_device):
    """Values between and behind the rows stay as they were."""
    q, k, w, _ = make(cuda_device, 2, 2, 2, 9, 40, BF16)
    rows = torch.full((2, 9, 7, 40), 7.0, dtype=BF16, device=cuda_device)
    slim.qk_norm_forward(q, k, *w, q_out=rows[:, :, 1:3].transpose(1, 2), k_out=rows[:, :, 4:6].transpose(1, 2))
    assert (rows[:, :, [0, 3, 6]] == 7.0).all() and (rows[:, :, 1] != 7.0).any()


def test_values_at_the_ends_of_the_range(cuda_device):
    """Rows whose squares overflow or vanish; an infinity or NaN stays in its row."""
    x = torch.randn(1, 1, 64, 64, generator=torch.Generator().manual_seed(3)).to(cuda_device)
    big, small = x * 1e38, x * 1e-30
    y = qk64(x.double(), None, None, None, False, 1e-30, 1.0)
    assert rel(slim.qk_norm_forward(big.clamp(-3e38, 3e38), None, eps=1e-6)[0],
               qk64(big.clamp(-3e38, 3e38).double(), None, None, None, False, 1e-6, 1.0)) < 1e-6
    assert rel(slim.qk_norm_forward(x * 1e18, None)[0], y) < 1e-6
    assert rel(slim.qk_norm_forward(small, None)[0], small.double() * 1e3) < 1e-6
    dq = slim.qk_norm_backward(x * 1e25, None, None, None, x.flip(2), None)[0]
    v = (x.double() * 1e25).requires_grad_()
    want = torch.autograd.grad((qk64(v, None, None, None, False, 1e-6, 1.0) * x.flip(2).double()).sum(), v)[0]
    assert rel(dq, want) < 1e-5
    bad = x.clone()
    bad[0, 0, 5, 3], bad[0, 0, 20, 60], bad[0, 0, 33] = float("inf"), float("nan"), -float("inf")
    ok = slim.qk_norm_forward(x, None, inv_freq=slim.rotary_frequencies(64))[0]
    got = slim.qk_norm_forward(bad, None, inv_freq=slim.rotary_frequencies(64))[0]
    rows = [i for i in range(64) if i not in (5, 20, 33)]
    assert torch.equal(got[:, :, rows], ok[:, :, rows])
    assert all(got[0, 0, i].isnan().any() for i in (5, 20, 33))


def test_nothing_to_do(cuda_device):
    w = torch.ones(8, device=cuda_device)
    for B, L in ((0, 4), (4, 0)):
        q = torch.zeros(B, 2, L, 8, device=cuda_device)
        a, b = slim.qk_norm_forward(q, q, w, w)
        assert a.shape == q.shape and b.shape == q.shape
        dq, dk, dwq, dwk = slim.qk_norm_backward(q, q, w, w, q, q)
        assert dq.shape == q.shape and (dwq == 0).all() and (dwk == 0).all()


def test_same_bits_streams_and_graphs(cuda_device):
    q, k, w, up = make(cuda_device, 2, 4, 2, 700, 64, BF16)
    how = dict(inv_freq=slim.rotary_frequencies(64))

    def both(**kw):
        return slim.qk_norm_forward(q, k, *w, **how, **kw) + slim.qk_norm_backward(q, k, *w, *up, **how, **kw)

    ref = both()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = both(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for t in (q, k, *up):
        t.copy_(t.flip(2))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, both()))
    assert not torch.equal(got[0], ref[0])


def test_differences(cuda_device):
    """The kernel's gradient against differences of the kernel's forward: along a random
    direction, steps of 2^-7 leave third-order terms of 2^-14 and roundings of 2^-24 * 2^7."""
    q, k, w, up = make(cuda_device, 2, 2, 2, 50, 32, F32, packed=False, zeros=False)
    how = dict(inv_freq=slim.rotary_frequencies(32))
    g = torch.Generator().manual_seed(5)
    args = [q, k, *w]
    grads = slim.qk_norm_backward(*args, *up, **how)
    for i, a in enumerate(args):
        size = a.double().square().mean().sqrt().item()
        v = torch.randn(a.shape, generator=g).to(cuda_device) * 2.0 ** -7 * min(size, 0.1)
        val = []
        for s in (1.0, -1.0):
            moved = [a + s * v if j == i else b for j, b in enumerate(args)]
            out = slim.qk_norm_forward(*moved, **how)
            val.append(sum((o.double() * u.double()).sum().item() for o, u in zip(out, up)))
        want = (grads[i].double() * v.double()).sum().item()
        scale = (grads[i].double().norm() * v.double().norm()).item()
        assert abs((val[0] - val[1]) / 2 - want) <= 2e-3 * scale


def test_autograd(cuda_device):
    """The differentiable call through a projection's rows, with a weight shared by both
    sides, against autograd on the formula."""
    q, k, w, up = make(cuda_device, 2, 4, 2, 33, 64, F32)
    freq = slim.rotary_frequencies(64)
    pos = (torch.arange(66, device=cuda_device).view(2, 33) * 7) % 50

    def run(call, cast):
        a, b, s = cast(q).requires_grad_(), cast(k).requires_grad_(), cast(w[0]).requires_grad_()
        out = call(a, b, s)
        return torch.autograd.grad(sum((o * cast(u)).sum() for o, u in zip(out, up)), (a, b, s))

    got = run(lambda a, b, s: slim.qk_norm(a, b, s, s, positions=pos, inv_freq=freq, scale=0.35),
              lambda t: t.detach().clone(memory_format=torch.preserve_format))
    want = run(lambda a, b, s: [qk64(t, s, pos, freq, False, 1e-6, 0.35) for t in (a, b)], lambda t: t.detach().double())
    for a, b in zip(got, want):
        assert rel(a, b) < 1e-5
    # one output unused, one input without a gradient
    a = q.detach().clone().requires_grad_()
    out, none = slim.qk_norm(a, None, None, None, inv_freq=freq)
    out.sum().backward()
    assert none is None and a.grad is not None


def test_offsets_past_32_bits(cuda_device):
    """Rows that lie further than 2^31 elements apart."""
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 12 GB")
    buf = torch.empty((1 << 32) + (1 << 31), dtype=BF16, device=cuda_device)
    q = torch.as_strided(buf, (2, 2, 3, 64), (1 << 32, 1 << 30, 1 << 20, 1))
    small = torch.randn(2, 2, 3, 64, generator=torch.Generator().manual_seed(1)).to(BF16).to(cuda_device)
    q.copy_(small)
    freq = slim.rotary_frequencies(64)
    want = slim.qk_norm_forward(small, None, inv_freq=freq)[0]
    slim.qk_norm_forward(q, None, inv_freq=freq, q_out=q)
    assert torch.equal(q.contiguous(), want)
