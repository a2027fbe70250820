"""Clipping by the global norm, against the definition in 64 bits.

Tolerances.  A thread adds at most 130 squares in fp32 before its sum moves to
fp64, so the sum of squares is within 131 * 2^-24 of the exact one and the norm,
its root rounded to fp32, within 67 * 2^-24.  A clipped element carries the
factor's error (the norm's plus one rounding) and its own product's rounding in
fp32 and in its type (2^-24 or 2^-8)."""
import math

import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
NORM_TOL = 67 * 2.0 ** -24


def norm64(ts):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


def check(grads, max_norm, out=None):
    """Clips copies of the grads and compares."""
    n = norm64(grads)
    factor = 1.0 if n <= max_norm else max_norm / n
    src = [g.clone() if out is None else g for g in grads]
    norm = slim.clip_grad_norm(src, max_norm, out=out)
    got = src if out is None else out
    assert norm.shape == (1,) and norm.dtype == F32
    assert abs(norm.item() - n) <= NORM_TOL * n
    for g, o in zip(grads, got):
        ref = g.double() * factor
        tol = NORM_TOL + 3 * 2.0 ** -24 + (UNIT[g.dtype] if factor != 1.0 else 0.0)
        assert ((o.double() - ref).abs() <= tol * ref.abs() + 2.0 ** -133).all()


def make(dev, sizes, dts, scale=1.0, seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return [(torch.randn(n, generator=g, device=dev) * scale).to(dts[i % len(dts)])
            for i, n in enumerate(sizes)]


@pytest.mark.parametrize("dts", [(F32,), (BF16,), (BF16, F32, BF16)])
@pytest.mark.parametrize("sizes", [(1,), (3, 1, 2), (0, 5, 0), (1023, 16384, 16385, 32768, 32769),
                                   (300007, 64, 9, 1 << 20), (257,) * 300, (65,) * 1500])
@pytest.mark.parametrize("clipped", [True, False])
def test_clip(cuda_device, dts, sizes, clipped):
    grads = make(cuda_device, sizes, dts)
    n = norm64(grads)
    check(grads, 0.3 * n if clipped else 2.0 * n + 1.0)
    check(grads, 0.3 * n if clipped else 2.0 * n + 1.0, out=[torch.empty_like(g) for g in grads])


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("a,b", [(0, 1), (1, 0), (1, 1), (3, 5), (7, 7), (5, 13)])
def test_slices_at_any_element(cuda_device, dt, a, b):
    """Source and target start a and b elements into their buffers."""
    n = 70001
    buf = make(cuda_device, (n + 20,), (dt,))[0]
    dst = torch.full((n + 40,), 7.0, device=cuda_device, dtype=dt)
    check([buf[a:a + n]], 3.0, out=[dst[b + 1:b + 1 + n]])
    assert (dst[:b + 1] == 7.0).all() and (dst[b + 1 + n:] == 7.0).all()
    check([buf[a:a + n]], 3.0)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("scale", [1e30, 1e-30, 1e18, 1e-22, 1e-38, 2.0 ** -140])
def test_range(cuda_device, dt, scale):
    """Squares outside fp32's range: the norm is still right."""
    if scale < 1e-38 and dt == F32:
        scale = 2.0 ** -130
    grads = make(cuda_device, (5000, 70000), (dt,), scale=scale)
    n = norm64(grads)
    norm = slim.clip_grad_norm([g.clone() for g in grads], 1.0)
    # a norm below 2^-126 is rounded to a multiple of 2^-149
    assert abs(norm.item() - n) <= NORM_TOL * n + 2.0 ** -149


def test_mixed_magnitudes(cuda_device):
    """Huge, tiny and zero tensors together."""
    grads = make(cuda_device, (4000, 4000, 4000, 4000), (F32,))
    for g, s in zip(grads, (1e25, 1e-25, 0.0, 1.0)):
        g.mul_(s)
    check(grads, 1e20)


def test_zero_gradients(cuda_device):
    grads = [torch.zeros(70000, device=cuda_device), torch.zeros(33, device=cuda_device, dtype=BF16)]
    norm = slim.clip_grad_norm(grads, 1.0)
    assert norm.item() == 0.0 and all((g == 0).all() for g in grads)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_nonfinite_is_reported_and_scales_nothing(cuda_device, bad, dt):
    grads = make(cuda_device, (30000, 100), (dt,))
    grads[0][29999] = bad
    before = [g.clone() for g in grads]
    out = [torch.empty_like(g) for g in grads]
    norm = slim.clip_grad_norm(grads, 1e-3, out=out)
    assert not math.isfinite(norm.item())
    for g, b, o in zip(grads, before, out):
        assert torch.equal(g.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(torch.nan_to_num(o), torch.nan_to_num(b))


def test_same_bits_again_and_on_another_stream(cuda_device):
    grads = make(cuda_device, (1 << 20, 12345, 3), (F32, BF16))
    outs = [[torch.empty_like(g) for g in grads] for _ in range(3)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    norms = [slim.clip_grad_norm(grads, 1.0, out=o, stream=st)
             for o, st in zip(outs, (None, None, s))]
    torch.cuda.synchronize()
    assert norms[0].item() == norms[1].item() == norms[2].item()
    for a, b, c in zip(*outs):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_infinite_max_norm_measures_only(cuda_device):
    grads = make(cuda_device, (999,), (F32,))
    check(grads, float("inf"))


def test_refusals(cuda_device):
    g = torch.ones(8, device=cuda_device)
    with pytest.raises(ValueError):
        slim.clip_grad_norm([g, g], 1.0)
    with pytest.raises(ValueError):
        slim.clip_grad_norm([g], 1.0, out=[])
    with pytest.raises(ValueError):
        slim.clip_grad_norm([g], 1.0, out=[g.to(BF16)])
    with pytest.raises(TypeError):
        slim.clip_grad_norm([g.half()], 1.0)
    with pytest.raises(RuntimeError):
        slim.clip_grad_norm([torch.ones(8, 8, device=cuda_device).t()[:, ::2]], 1.0)
    with pytest.raises(slim.SlimError) as e:
        slim.clip_grad_norm([g], 0.0)
    assert e.value.status == 1
