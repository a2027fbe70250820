"""Clipping by the global norm at the edges of its lists and of fp32's range.

Tolerances as in test_clip_gpu.py: the norm within 67 * 2^-24 of the one in 64
bits, an element within that, three roundings in fp32 and one to its type."""
import math

import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NORM_TOL = 67 * 2.0 ** -24


def norm64(ts):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))


@pytest.mark.parametrize("live", [127, 128, 129, 1023, 1024, 1025])
@pytest.mark.parametrize("lead,trail", [(0, 0), (0, 1), (3, 700), (1, 1100)])
def test_empty_tensors_around_a_full_list(cuda_device, live, lead, trail):
    """As many tensors as a launch holds, with empty ones around them, and enough
    elements for every block to leave a partial sum: nothing is written past the
    workspace, and every element is counted once."""
    g = torch.Generator(device=cuda_device).manual_seed(live)
    sizes = [0] * lead + [8192] * live + [0] * trail
    grads = [torch.randn(n, generator=g, device=cuda_device) for n in sizes]
    n = norm64(grads)
    before = [t.clone() for t in grads]
    need = slim.clip_workspace_size(len(grads))
    held = torch.full((need + 65536,), 0xA5, dtype=torch.uint8, device=cuda_device)
    launches = slim.launch_count()
    norm = slim.clip_grad_norm(grads, 0.5 * n, workspace=held[:need])
    assert slim.launch_count() - launches == 2 * (1 if live <= 128 else -(-live // 1024))
    assert (held[need:] == 0xA5).all()
    assert abs(norm.item() - n) <= NORM_TOL * n
    tol = NORM_TOL + 5 * 2.0 ** -24
    for a, b in zip(grads, before):
        ref = b.double() * 0.5
        assert ((a.double() - ref).abs() <= tol * ref.abs()).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n", [20, 100000])
def test_finite_gradients_whose_norm_passes_fp32(cuda_device, dt, in_place, n):
    """What the caller reads is an infinity: as for any norm that is not finite,
    the gradients are passed on as they are.  One step below, they are clipped."""
    value = 3.0e38 / math.sqrt(n) * 1.5
    grads = [torch.full((n,), value, dtype=dt, device=cuda_device), torch.ones(9, device=cuda_device)]
    before = [g.clone() for g in grads]
    out = None if in_place else [torch.empty_like(g) for g in grads]
    norm = slim.clip_grad_norm(grads, 1e30, out=out)
    assert math.isinf(norm.item())
    for b, o in zip(before, grads if in_place else out):
        assert torch.equal(b, o)
    grads[0].copy_(before[0].double() * 0.5)
    n64 = norm64(grads)
    assert n64 < torch.finfo(F32).max
    ref = [g.double() * (1e30 / n64) for g in grads]
    norm = slim.clip_grad_norm(grads, 1e30, out=out)
    assert abs(norm.item() - n64) <= NORM_TOL * n64
    unit = 2.0 ** -24 if dt == F32 else 2.0 ** -8
    for r, o in zip(ref, grads if in_place else out):
        assert ((o.double() - r).abs() <= (NORM_TOL + 5 * 2.0 ** -24 + unit) * r.abs()).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("value,max_norm", [(1e36, 1.0), (1e36, 1e-3), (1e36, 1e-7), (1e33, 1e-9),
                                            (1e36, 1e-30), (1e36, 1e-37)])
def test_factors_below_fp32s_normal_range(cuda_device, dt, value, max_norm):
    """max_norm / norm down to 1e-75: the clipped gradients keep their digits (an
    element below 2^-126 to a multiple of the type's least number)."""
    g = torch.Generator(device=cuda_device).manual_seed(1)
    grads = [(torch.randn(n, generator=g, device=cuda_device) * value).to(dt) for n in (70001, 300)]
    n64 = norm64(grads)
    ref = [t.double() * (max_norm / n64) for t in grads]
    # max_norm reaches the kernel in fp32
    assert abs(slim.clip_grad_norm(grads, max_norm).item() - n64) <= NORM_TOL * n64
    unit, least = (2.0 ** -24, 2.0 ** -149) if dt == F32 else (2.0 ** -8, 2.0 ** -133)
    for r, o in zip(ref, grads):
        tol = (NORM_TOL + 6 * 2.0 ** -24 + unit) * r.abs() + least
        assert ((o.double() - r).abs() <= tol).all()
