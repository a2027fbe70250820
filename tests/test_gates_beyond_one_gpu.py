"""Gates beyond 1 whose product passes fp32's range where nothing is there to grow: a
state of zero stays zero, and a gradient of zero, in any length and form."""
import math

import pytest
import torch

from layer_common import BF16, F32, rel
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

LENGTHS = [5, 9, 64, 200, 1500, 5000]


def full(shape, kind, dt, dev):
    return torch.full(shape, 100.0 if kind == "value" else math.log(100.0), device=dev).to(dt)


def noise(dev, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(0)).to(dev)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("kind", ["value", "log"])
@pytest.mark.parametrize("L", LENGTHS)
def test_a_state_of_zero_stays(cuda_device, L, kind, dt):
    gate = full((2, L, 6), kind, dt, cuda_device)
    x = torch.zeros_like(gate)
    h, last, kept = slim.gated_scan_forward(gate, x, kind, keep=True)
    assert (h == 0).all() and (last == 0).all() and (kept == 0).all()
    dgate, dx, dh0 = slim.gated_scan_backward(gate, x, kept, x, kind)
    assert (dgate == 0).all() and (dx == 0).all() and (dh0 == 0).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("start", [False, True])
@pytest.mark.parametrize("L", LENGTHS)
def test_what_comes_behind(cuda_device, L, start, dt):
    """Inputs begin behind the large gates (`start`: after a new start among them, which a
    state forgets): the same as the sequence from there on."""
    cut = L // 2
    gate = full((2, L, 6), "value", dt, cuda_device)
    gate[:, cut:] = (0.5 + 0.4 * noise(cuda_device, 2, L - cut, 6).tanh()).to(dt)
    x = torch.zeros_like(gate)
    x[:, cut:] = noise(cuda_device, 2, L - cut, 6).to(dt)
    h0 = torch.zeros(2, 6, device=cuda_device)
    if start:
        h0 += 3.0
        gate[:, 0] = 0.0
    h, last = slim.gated_scan_forward(gate, x, "value", h0=h0)
    clean, clean_last = slim.gated_scan_forward(gate[:, cut:].contiguous(), x[:, cut:].contiguous(), "value")
    assert (h[:, :cut] == 0).all()
    # steps are joined in another order: a rounding a step that counts (ten, gates below 0.9)
    assert rel(last, clean_last) <= 1e-5 and rel(h[:, cut:], clean) <= (1e-5 if dt == F32 else 4e-3)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("L", LENGTHS)
def test_gradients_from_before(cuda_device, L, dt):
    """Gradients of the first half alone; the gates of the second are the large ones."""
    cut = L // 2
    gate = full((2, L, 6), "value", dt, cuda_device)
    gate[:, :cut] = (0.5 + 0.4 * noise(cuda_device, 2, cut, 6).tanh()).to(dt)
    x = torch.zeros_like(gate)
    dh = torch.zeros_like(gate)
    dh[:, :cut] = noise(cuda_device, 2, cut, 6).to(dt)
    _, _, kept = slim.gated_scan_forward(gate, x, "value", keep=True)
    dgate, dx, dh0 = slim.gated_scan_backward(gate, x, kept, dh, "value")
    assert (dgate == 0).all() and (dx[:, cut:] == 0).all()
    a, b, c = (t[:, :cut].contiguous() for t in (gate, x, dh))
    _, _, kept = slim.gated_scan_forward(a, b, "value", keep=True)
    _, want, want0 = slim.gated_scan_backward(a, b, kept, c, "value")
    assert rel(dh0, want0) <= 1e-5 and rel(dx[:, :cut], want) <= (1e-5 if dt == F32 else 4e-3)


@pytest.mark.parametrize("L", [64, 1500, 5000])
def test_a_state_that_is_not_a_number_stays(cuda_device, L):
    """A NaN among the gates, an infinite input: not taken for a state of zero."""
    gate = full((1, L, 4), "value", F32, cuda_device)
    x = torch.zeros_like(gate)
    gate[0, 3, 1], x[0, 3, 2] = math.nan, math.inf
    h, last = slim.gated_scan_forward(gate, x, "value")
    assert (h[0, :, [0, 3]] == 0).all() and (last[0, [0, 3]] == 0).all()
    assert (h[0, :3] == 0).all() and not h[0, 3:, 1:3].isfinite().any() and not last[0, 1:3].isfinite().any()
