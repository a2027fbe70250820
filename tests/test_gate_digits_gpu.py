"""The gates of the recurrence to their last digits: a gate that keeps nearly everything
is applied to a state thousands of times over, and its error counts as often.

Tolerances, from the arithmetic.  A step from h0 = 1 with x = 0 gives the gate itself.
Rounded once, a gate below 1 is off by at most 2^-25 and one above by 2^-24; a series cut
off behind its last term adds less than a fourth of that.  Log gates further out are off
by 2^-22 (the exponential's own bound), with fp32 inputs by 2^-24 for a last rounding and
|g| 2^-28 for a constant's, with bf16 inputs by 1.25 |g| 2^-24 through the argument of
2^(g log2 e).  A sigmoid gate is 1 - small with small = e^-g / (1 + e^-g) off by 2^-21 of
itself (the exponential as above, a sum, a reciprocal and a product)."""
import math

import pytest
import torch

from layer_common import BF16, F32
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


def gates_at(g, kind, L, at):
    """The gates themselves: each channel's applied once, at step `at`, to a state of 1."""
    keep = {"log": 0.0, "sigmoid": math.inf}[kind]  # gates of one
    gate = torch.full((1, L, g.numel()), keep, dtype=g.dtype, device=g.device)
    gate[0, at] = g
    x = torch.zeros_like(gate)
    _, last = slim.gated_scan_forward(gate, x, kind, h0=torch.ones(1, g.numel(), device=g.device))
    return last[0].double()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("L,at", [(1, 0), (9, 3), (700, 500), (70000, 40001)])
def test_log_gates(cuda_device, L, at, dt):
    near = torch.logspace(-9, math.log10(2.0 ** -6) - 1e-3, 500, device=cuda_device).to(dt)
    a = gates_at(torch.cat([-near, near]), "log", L, at)
    g = torch.cat([-near, near]).double()
    half = torch.where(g < 0, 2.0 ** -25, 2.0 ** -24)
    assert ((a - g.exp()).abs() <= 1.25 * half).all()
    far = -torch.logspace(math.log10(2.0 ** -6), math.log10(86.0), 500, device=cuda_device).to(dt)
    a, g = gates_at(far, "log", L, at), far.double()
    tol = 2.0 ** -22 + (2.0 ** -24 + g.abs() * 2.0 ** -28 if dt == F32 else 1.25 * g.abs() * 2.0 ** -24)
    assert ((a - g.exp()).abs() <= tol * g.exp()).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("L,at", [(1, 0), (9, 3), (700, 500), (70000, 40001)])
def test_sigmoid_gates(cuda_device, L, at, dt):
    size = torch.linspace(0.0, 40.0, 400, device=cuda_device).to(dt)
    g = size.double()
    rest = torch.sigmoid(-g)
    more = 0.0 if dt == F32 else 1.25 * g * 2.0 ** -24
    a = gates_at(size, "sigmoid", L, at)
    assert ((a - torch.sigmoid(g)).abs() <= 1.25 * 2.0 ** -25 + (2.0 ** -21 + more) * rest).all()
    a = gates_at(-size, "sigmoid", L, at)
    assert ((a - rest).abs() <= (2.0 ** -21 + more) * rest).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("kind", ["log", "sigmoid"])
def test_long_memories(cuda_device, kind, dt):
    """65536 steps of one gate and one input a channel, memories of a hundred to a million
    steps, against the sum in closed form.  Each step's gate, the products that join
    steps and the state round once: 2^-25 and 2 * 2^-24 a step, over the steps that count."""
    L = 65536
    g = torch.logspace(-6, -2, 32, device=cuda_device)
    g = (-g if kind == "log" else -(g.log())).to(dt)
    x = torch.full((1, L, 32), 0.5, device=cuda_device).to(dt)
    h0 = torch.linspace(0.5, 2.0, 32, device=cuda_device).view(1, 32)
    h, last = slim.gated_scan_forward(g.expand(1, L, 32).contiguous(), x, kind, h0=h0)
    lg = g.double() if kind == "log" else -torch.nn.functional.softplus(-g.double())
    rest = -torch.expm1(lg)
    ones = (0.5 if kind == "sigmoid" else 0.5 / rest) * -torch.expm1(L * lg)
    want = (L * lg).exp() * h0.double() + ones
    steps = torch.clamp(1.0 / rest, max=float(L))
    # (a sigmoid's own factor of x adds 2^-21)
    tol = 1.25 * 2.5 * 2.0 ** -24 * steps + 2.0 ** -20
    assert ((last.double() - want).abs() <= tol * want).all()
