"""Sizes whose offsets pass 32 bits: rows far apart in the gated recurrence, more than
2^31 features and rows in the gated feed-forward."""
import pytest
import torch

from layer_common import BF16, F32, U, ff64, rel
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


def test_scan_rows_far_apart(cuda_device):
    """Slices of rows of 65536 give the bits of dense ones, read and written."""
    B, L, D, pitch = 2, 40000, 64, 65536
    g = torch.Generator(device=cuda_device).manual_seed(1)
    wide = torch.empty(B, L, pitch, dtype=BF16, device=cuda_device)
    gate, x = wide[..., 64:128], wide[..., -64:]
    gate.copy_(1.5 * torch.randn(B, L, D, generator=g, device=cuda_device) + 2.0)
    x.copy_(torch.randn(B, L, D, generator=g, device=cuda_device))
    dh = torch.randn(B, L, D, generator=g, device=cuda_device).to(BF16)
    out = slim.gated_scan_forward(gate, x, keep=True)
    a, b = gate.contiguous(), x.contiguous()
    ref = slim.gated_scan_forward(a, b, keep=True)
    assert all(torch.equal(p, q) for p, q in zip(out, ref))
    refg = slim.gated_scan_backward(a, b, ref[2], dh)
    got = slim.gated_scan_backward(gate, x, out[2], dh, dgate=gate, dx=x)
    assert all(torch.equal(p, q) for p, q in zip(got, refg))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_feed_forward_past_32_bits(cuda_device, dt):
    """More than 2^31 features and rows: the first and last rows, and dw's sums.  A row's
    error is that of 16 products and of one rounding of h (of dz as well for dx); dw adds
    2^20 of them, in parts of 32768 joined in fp32, each low by at most 2.4e-4 where all
    have one sign."""
    N, D, F = (1 << 20) + 300, 16, 2064
    assert N * F > 1 << 31
    g = torch.Generator(device=cuda_device).manual_seed(2)
    x = torch.randn(N, D, generator=g, device=cuda_device).to(dt)
    w = (torch.randn(2 * F, D, generator=g, device=cuda_device) / 4).to(dt)
    dh = torch.empty(N, F, dtype=dt, device=cuda_device)
    for a in range(0, N, 1 << 17):
        dh[a:a + (1 << 17)] = torch.randn(min(1 << 17, N - a), F, generator=g, device=cuda_device).to(dt)
    h, z = slim.gated_ff_forward(x, w, "silu", keep=True)
    dx, dw = slim.gated_ff_backward(x, w, dh, "silu", z=z)
    w64 = w.double()
    want_dw = torch.zeros(2 * F, D, dtype=torch.float64, device=cuda_device)
    for a in range(0, N, 1 << 15):
        rows = x[a:a + (1 << 15)].double().requires_grad_()
        out = ff64(rows, w64, "silu")
        zz = (rows @ w64.T).detach()
        s = torch.sigmoid(zz[:, :F])
        d64 = dh[a:a + (1 << 15)].double()
        dz = torch.cat([d64 * zz[:, F:] * s * (1 + zz[:, :F] * (1 - s)), d64 * zz[:, :F] * s], 1)
        want_dw += dz.T @ rows.detach()
        if a == 0 or a + (1 << 15) >= N:
            assert rel(h[a:a + (1 << 15)], out.detach()) <= U[dt] + 2.0 ** -20
            assert rel(dx[a:a + (1 << 15)], dz @ w64) <= 2 * U[dt] + 2.0 ** -20
    assert rel(dw, want_dw) <= 2 * U[dt] + 2.4e-4
