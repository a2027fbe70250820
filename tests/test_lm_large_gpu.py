"""Sizes whose offsets pass 32 bits: more than 2^31 elements in the backward's
piece, in an embedding table and in one gradient."""
import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu


def test_vocab_loss_piece_past_32_bits(cuda_device):
    """One piece of 65537 x 65536 elements of g against pieces of 8192: dw takes the
    same sums either way; dx's differ in order only, each within the bf16 result's
    rounding of the other (two roundings of 2^-8)."""
    g = torch.Generator(device=cuda_device).manual_seed(1)
    N, D, V = 65537, 32, 65536
    x = torch.randn(N, D, generator=g, device=cuda_device).bfloat16()
    w = torch.randn(V, D, generator=g, device=cuda_device).bfloat16()
    t = torch.randint(0, V, (N,), generator=g, device=cuda_device)
    _, lse, total = slim.vocab_loss_forward(x, w, t)
    one = torch.ones(1, device=cuda_device)
    dx, dw = slim.vocab_loss_backward(x, w, t, lse, one, count=total[1:], piece=V)
    ex, ew = slim.vocab_loss_backward(x, w, t, lse, one, count=total[1:], piece=8192)
    assert torch.equal(dw, ew)
    assert ((dx.double() - ex.double()).norm() <= 2.0 ** -7 * ex.double().norm()).item()
    # the last rows against the definition (rel-L2 5e-3, as for every bf16 gradient)
    a = x[-50:].double()
    z = a @ w.double().T
    p = torch.softmax(z, 1)
    p[torch.arange(50), t[-50:]] -= 1
    ref = p @ w.double() / N
    assert ((dx[-50:].double() - ref).norm() <= 5e-3 * ref.norm()).item()


def test_embedding_table_past_32_bits(cuda_device):
    V, D = (1 << 22) + 5, 520
    table = torch.zeros(V, D, dtype=torch.bfloat16, device=cuda_device)
    ids = torch.tensor([0, V - 1, V - 2, V, (1 << 32) + 1, V - 1, 1 << 21], device=cuda_device)
    ok = (ids >= 0) & (ids < V)
    rows = torch.randn(7, D, device=cuda_device).bfloat16()
    table[ids[ok]] = rows[ok]
    out = slim.embed_forward(ids, table, 2.0)
    assert torch.equal(out[ok], 2 * table[ids[ok]]) and (out[~ok] == 0).all()
    grad = slim.embed_backward(ids, rows, V, 1.0)
    ref = torch.zeros(7, D, dtype=torch.float64, device=cuda_device)
    for i in range(7):
        ref[i] = sum(rows[k].double() for k in range(7) if ids[k] == ids[i])
    assert torch.equal(grad[ids[ok]], ref[ok].bfloat16())
    assert torch.count_nonzero(grad) == torch.count_nonzero(grad[ids[ok].unique()])


def test_one_gradient_past_32_bits(cuda_device):
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.5, dtype=torch.bfloat16, device=cuda_device)
    g[-1] = 4096.0
    norm = (n * 0.25 - 0.25 + 4096.0 ** 2) ** 0.5
    got = slim.clip_grad_norm([g], norm / 4)
    assert abs(got.item() - norm) <= 67 * 2.0 ** -24 * norm
    assert g[-1].item() == 1024.0 and g[0].item() == 0.125
    assert (g[:-1].view(torch.int16) == g[0].view(torch.int16)).all()
