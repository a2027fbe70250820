"""Embedding lookup with scaling and its table gradient, against the definition
in 64 bits.

Tolerances.  The forward is one fp32 product rounded once more for bf16: fp32
results equal the rounded exact product, bf16 ones are within 2^-8 (1 + 2^-10)
of it (a second rounding on top of fp32's).  A gradient element is a sum of n
fp32 terms in some order, scaled, and rounded: within (n + 2) 2^-24 of the sum
of the terms' magnitudes, plus the rounding to its type (2^-24 or 2^-8)."""
import pytest
import torch

from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def inputs(dev, N, D, V, dt, it=torch.int64, kind="skewed", seed=0):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(N, generator=g)
    ids = {"skewed": (u ** 3 * V).long().clamp(0, V - 1),
           "one": torch.full((N,), V // 2),
           "outside": torch.full((N,), -1),
           "last": torch.full((N,), V - 1),
           "spread": (torch.arange(N) * 7919) % V}[kind]
    if kind == "skewed" and N > 3:
        ids[::17] = -1
        ids[1::29] = V
        ids[2::31] = V + 12345
    rows = torch.randn(max(N, V), D, generator=g)
    return ids.to(it).to(dev), rows.to(dt).to(dev)


def grad64(ids, dout, V, scale):
    ids, d = ids.long(), dout.double()
    ok = (ids >= 0) & (ids < V)
    total = torch.zeros(V, d.shape[1], dtype=torch.float64, device=d.device)
    size, count = torch.zeros_like(total), torch.zeros(V, dtype=torch.float64, device=d.device)
    total.index_put_((ids[ok],), d[ok], accumulate=True)
    size.index_put_((ids[ok],), d[ok].abs(), accumulate=True)
    count.index_put_((ids[ok],), torch.ones_like(ids[ok], dtype=torch.float64), accumulate=True)
    return scale * total, abs(scale) * size, count[:, None]


SHAPES = [(1, 1, 1), (1, 64, 5), (2, 7, 300), (31, 16, 1), (1000, 33, 257), (4096, 64, 256),
          (4097, 130, 255), (9001, 512, 70000), (20000, 100, 1000), (33000, 8, 65536)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("it", [torch.int32, torch.int64])
@pytest.mark.parametrize("N,D,V", SHAPES)
def test_forward(cuda_device, N, D, V, dt, it):
    ids, rows = inputs(cuda_device, N, D, V, dt, it)
    table = rows[:V].contiguous()
    scale = 5.65625
    out = slim.embed_forward(ids, table, scale)
    ok = (ids >= 0) & (ids < V)
    ref = table.double()[torch.where(ok, ids, 0).long()] * scale * ok[:, None]
    if dt == torch.float32:
        assert torch.equal(out, ref.float())
    else:
        assert ((out.double() - ref).abs() <= 2.0 ** -8 * (1 + 2.0 ** -10) * ref.abs()).all()


def test_forward_keeps_the_ids_shape(cuda_device):
    ids, table = inputs(cuda_device, 24, 16, 10, torch.float32)
    out = slim.embed_forward(ids.view(2, 3, 4), table[:10].contiguous(), 2.0)
    assert out.shape == (2, 3, 4, 16)
    assert torch.equal(out.view(24, 16), slim.embed_forward(ids, table[:10].contiguous(), 2.0))
    assert slim.embed_forward(ids[:0], table[:10].contiguous()).shape == (0, 16)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["skewed", "one", "outside", "last", "spread"])
@pytest.mark.parametrize("N,D,V", SHAPES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_backward(cuda_device, N, D, V, dt, kind, accumulate):
    ids, rows = inputs(cuda_device, N, D, V, dt, kind=kind,
                       it=torch.int32 if kind == "one" else torch.int64)
    dout, scale = rows[:N].contiguous(), -1.5
    ref, size, count = grad64(ids, dout, V, scale)
    given = None
    if accumulate:
        given = torch.randn(V, D, device=cuda_device).to(dt)
        ref, size = ref + given.double(), size + given.double().abs()
        before = given.clone()
    got = slim.embed_backward(ids, dout, V, scale, dtable=given)
    assert got.dtype == dt
    bound = (count + 2) * 2.0 ** -24 * size + UNIT[dt] * (1 + 2.0 ** -10) * ref.abs()
    assert ((got.double() - ref).abs() <= bound).all()
    untouched = (count == 0).expand_as(got)
    assert torch.equal(got[untouched], before[untouched] if accumulate
                       else torch.zeros_like(got)[untouched])
    if not accumulate:
        assert torch.equal(got, slim.embed_backward(ids, dout, V, scale))  # bit for bit


def test_backward_leaves_rows_of_other_ids_finite(cuda_device):
    """Infinities and NaN in the rows of padding tokens reach no row; those of a
    token reach its own row only."""
    N, D, V = 5000, 24, 40
    ids, dout = inputs(cuda_device, N, D, V, torch.float32)
    pad = (ids < 0) | (ids >= V)
    dout = dout[:N].contiguous()
    dout[pad] = float("nan")
    dout[(ids == 3).nonzero()[0]] = float("inf")
    got = slim.embed_backward(ids, dout, V)
    rows = torch.arange(V, device=cuda_device) != 3
    assert torch.isfinite(got[rows]).all() and torch.isinf(got[3]).all()


def test_backward_against_differences(cuda_device):
    """The lookup is linear in the table: a difference quotient along a random
    direction is the inner product with the gradient, up to fp32 rounding of the
    2 N D products (each within 2^-23 of its terms' magnitudes)."""
    N, D, V, scale = 700, 48, 90, 3.25
    ids, rows = inputs(cuda_device, N, D, V, torch.float32)
    table, dout = rows[:V].contiguous(), rows[:N].flip(0).contiguous()
    step = torch.randn(V, D, device=cuda_device)
    up, down = table + step, table - step
    diff = ((slim.embed_forward(ids, up, scale).double()
             - slim.embed_forward(ids, down, scale).double()) / 2 * dout.double())
    grad = slim.embed_backward(ids, dout, V, scale).double()
    lhs, rhs = diff.sum().item(), (grad * ((up.double() - down.double()) / 2)).sum().item()
    size = (slim.embed_forward(ids, up.abs() + down.abs(), scale).double() * dout.double().abs())
    _, gsize, count = grad64(ids, dout, V, scale)
    bound = 2.0 ** -23 * size.sum().item() + \
        ((count + 3) * 2.0 ** -24 * gsize * step.double().abs()).sum().item()
    assert abs(lhs - rhs) <= bound


def test_autograd_and_another_stream(cuda_device):
    ids, rows = inputs(cuda_device, 3000, 64, 500, torch.float32)
    table = rows[:500].contiguous().requires_grad_()
    w = rows[:3000].contiguous()
    (slim.embedding(ids, table, 2.0) * w).sum().backward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = slim.embed_backward(ids, w, 500, 2.0, stream=s)
    s.synchronize()
    assert torch.equal(table.grad, other)


def test_refusals(cuda_device):
    ids, rows = inputs(cuda_device, 8, 16, 4, torch.float32)
    table = rows[:4].contiguous()
    with pytest.raises(TypeError):
        slim.embed_forward(ids.float(), table)
    with pytest.raises(TypeError):
        slim.embed_forward(ids, table.half())
    with pytest.raises(ValueError):
        slim.embed_forward(ids, table[0])
    with pytest.raises(ValueError):
        slim.embed_forward(ids, table, out=torch.empty(8, 15, device=cuda_device))
    with pytest.raises(ValueError):
        slim.embed_backward(ids, rows[:7].contiguous(), 4)
    with pytest.raises(ValueError):
        slim.embed_backward(ids, rows[:8].contiguous(), 4, dtable=torch.zeros(5, 16, device=cuda_device))
    with pytest.raises(RuntimeError):
        slim.embed_forward(ids, rows[:, ::2])
    ws = torch.empty(256, dtype=torch.uint8, device=cuda_device)
    with pytest.raises(slim.SlimError) as e:
        slim.embed_backward(ids, rows[:8].contiguous(), 4, workspace=ws)
    assert e.value.status == 3
