"""A model's layer out of the library's operators: rows are projected once; queries and
keys are normed, turned and attended to; a gated recurrence runs beside; a gated
feed-forward follows.  Its gradients against autograd on the plain formulas in 64 bits,
the same layer token by token with its states carried, and as a captured graph."""
import math

import pytest
import torch

from layer_common import BF16, F32, ff64, qk64, rel, scan64
from paper_2012_11346_gb300 import slim

pytestmark = pytest.mark.gpu

H, d, M, F, C = 2, 32, 64, 160, 32
D = H * d
FREQ = slim.rotary_frequencies(d // 2)
HOW = dict(inv_freq=FREQ, interleaved=False, eps=1e-6, scale=d ** -0.25)


def weights(dev, dt=F32, seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g) / math.sqrt(s[-1])
    p = dict(rows=n(5 * D, D), out=n(D, 2 * D), ff=n(2 * F, D), down=n(D, F))
    p = {k: v.to(dt).to(dev) for k, v in p.items()}
    p["wq"], p["wk"] = ((1 + 0.2 * torch.randn(d, generator=g)).to(dev) for _ in range(2))
    p["omega"] = torch.randn(M, d, generator=g).to(dev)
    return p


def split(x, p):
    """q, k, v [B, H, L, d] and gate, u [B, L, D], all slices of one projection's rows."""
    B, L, _ = x.shape
    rows = x @ p["rows"].T
    q, k, v = (rows[..., i * D:(i + 1) * D].view(B, L, H, d).transpose(1, 2) for i in range(3))
    return q, k, v, rows[..., 3 * D:4 * D] + 2.0, rows[..., 4 * D:]


def join(x, a, h, p, ff):
    B, L, _ = x.shape
    y = x + torch.cat([a.transpose(1, 2).reshape(B, L, D), h], -1) @ p["out"].T
    return y + ff(y) @ p["down"].T


def layer(x, p, positions, h0):
    q, k, v, gate, u = split(x, p)
    q, k = slim.qk_norm(q, k, p["wq"], p["wk"], positions, **HOW)
    a = slim.slim_attention(q, k, v.contiguous(), p["omega"], C)
    h, last = slim.gated_scan(gate, u, "sigmoid", h0)
    return join(x, a, h, p, lambda y: slim.gated_ff(y, p["ff"], "silu")), last


def layer64(x, p, positions, h0):
    q, k, v, gate, u = split(x, p)
    how = dict(positions=positions, **HOW)
    q, k = (qk64(t, w, how["positions"], FREQ, False, 1e-6, d ** -0.25) for t, w in ((q, p["wq"]), (k, p["wk"])))
    phi = lambda t: (t @ p["omega"].T - t.pow(2).sum(-1, keepdim=True) / 2).exp() / math.sqrt(M)
    A = (phi(q) @ phi(k).transpose(-1, -2)).tril()
    a = (A @ v) / A.sum(-1, keepdim=True)
    h, last = scan64(gate, u, "sigmoid", h0)
    return join(x, a, h, p, lambda y: ff64(y, p["ff"], "silu")), last


def inputs(dev, B, L, dt=F32):
    g = torch.Generator().manual_seed(L)
    x, h0 = torch.randn(B, L, D, generator=g).to(dt).to(dev), torch.randn(B, D, generator=g).to(dev)
    start = torch.randint(0, 100000, (B, 1), generator=g)
    return x, (start + torch.arange(L)).to(dev), h0


@pytest.mark.parametrize("B,L", [(2, 200), (1, 67), (3, 1)])
def test_gradients(cuda_device, B, L):
    """fp32.  The attention's gradients are held to 1e-5 of their norm, the others to less,
    and a library product of K terms to K 2^-24: the chain of five to 5e-5."""
    x, positions, h0 = inputs(cuda_device, B, L)
    p = weights(cuda_device)
    up = torch.randn(x.shape, generator=torch.Generator().manual_seed(1)).to(cuda_device)

    def run(call, cast):
        args = {n: cast(t).requires_grad_() for n, t in p.items()}
        xs, hs = cast(x).requires_grad_(), cast(h0).requires_grad_()
        y, last = call(xs, args, positions, hs)
        loss = (y * cast(up)).sum() + last.sum()
        return [y, last], torch.autograd.grad(loss, [xs, hs, *args.values()])

    was = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        got = run(layer, lambda t: t.detach().clone())
    finally:
        torch.backends.cuda.matmul.allow_tf32 = was
    want = run(layer64, lambda t: t.detach().double())
    # One token attends to itself alone: a = v, and the gradients through the features are
    # two equal terms, (da . v) (omega - q) and its like, taken from each other.  What is
    # left is their rounding: 5e-5 of their size, for which sum |up| max|v| max|omega| stands.
    alone = {"wq", "wk", "omega"} if L == 1 else set()
    v = split(x.double(), {n: t.double() for n, t in p.items()})[2]
    size = float(up.double().abs().sum() * v.abs().max() * p["omega"].double().abs().max())
    for name, a, b in zip(["y", "last", "x", "h0", *p], got[0] + list(got[1]), want[0] + list(want[1])):
        if name in alone:
            assert float(b.detach().norm()) < 1e-12 and float(a.norm()) <= 5e-5 * size
        else:
            assert rel(a.detach(), b.detach()) <= 5e-5, name


def forward(x, p, positions, h0, S=None, z=None, chunk=C, **kw):
    """Without gradients, as a serving program calls it; the carried states come back."""
    q, k, v, gate, u = split(x, p)
    q, k = slim.qk_norm_forward(q, k, p["wq"], p["wk"], positions=positions, **HOW, **kw)
    a, S, z = slim.forward(q, k, v.contiguous(), p["omega"], chunk, S_init=S, z_init=z, **kw)
    h, last = slim.gated_scan_forward(gate, u, "sigmoid", h0=h0, **kw)
    return join(x, a, h, p, lambda y: slim.gated_ff_forward(y, p["ff"], "silu", **kw)), last, S, z


@pytest.mark.parametrize("dt,tol", [(F32, 2e-5), (BF16, 2e-2)])
def test_token_by_token(cuda_device, dt, tol):
    """A prompt in one call and tokens one a call, states carried, is the sequence in one
    call: within the roundings of another order in fp32, and in bf16 of the eight tensors
    between the operators, half a step (2^-8) each."""
    x, positions, h0 = inputs(cuda_device, 2, 100, dt)
    p = weights(cuda_device, dt)
    whole, last, *_ = forward(x, p, positions, h0)
    at = 80
    y, s, S, z = forward(x[:, :at], p, positions[:, :at].contiguous(), h0)
    parts = [y]
    for t in range(at, 100):
        y, s, S, z = forward(x[:, t:t + 1], p, positions[:, t:t + 1].contiguous(), s, S, z, chunk=1)
        parts.append(y)
    assert rel(torch.cat(parts, 1), whole) <= tol and rel(s, last) <= tol


def test_captured(cuda_device):
    """The layer as one graph, replayed on new inputs, gives the eager call's bits; two
    graphs of it at once, each with the memory it was captured with."""
    p = weights(cuda_device, BF16)
    sets = [inputs(cuda_device, 2, L, BF16) for L in (1500, 300)]
    graphs, outs = [], []
    for x, positions, h0 in sets:
        forward(x, p, positions, h0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(forward(x, p, positions, h0))
        graphs.append(graph)
    for x, _, h0 in sets:
        x.copy_(x.flip(1))
        h0.neg_()
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for stream, graph in zip(streams, graphs):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    for (x, positions, h0), got in zip(sets, outs):
        assert all(torch.equal(a, b) for a, b in zip(got, forward(x, p, positions, h0)))
