"""The differentiable calls give first derivatives.  Differentiating their
gradients again has to be an error: the library's kernels leave no graph behind,
and terms that silently went missing would be a wrong answer.  The kernels are
replaced by plain formulas here, so that this runs without a GPU."""
import pytest
import torch

from paper_2012_11346_gb300 import slim


@pytest.fixture
def on_cpu(monkeypatch):
    def loss_forward(x, w, targets, ignore_index=-100):
        z = x.reshape(-1, w.shape[1]).double() @ w.double().T
        lse = torch.logsumexp(z, 1)
        loss = lse - z.gather(1, targets.reshape(-1, 1))[:, 0]
        return (loss.float().reshape(targets.shape), lse.float().reshape(targets.shape),
                torch.stack([loss.sum(), torch.tensor(float(len(loss)))]).float())

    def loss_backward(x, w, targets, lse, dloss, count=None, ignore_index=-100, piece=None):
        with torch.no_grad():
            a = x.reshape(-1, w.shape[1])
            g = (a @ w.T - lse.reshape(-1, 1)).exp()
            g = g.scatter_add(1, targets.reshape(-1, 1), -torch.ones(len(a), 1))
            g = g * dloss.reshape(-1, 1) / (1.0 if count is None else count)
            return (g @ w).reshape(x.shape), g.T @ a

    def embed_forward(ids, table, scale=1.0):
        return (scale * table[ids]).detach()

    def embed_backward(ids, dout, V, scale=1.0):
        with torch.no_grad():
            return torch.zeros(V, dout.shape[-1]).index_add_(0, ids, scale * dout)

    monkeypatch.setattr(slim, "vocab_loss_forward", loss_forward)
    monkeypatch.setattr(slim, "vocab_loss_backward", loss_backward)
    monkeypatch.setattr(slim, "embed_forward", embed_forward)
    monkeypatch.setattr(slim, "embed_backward", embed_backward)


def leaf(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).requires_grad_()


REFUSAL = "once"


def loss_of(x, w, kind):
    t = torch.arange(6) % 5
    if kind == "transposed":  # operands that the call copies
        x = x.t().contiguous().t()
    out = slim.vocab_loss(x, w, t, reduction="none" if kind == "none" else "mean")
    return out.sum() if kind == "none" else out


@pytest.mark.parametrize("kind", ["mean", "none", "transposed"])
def test_vocab_loss_refuses_second_derivatives(on_cpu, kind):
    x, w = leaf(6, 4), leaf(5, 4, seed=1)
    y = loss_of(x, w, kind)
    dx, dw = torch.autograd.grad(y, (x, w), create_graph=True)
    for g in (dx, dw):
        with pytest.raises(RuntimeError, match=REFUSAL):
            torch.autograd.grad(g.pow(2).sum() + x.pow(3).sum() + w.pow(3).sum(), (x, w),
                                retain_graph=True)
    with pytest.raises(RuntimeError, match=REFUSAL):
        dx.sum().backward()


def test_vocab_loss_refuses_the_derivative_by_its_upstream(on_cpu):
    x, w, c = leaf(6, 4), leaf(5, 4, seed=1), leaf(6, seed=2)
    y = slim.vocab_loss(x.detach(), w, torch.arange(6) % 5, reduction="none")
    (dw,) = torch.autograd.grad((y * c).sum(), w, create_graph=True)
    with pytest.raises(RuntimeError, match=REFUSAL):
        torch.autograd.grad(dw.sum() + c.sum(), c)


def test_embedding_refuses_second_derivatives(on_cpu):
    table, c = leaf(5, 4), leaf(6, 4, seed=1)
    ids = torch.tensor([0, 1, 1, 4, 2, 0])
    (d,) = torch.autograd.grad((slim.embedding(ids, table, 2.0) * c).sum(), table, create_graph=True)
    with pytest.raises(RuntimeError, match=REFUSAL):
        torch.autograd.grad(d.pow(2).sum() + c.pow(2).sum(), c)


def test_first_derivatives_are_as_before(on_cpu):
    x, w, u = leaf(6, 4), leaf(5, 4, seed=1), leaf(3, seed=2)
    t = torch.arange(6) % 5
    want = torch.autograd.grad(torch.nn.functional.cross_entropy(x @ w.T, t), (x, w))
    got = torch.autograd.grad(slim.vocab_loss(x, w, t), (x, w))
    kept = torch.autograd.grad(slim.vocab_loss(x, w, t), (x, w), create_graph=True)
    for a, b, c in zip(want, got, kept):
        assert torch.allclose(a, b, atol=1e-6) and torch.equal(b, c.detach())
        assert not b.requires_grad
    # a transposed operand is copied: what it becomes afterwards does not matter
    v = w.detach().t().contiguous()
    y = slim.vocab_loss(x, v.t(), t)
    v.zero_()
    assert torch.equal(torch.autograd.grad(y, x)[0], got[0])
    # a graph of other terms of the same step stays usable
    y = slim.vocab_loss(x, w, t) + u.pow(3).sum()
    dx, du = torch.autograd.grad(y, (x, u), create_graph=True)
    (ddu,) = torch.autograd.grad(du.sum(), u)
    assert torch.allclose(ddu, 6 * u)


def test_attention_refuses_second_derivatives(monkeypatch):
    """slim_attention's kernels, stood in for by out = q omega_00."""
    def forward(q, k, v, omega, C, feature, residuals):
        return ((q * omega[0, 0]).detach(),) + tuple(torch.zeros(1) for _ in range(4))

    def backward(q, k, v, omega, out, dout, S, z, C, feature, S_lo, z_lo):
        with torch.no_grad():
            return dout * omega[0, 0], torch.zeros_like(k), torch.zeros_like(v), \
                torch.zeros_like(omega).index_put_((torch.tensor(0), torch.tensor(0)), (dout * q).sum())

    monkeypatch.setattr(slim, "forward", forward)
    monkeypatch.setattr(slim, "backward", backward)
    q, omega = leaf(1, 1, 4, 2), leaf(3, 2, seed=1)
    y = slim.slim_attention(q, q.detach(), q.detach(), omega, 2)
    plain = torch.autograd.grad(y.pow(2).sum(), q, retain_graph=True)[0]
    assert torch.allclose(plain, 2 * q * omega[0, 0] ** 2) and not plain.requires_grad
    (dq,) = torch.autograd.grad(y.pow(2).sum(), q, create_graph=True)
    assert torch.equal(dq.detach(), plain)
    with pytest.raises(RuntimeError, match=REFUSAL):
        torch.autograd.grad(dq.sum() + q.sum() + omega.sum(), (q, omega))
