"""Plain forms in 64 bits of the operators around the attention, differentiable by
autograd, and the comparison helpers of their tests."""
import math

import torch

F32, BF16 = torch.float32, torch.bfloat16
# half a step relative to the value: what one rounding to the type may cost
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def rel(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm().clamp(min=1e-300))


def angles64(positions, inv_freq, B, L, device):
    """[B, 1, L, pairs] angles in radians."""
    at = torch.arange(L, device=device).expand(B, L) if positions is None else positions
    f = torch.tensor(list(inv_freq), dtype=torch.float64, device=device)
    return at[:, None, :, None].double() * f


def pairs_of(d, pairs, interleaved):
    """Indices of the first and second member of each turned pair."""
    p = torch.arange(pairs)
    return (2 * p, 2 * p + 1) if interleaved else (p, p + pairs)


def qk64(x, weight, positions, inv_freq, interleaved, eps, scale):
    """One side of qk_norm on x [B, H, L, d] in 64 bits."""
    B, _, L, d = x.shape
    y = scale * x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        y = y * weight
    if inv_freq is None or len(inv_freq) == 0:
        return y
    angle = angles64(positions, inv_freq, B, L, x.device)
    i, k = (t.to(x.device) for t in pairs_of(d, len(inv_freq), interleaved))
    a, b = y[..., i], y[..., k]
    out = y.clone()
    out[..., i] = a * angle.cos() - b * angle.sin()
    out[..., k] = a * angle.sin() + b * angle.cos()
    return out


def partner(x, pairs, interleaved):
    """|x| with each turned feature's partner added: the size that a turn's errors go by."""
    m = x.abs()
    if not pairs:
        return m
    i, k = (t.to(x.device) for t in pairs_of(x.shape[-1], pairs, interleaved))
    out = m.clone()
    out[..., i] = out[..., k] = m[..., i] + m[..., k]
    return out


def gates64(gate, kind):
    """(a, b): h_t = a_t h_(t-1) + b_t x_t."""
    if kind == "sigmoid":
        return torch.sigmoid(gate), torch.sigmoid(-gate)
    return (gate if kind == "value" else gate.exp()), torch.ones_like(gate)


def scan64(gate, x, kind, h0=None):
    a, b = gates64(gate, kind)
    h = torch.zeros_like(x[:, 0]) if h0 is None else h0
    out = []
    for t in range(x.shape[1]):
        h = a[:, t] * h + b[:, t] * x[:, t]
        out.append(h)
    return torch.stack(out, 1), h


ACTS = {
    "silu": lambda g: g * torch.sigmoid(g),
    # 1 + erf leaves no digits in the lower tail
    "gelu": lambda g: 0.5 * g * torch.erfc(-g * math.sqrt(0.5)),
    "gelu_tanh": lambda g: 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))),
    "relu": torch.relu,
    "sigmoid": torch.sigmoid,
}


def ff64(x, w, act):
    F = w.shape[0] // 2
    return ACTS[act](x @ w[:F].T) * (x @ w[F:].T)
