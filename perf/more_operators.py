"""Cases and plain forms of the operators of a language model's layer around the
sliced attention: what turns a projection's rows into its queries and keys, the
gated recurrence that mixes tokens beside it, and the gated feed-forward behind it.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU, `run`
makes one pass through an operator (the framework's with `own`, elementary torch
operations in 32 bits without), `exact` is the same from the definition in 64
bits, and `work` counts the bytes and operations a pass cannot do without.

  qk_norm  q [B, Hq, L, d], k [B, Hk, L, d]: per token and head
           y = scale * x / sqrt(mean(x^2) + eps) * weight, then its pairs of
           features turned by position * frequency; "backward" is the gradient
           with respect to q, k and the two weights.
  scan     gate, x [B, L, D]: h_t = a_t h_(t-1) + u_t per channel, with a = gate,
           u = x ("value"); a = exp(gate), u = x ("log"); or a = sigmoid(gate),
           u = (1 - a) x ("sigmoid").  "forward" returns h and the last state,
           "step" also the gradients.
  ff       x [N, D], w [2F, D]: h = act(x w_gate^T) * (x w_up^T), w_gate the first
           F rows of w and w_up the others; "step" also returns dx and dw.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # one decoding step of 8 requests, each at its own place of a long text: latency
        dict(name="qk_decode", op="qk_norm", B=8, L=1, Hq=8, Hk=8, d=64, rotary=64, interleaved=False, positions="far",
             dtype="bf16", pass_="forward"),
        # a training batch of 8 sequences of 4096 tokens, 8 heads of 64
        dict(name="qk_train", op="qk_norm", B=8, L=4096, Hq=8, Hk=8, d=64, rotary=64, interleaved=False, positions="none",
             dtype="bf16", pass_="forward"),
        # its gradient at 12 heads in fp32, documents packed into each sequence
        dict(name="qk_grad_f32", op="qk_norm", B=4, L=8192, Hq=12, Hk=12, d=64, rotary=64, interleaved=False,
             positions="packed", dtype="f32", pass_="backward"),
        # odd lengths, key heads shared by query heads, a width of whole pairs only, half of it turned
        dict(name="qk_grad_odd", op="qk_norm", B=3, L=1021, Hq=6, Hk=2, d=36, rotary=18, interleaved=True, positions="packed",
             dtype="bf16", pass_="backward"),
        # one decoding step of 8 requests
        dict(name="scan_decode", op="scan", B=8, L=1, D=512, kind="sigmoid", dtype="bf16", pass_="forward"),
        # one sequence of 65536 tokens read once
        dict(name="scan_long", op="scan", B=1, L=65536, D=512, kind="log", dtype="f32", pass_="forward"),
        # a training step on 8 sequences of 4096 tokens
        dict(name="scan_train", op="scan", B=8, L=4096, D=512, kind="sigmoid", dtype="bf16", pass_="step"),
        # odd lengths and channels, documents packed into each sequence
        dict(name="scan_odd", op="scan", B=3, L=1021, D=201, kind="value", dtype="f32", pass_="step"),
        # one decoding step of 4 requests
        dict(name="ff_decode", op="ff", N=4, D=512, F=2048, act="silu", dtype="bf16", pass_="forward"),
        # scoring 16 k tokens at 12 heads of 64
        dict(name="ff_eval", op="ff", N=16384, D=768, F=2048, act="gelu_tanh", dtype="bf16", pass_="forward"),
        # a small fp32 model, odd everything
        dict(name="ff_odd_f32", op="ff", N=1021, D=200, F=533, act="gelu", dtype="f32", pass_="step"),
        # a training step on 8 sequences of 4096 tokens, 8 heads of 64
        dict(name="ff_train", op="ff", N=32768, D=512, F=2048, act="silu", dtype="bf16", pass_="step"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return min(max(int(round(math.exp(rng.uniform(math.log(low), math.log(high))))), low), high)


def draw(rng):
    op = rng.choice(("qk_norm", "scan", "ff"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "qk_norm":
        while True:
            Hk = _spread(rng, 1, 12)
            d = rng.choice((16, 32, 64, 64, 128, 2 * _spread(rng, 4, 128)))
            case = dict(op=op, B=_spread(rng, 1, 16), L=_spread(rng, 1, 65536), Hq=Hk * rng.choice((1, 1, 2, 3)), Hk=Hk, d=d,
                        rotary=rng.choice((d, d, d // 4 * 2, 0)), interleaved=rng.random() < 0.4,
                        positions=rng.choice(("none", "packed", "far")), dtype=dtype,
                        pass_=rng.choice(("forward", "backward")))
            if case["B"] * case["L"] * (case["Hq"] + Hk) * d <= 4 * 8192 * 24 * 64:
                return case
    if op == "scan":
        while True:
            D = _spread(rng, 16, 4096)
            case = dict(op=op, B=_spread(rng, 1, 32), L=_spread(rng, 1, 65536), D=D if rng.random() < 0.5 else max(16, D // 64 * 64),
                        kind=rng.choice(("value", "log", "sigmoid")), dtype=dtype, pass_=rng.choice(("forward", "step", "step")))
            if case["B"] * case["L"] * D <= 65536 * 512:
                return case
    while True:
        D, F = _spread(rng, 32, 2048), _spread(rng, 64, 8192)
        if rng.random() < 0.6:  # most widths are whole heads
            D, F = max(64, D // 64 * 64), max(64, F // 64 * 64)
        case = dict(op=op, N=_spread(rng, 1, 65536), D=D, F=F, act=rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu", "sigmoid")),
                    dtype=dtype, pass_=rng.choice(("forward", "step", "step")))
        limit = 12.0 * 32768 * 512 * 2048 * (1.0 if dtype == "bf16" else 0.2)
        if work(case)["flops"] <= limit and case["N"] * F <= 32768 * 4096:
            return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    dt = DTYPE[case["dtype"]]
    if case["op"] == "qk_norm":
        B, L, Hq, Hk, d = (case[n] for n in ("B", "L", "Hq", "Hk", "d"))

        def heads(H):
            # values of one size per head, one token in sixty padded with zeros
            return (normal(B, L, H, d) * (0.2 + 3.0 * uniform(H, 1)) * (uniform(B, L, 1, 1) > 1.0 / 60.0)).to(dt)

        # queries, keys and values lie side by side in the rows of one projection
        rows = torch.cat([heads(Hq), heads(Hk), heads(Hk)], dim=2)
        state = dict(case=case, q=rows[:, :, :Hq].transpose(1, 2), k=rows[:, :, Hq:Hq + Hk].transpose(1, 2),
                     wq=1.0 + 0.2 * normal(d), wk=1.0 + 0.2 * normal(d), scale=d ** -0.25, positions=None, inv_freq=None)
        if case["positions"] == "packed":
            # documents of a few hundred tokens follow each other, each counted from 0
            at = torch.arange(L, device="cuda").expand(B, L)
            start = torch.where(uniform(B, L) < 1.0 / 300.0, at, 0).cummax(dim=1).values
            state["positions"] = (at - start).int()
        elif case["positions"] == "far":
            state["positions"] = (uniform(B, 1) * 131072).long() + torch.arange(L, device="cuda")
        if case["rotary"]:
            state["inv_freq"] = _frequencies(case["rotary"])
        if case["pass_"] == "backward":
            state["dq"], state["dk"] = normal(B, Hq, L, d).to(dt), normal(B, Hk, L, d).to(dt)
        return state
    if case["op"] == "scan":
        B, L, D = case["B"], case["L"], case["D"]
        # memories from a few tokens to some hundreds; a document ends every 500 tokens or so
        gate, border = 1.5 * normal(B, L, D) + 2.0 + 2.0 * uniform(D), (uniform(B, L, 1) < 1.0 / 500.0)
        if case["kind"] == "value":
            gate = torch.where(border, 0.0, torch.sigmoid(gate))
        elif case["kind"] == "log":
            gate = torch.where(border, -math.inf, -torch.nn.functional.softplus(-gate))
        state = dict(case=case, gate=gate.to(dt), x=normal(B, L, D).to(dt), h0=normal(B, D))
        if case["pass_"] == "step":
            state["dh"], state["dlast"] = normal(B, L, D).to(dt), normal(B, D)
        return state
    N, D, F = case["N"], case["D"], case["F"]
    state = dict(case=case, x=(normal(N, D) * (0.5 + uniform(N, 1))).to(dt), w=(normal(2 * F, D) / math.sqrt(D)).to(dt))
    if case["pass_"] == "step":
        state["dh"] = normal(N, F).to(dt)
    return state


def _frequencies(rotary):
    """Radians per position of each pair, as the usual powers of 10000."""
    import array
    return array.array("d", [10000.0 ** (-2.0 * i / rotary) for i in range(rotary // 2)])


# ---------------------------------------------------------------- plain forms, 32 bits
def _turn(y, cos, sin, interleaved):
    """Turns the pairs of the first 2 * cos.shape[-1] features of y [B, H, L, d]."""
    half = cos.shape[-1]
    a, b, rest = (y[..., 0:2 * half:2], y[..., 1:2 * half:2], y[..., 2 * half:]) if interleaved else \
        (y[..., :half], y[..., half:2 * half], y[..., 2 * half:])
    c, s = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([c, s], dim=-1).flatten(-2) if interleaved else torch.cat([c, s], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _plain_angles(state):
    case = state["case"]
    if state["inv_freq"] is None:
        return None
    at = state["positions"]
    if at is None:
        at = torch.arange(case["L"], device="cuda")[None]
    # positions times frequencies lose their fraction of a turn in 32 bits
    angle = at[:, None, :, None].double() * torch.tensor(state["inv_freq"], dtype=torch.float64, device="cuda")
    return angle.cos().float(), angle.sin().float()


def _plain_qk(state):
    case, turns = state["case"], _plain_angles(state)
    out = {}
    for name, weight in (("q", state["wq"]), ("k", state["wk"])):
        x = state[name].float()
        r = (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
        if case["pass_"] == "forward":
            y = x * r * (weight * state["scale"])
            out[name] = (_turn(y, *turns, case["interleaved"]) if turns else y).to(state[name].dtype)
            continue
        dy = state["d" + name].float()
        if turns:  # a turn's gradient is the turn back
            dy = _turn(dy, turns[0], -turns[1], case["interleaved"])
        dy = dy * state["scale"]
        n = x * r
        g = dy * weight
        out["d" + name] = (r * (g - n * (g * n).mean(dim=-1, keepdim=True))).to(state[name].dtype)
        out["dw" + name] = (dy * n).sum(dim=(0, 1, 2))
    return out


def _doubling(a, u):
    """All h_t = a_t h_(t-1) + u_t along dim 1 from h = 0, in log2(L) rounds."""
    a, h, step = a.clone(), u.clone(), 1
    while step < h.shape[1]:
        h[:, step:] += a[:, step:] * h[:, :-step].clone()
        a[:, step:] *= a[:, :-step].clone()
        step *= 2
    return h


def _plain_scan(state):
    case = state["case"]
    gate, x, h0 = state["gate"].float(), state["x"].float(), state["h0"]
    a = {"value": lambda: gate, "log": gate.exp, "sigmoid": gate.sigmoid}[case["kind"]]()
    keep = (-gate).sigmoid() if case["kind"] == "sigmoid" else None
    u = x if keep is None else keep * x
    u = torch.cat([u[:, :1] + a[:, :1] * h0[:, None], u[:, 1:]], dim=1)
    h = _doubling(a, u)
    out = {"h": h.to(state["x"].dtype), "last": h[:, -1]}
    if case["pass_"] == "step":
        up = state["dh"].float()
        up = torch.cat([up[:, :-1], up[:, -1:] + state["dlast"][:, None]], dim=1)
        back = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)  # h_t reaches h_(t+1) by a_(t+1)
        g = _doubling(back.flip(1), up.flip(1)).flip(1)
        before = torch.cat([h0[:, None], h[:, :-1]], dim=1)
        if case["kind"] == "sigmoid":
            dgate, dx = g * (before - x) * a * keep, g * keep
        else:
            dgate, dx = g * before * (1.0 if case["kind"] == "value" else a), g
        out.update(dgate=dgate.to(state["gate"].dtype), dx=dx.to(state["x"].dtype), dh0=a[:, 0] * g[:, 0])
    return out


def _plain_act(act, g):
    """act(g) and its derivative."""
    if act == "relu":
        return g.clamp(min=0.0), (g > 0).float()
    if act in ("silu", "sigmoid"):
        s = g.sigmoid()
        return (s, s * (1.0 - s)) if act == "sigmoid" else (g * s, s * (1.0 + g * (1.0 - s)))
    if act == "gelu":
        c = 0.5 * (1.0 + (g * math.sqrt(0.5)).erf())
        return g * c, c + g * (-0.5 * g * g).exp() * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    t = (k * (g + 0.044715 * g * g * g)).tanh()
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * g * g)


def _plain_ff(state):
    case, F = state["case"], state["case"]["F"]
    x, w = state["x"].float(), state["w"].float()
    z = x @ w.T
    a, da = _plain_act(case["act"], z[:, :F])
    out = {"h": (a * z[:, F:]).to(state["x"].dtype)}
    if case["pass_"] == "step":
        dh = state["dh"].float()
        dz = torch.cat([dh * z[:, F:] * da, dh * a], dim=1)
        out["dx"], out["dw"] = (dz @ w).to(state["x"].dtype), (dz.T @ x).to(state["w"].dtype)
    return out


# ---------------------------------------------------------------- the framework's
def _own(state):
    from paper_2012_11346_gb300 import slim

    case = state["case"]
    if case["op"] == "qk_norm":
        how = dict(positions=state["positions"], inv_freq=state["inv_freq"], interleaved=case["interleaved"], eps=EPS,
                   scale=state["scale"])
        if case["pass_"] == "forward":
            q, k = slim.qk_norm_forward(state["q"], state["k"], state["wq"], state["wk"], **how)
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = slim.qk_norm_backward(state["q"], state["k"], state["wq"], state["wk"], state["dq"], state["dk"], **how)
        return {"dq": dq, "dwq": dwq, "dk": dk, "dwk": dwk}
    if case["op"] == "scan":
        step = case["pass_"] == "step"
        # a step keeps the states between pieces of the sequence, from which the backward starts its own again
        h, last, *kept = slim.gated_scan_forward(state["gate"], state["x"], case["kind"], h0=state["h0"], keep=step)
        out = {"h": h, "last": last}
        if step:
            dgate, dx, dh0 = slim.gated_scan_backward(state["gate"], state["x"], kept[0], state["dh"], case["kind"],
                                                      dlast=state["dlast"])
            out.update(dgate=dgate, dx=dx, dh0=dh0)
        return out
    if case["pass_"] == "forward":
        return {"h": slim.gated_ff_forward(state["x"], state["w"], case["act"])}
    # a step with memory for both projections keeps them for the backward
    h, z = slim.gated_ff_forward(state["x"], state["w"], case["act"], keep=True)
    dx, dw = slim.gated_ff_backward(state["x"], state["w"], state["dh"], case["act"], z=z)
    return {"h": h, "dx": dx, "dw": dw}


def run(state):
    if own:
        return _own(state)
    return {"qk_norm": _plain_qk, "scan": _plain_scan, "ff": _plain_ff}[state["case"]["op"]](state)


def work(case):
    es, step = SIZE[case["dtype"]], case["pass_"] != "forward"
    if case["op"] == "qk_norm":
        # rows read and written once; the gradient also reads what comes from above
        n = case["B"] * case["L"] * (case["Hq"] + case["Hk"]) * case["d"]
        at = {"none": 0, "packed": 4, "far": 8}[case["positions"]] * case["B"] * case["L"]
        return {"bytes": (3 if step else 2) * n * es + at, "flops": (20 if step else 8) * n}
    if case["op"] == "scan":
        # gate and x read, h written; a step also reads the gradient of h and writes those of gate and x
        n, ends = case["B"] * case["L"] * case["D"], case["B"] * case["D"]
        return {"bytes": (6 if step else 3) * n * es + (16 if step else 8) * ends, "flops": (14 if step else 4) * n}
    N, D, F = case["N"], case["D"], case["F"]
    # x and w read, h written; a step reads the gradient of h and writes those of x and w
    once = (N * D + 2 * F * D + N * F) * es
    return {"bytes": 2 * once if step else once, "flops": (12 if step else 4) * N * D * F}


# ---------------------------------------------------------------- from the definitions, 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"qk_norm": _exact_qk, "scan": _exact_scan, "ff": _exact_ff}[case["op"]](case, state)


def _exact_qk(case, s):
    """The turn as a product of complex numbers, the norm's gradient as a projection."""
    d, half = case["d"], case["rotary"] // 2
    order = list(range(d))  # the features of pair p at places 2p and 2p + 1
    if half and not case["interleaved"]:
        order = [i for p in range(half) for i in (p, p + half)] + list(range(2 * half, d))
    back = torch.tensor(order, device="cuda").argsort()
    unit = None
    if half:
        at = s["positions"] if s["positions"] is not None else torch.arange(case["L"], device="cuda").unsqueeze(0)
        turn = torch.einsum("bl,f->blf", at.double(), torch.tensor(list(s["inv_freq"]), device="cuda", dtype=torch.float64))
        unit = torch.polar(torch.ones_like(turn), turn).unsqueeze(1)

    def rotate(y, u):
        if u is None:
            return y
        z = torch.view_as_complex(y[..., order][..., :2 * half].reshape(*y.shape[:-1], half, 2).contiguous()) * u
        return torch.cat([torch.view_as_real(z).reshape(*y.shape[:-1], 2 * half), y[..., order][..., 2 * half:]], -1)[..., back]

    out = {}
    for n in ("q", "k"):
        x, w = s[n].double(), s["w" + n].double()
        size = torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS)
        if case["pass_"] == "forward":
            out[n] = rotate(s["scale"] * w * x / size, unit)
        else:
            dy = s["scale"] * rotate(s["d" + n].double(), None if unit is None else unit.conj())
            g = w * dy
            out["d" + n] = g / size - x * (g * x).sum(-1, keepdim=True) / (d * size ** 3)
            out["dw" + n] = torch.einsum("bhld,bhld->d", dy, x / size)
    return out


def _exact_scan(case, s):
    """One token after the other."""
    L, kind, step = case["L"], case["kind"], case["pass_"] == "step"
    gate, x = s["gate"].double().transpose(0, 1).contiguous(), s["x"].double().transpose(0, 1).contiguous()
    if kind == "sigmoid":
        a, b = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    else:
        a, b = (gate if kind == "value" else torch.exp(gate)), torch.ones_like(gate)
    h = torch.empty(L + 1, *gate.shape[1:], dtype=torch.float64, device="cuda")
    h[0] = s["h0"].double()
    u = b * x
    for t in range(L):
        torch.addcmul(u[t], a[t], h[t], out=h[t + 1])
    out = {"h": h[1:].transpose(0, 1), "last": h[L]}
    if step:
        g = s["dh"].double().transpose(0, 1).contiguous()
        g[L - 1] += s["dlast"].double()
        for t in range(L - 2, -1, -1):
            g[t].addcmul_(a[t + 1], g[t + 1])
        if kind == "sigmoid":
            dgate = g * (h[:L] - x) * a * b
        else:
            dgate = g * h[:L] if kind == "value" else g * h[:L] * a
        out.update(dgate=dgate.transpose(0, 1), dx=(g * b).transpose(0, 1), dh0=g[0] * a[0])
    return out


def _exact_ff(case, s):
    """Rows in pieces, the activation's derivative from autograd."""
    from torch.nn import functional as nf
    x, w, step = s["x"].double(), s["w"].double(), case["pass_"] == "step"
    wg, wu = w.chunk(2)
    acts = {"silu": nf.silu, "gelu": nf.gelu, "gelu_tanh": lambda v: nf.gelu(v, approximate="tanh"), "relu": nf.relu,
            "sigmoid": torch.sigmoid}
    h, dx, dw = [], [], torch.zeros_like(w)
    for a in range(0, case["N"], 8192):
        rows = x[a:a + 8192]
        gate, up = torch.einsum("nd,fd->nf", rows, wg), torch.einsum("nd,fd->nf", rows, wu)
        with torch.enable_grad():
            gate, up = gate.detach().requires_grad_(), up.detach().requires_grad_()
            out = acts[case["act"]](gate) * up
        h.append(out.detach())
        if step:
            dg, du = torch.autograd.grad(out, (gate, up), s["dh"][a:a + 8192].double())
            dx.append(torch.einsum("nf,fd->nd", dg, wg) + torch.einsum("nf,fd->nd", du, wu))
            dw += torch.cat([torch.einsum("nf,nd->fd", dg, rows), torch.einsum("nf,nd->fd", du, rows)])
    out = {"h": torch.cat(h)}
    return {**out, "dx": torch.cat(dx), "dw": dw} if step else out
