"""Cases and plain forms of the language-model operators around the attention:
the embedding lookup at a model's input, the vocabulary loss at its output, and
the clipping of its gradients by their global norm.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU, `run`
makes one pass through an operator (the framework's with `own`, elementary torch
operations in 32 bits without), `exact` is the same from the definition in 64
bits, and `work` counts the bytes and operations a pass cannot do without.

  vocab_loss  x [N, D], w [V, D], targets [N]: per row i with a target,
              loss_i = log(sum_v exp(x_i.w_v)) - x_i.w_target; "forward" returns
              the rows' losses and log-sums, "step" also the gradients of the
              mean loss (or of a weighted sum) with respect to x and w.
  embed       ids [N], table [V, D]: out_i = scale * table[ids_i], zero where the
              id lies outside the table (padding); "backward" is the gradient
              with respect to the table.
  clip        a list of gradients: their global 2-norm, and the gradients scaled
              by min(1, max_norm / norm) into a second list.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
IGNORE = -100
VOCAB_SIZES = (64, 65536)


def listed():
    return [
        # one drafted token scored against a word-piece vocabulary: latency
        dict(name="loss_one_row", op="vocab_loss", N=1, D=512, V=32768, dtype="bf16", pass_="forward", weights="mean"),
        # perplexity of 16 k tokens, odd vocabulary
        dict(name="loss_eval", op="vocab_loss", N=16384, D=512, V=50021, dtype="bf16", pass_="forward", weights="mean"),
        # a byte model in fp32 with a 257th symbol and an odd width: small, ragged
        dict(name="loss_bytes_f32", op="vocab_loss", N=1021, D=200, V=257, dtype="f32", pass_="step", weights="rows"),
        # a training step on a word vocabulary, odd batch
        dict(name="loss_words", op="vocab_loss", N=4093, D=512, V=10001, dtype="bf16", pass_="step", weights="mean"),
        # the same in fp32 at 12 heads of 64
        dict(name="loss_words_f32", op="vocab_loss", N=8192, D=768, V=10000, dtype="f32", pass_="step", weights="mean"),
        # a training step at 8 sequences of 4096 tokens, 8 heads of 64
        dict(name="loss_large", op="vocab_loss", N=32768, D=512, V=32768, dtype="bf16", pass_="step", weights="mean"),
        # the input side of one decoding step of 8 requests
        dict(name="embed_decode", op="embed", N=8, D=512, V=32768, dtype="bf16", pass_="forward"),
        # the input side of a training step, fp32 rows
        dict(name="embed_train", op="embed", N=65536, D=768, V=50021, dtype="f32", pass_="forward"),
        # the table's gradient of a byte model: few rows, each hit by many tokens
        dict(name="embed_grad_bytes", op="embed", N=32768, D=512, V=256, dtype="bf16", pass_="backward"),
        # the table's gradient on a large vocabulary: many rows hit by none
        dict(name="embed_grad_words", op="embed", N=65536, D=768, V=32768, dtype="f32", pass_="backward"),
        # a small model's 26 gradients, odd sizes, both types, clipped
        dict(name="clip_small", op="clip", tensors=26, largest=200003, dtype="both", clipped=True),
        # a model's 60 gradients in fp32, clipped
        dict(name="clip_large", op="clip", tensors=60, largest=16777216, dtype="f32", clipped=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return 3073 if n == 3072 else min(max(n, low), high)


def draw(rng):
    op = rng.choice(("vocab_loss", "vocab_loss", "embed", "clip"))
    if op == "vocab_loss":
        while True:
            case = dict(op=op, N=_spread(rng, 1, 65536), D=_spread(rng, 32, 2048), V=_spread(rng, *VOCAB_SIZES),
                        dtype=rng.choice(("bf16", "bf16", "f32")), pass_=rng.choice(("forward", "step", "step")),
                        weights=rng.choice(("mean", "rows")))
            if rng.random() < 0.6:  # most widths are whole heads
                case["D"] = max(32, case["D"] // 64 * 64)
            limit = 6.0 * 32768 * 512 * 32768 * (1.0 if case["dtype"] == "bf16" else 0.2)
            if work(case)["flops"] <= limit and case["N"] * case["V"] <= 32768 * 32768:
                return case
    if op == "embed":
        return dict(op=op, N=_spread(rng, 1, 131072), D=_spread(rng, 16, 1024), V=_spread(rng, *VOCAB_SIZES),
                    dtype=rng.choice(("bf16", "f32")), pass_=rng.choice(("forward", "backward", "backward")))
    return dict(op=op, tensors=_spread(rng, 2, 60), largest=_spread(rng, 1000, 16777216),
                dtype=rng.choice(("bf16", "f32", "both")), clipped=rng.random() < 0.75)


def _clip_sizes(case):
    """The gradients' sizes: a model's mix of matrices, their halves and quarters, and short vectors."""
    big = case["largest"]
    mix = (big, big // 4 + 1, 511, big // 2, big // 4, 64 + big % 97, 1, big // 8 + 3)
    return [max(1, mix[i % len(mix)]) for i in range(case["tensors"])]


def _clip_dtypes(case):
    return [case["dtype"] if case["dtype"] != "both" else ("bf16", "f32")[i % 3 == 0] for i in range(case["tensors"])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["op"] == "vocab_loss":
        N, D, V = case["N"], case["D"], case["V"]
        w = normal(V, D) / math.sqrt(D)
        # tokens fall off with their rank; one row in twelve carries no target
        targets = (uniform(N) ** 3 * V).long().clamp_(0, V - 1)
        # rows lean towards their target by different amounts, as in a model part way through training
        x = 2.0 * normal(N, D) + 9.0 * uniform(N, 1) * w[targets]
        targets[uniform(N) < (1.0 / 12.0 if N > 1 else -1.0)] = IGNORE
        dloss = torch.ones(1, device="cuda") if case["weights"] == "mean" else 0.5 + uniform(N)
        dt = DTYPE[case["dtype"]]
        return dict(case=case, x=x.to(dt), w=w.to(dt), targets=targets, dloss=dloss)
    if case["op"] == "embed":
        N, D, V = case["N"], case["D"], case["V"]
        ids = (uniform(N) ** 3 * V).long().clamp_(0, V - 1)
        ids[uniform(N) < 0.03] = -1
        rows = normal(V, D) if case["pass_"] == "forward" else normal(N, D)
        return dict(case=case, ids=ids, rows=rows.to(DTYPE[case["dtype"]]), scale=math.sqrt(D))
    # every fifth gradient starts one element into its buffer, as a slice of a larger one does
    grads = [(normal(n + 1) * 0.02).to(DTYPE[t])[i % 5 == 4:][:n]
             for i, (n, t) in enumerate(zip(_clip_sizes(case), _clip_dtypes(case)))]
    norm = 0.02 * math.sqrt(sum(_clip_sizes(case)))
    return dict(case=case, grads=grads, out=[torch.empty_like(g) for g in grads],
                max_norm=norm * (0.25 if case["clipped"] else 4.0))


def _loss_parts(x, w, targets):
    """Logits, whether a row has a target, that target (0 where none), the rows' log-sums and losses, in the type of x."""
    logits = x @ w.T
    has = targets != IGNORE
    at = torch.where(has, targets, 0)[:, None]
    top = logits.amax(dim=1, keepdim=True)
    lse = top + (logits - top).exp().sum(dim=1, keepdim=True).log()
    loss = torch.where(has, (lse - logits.gather(1, at))[:, 0], 0.0)
    return logits, has, at, lse, loss


def _loss_grads(logits, has, at, lse, coef, x, w):
    p = (logits - lse).exp()
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p *= torch.where(has, coef, 0.0)[:, None]
    return p @ w, p.T @ x


def _plain(state):
    case = state["case"]
    if case["op"] == "vocab_loss":
        x, w, targets = state["x"].float(), state["w"].float(), state["targets"]
        logits, has, at, lse, loss = _loss_parts(x, w, targets)
        out = {"loss": loss, "lse": lse[:, 0], "total": torch.stack([loss.sum(), has.sum().float()])}
        if case["pass_"] == "step":
            coef = state["dloss"] / out["total"][1] if case["weights"] == "mean" else state["dloss"]
            dx, dw = _loss_grads(logits, has, at, lse, coef, x, w)
            out["dx"], out["dw"] = dx.to(state["x"].dtype), dw.to(state["w"].dtype)
        return out
    if case["op"] == "embed":
        ids, rows = state["ids"], state["rows"]
        inside = (ids >= 0) & (ids < case["V"])
        at = torch.where(inside, ids, 0)
        if case["pass_"] == "forward":
            return (rows[at].float() * (inside * state["scale"])[:, None]).to(rows.dtype)
        total = torch.zeros(case["V"], case["D"], device=rows.device)
        total.index_add_(0, at, rows.float() * (inside * state["scale"])[:, None])
        return total.to(rows.dtype)
    norm = torch.stack([g.float().square().sum() for g in state["grads"]]).sum().sqrt()
    coef = (state["max_norm"] / norm).clamp(max=1.0)
    return {"norm": norm.reshape(1), "grads": [(g.float() * coef).to(g.dtype) for g in state["grads"]]}


def _own(state):
    from paper_2012_11346_gb300 import slim

    case = state["case"]
    if case["op"] == "vocab_loss":
        x, w, targets = state["x"], state["w"], state["targets"]
        loss, lse, total = slim.vocab_loss_forward(x, w, targets, ignore_index=IGNORE)
        out = {"loss": loss, "lse": lse, "total": total}
        if case["pass_"] == "step":
            count = total[1:] if case["weights"] == "mean" else None
            out["dx"], out["dw"] = slim.vocab_loss_backward(x, w, targets, lse, state["dloss"], count=count,
                                                            ignore_index=IGNORE)
        return out
    if case["op"] == "embed":
        if case["pass_"] == "forward":
            return slim.embed_forward(state["ids"], state["rows"], scale=state["scale"])
        return slim.embed_backward(state["ids"], state["rows"], case["V"], scale=state["scale"])
    norm = slim.clip_grad_norm(state["grads"], state["max_norm"], out=state["out"])
    return {"norm": norm, "grads": state["out"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    if case["op"] == "vocab_loss":
        N, D, V, es = case["N"], case["D"], case["V"], SIZE[case["dtype"]]
        step = case["pass_"] == "step"
        # x and w read; targets read, losses and log-sums written; a step writes both gradients
        return {"bytes": (2 if step else 1) * (N + V) * D * es + 16 * N, "flops": (6 if step else 2) * N * D * V}
    if case["op"] == "embed":
        N, D, V, es = case["N"], case["D"], case["V"], SIZE[case["dtype"]]
        if case["pass_"] == "forward":
            # expected number of different rows among N draws of rank = V u^3
            rows = sum(1.0 - math.exp(-N * (((r + 64) / V) ** (1 / 3) - (r / V) ** (1 / 3)) / 64) for r in range(0, V, 64)) * 64
            return {"bytes": int(8 * N + (N + min(N, V, rows)) * D * es), "flops": N * D}
        return {"bytes": 8 * N + (N + V) * D * es, "flops": 2 * N * D}
    held = sum(n * SIZE[t] for n, t in zip(_clip_sizes(case), _clip_dtypes(case)))
    return {"bytes": 2 * held, "flops": 3 * sum(_clip_sizes(case))}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "vocab_loss":
        N, V = case["N"], case["V"]
        x, w, t = state["x"].double(), state["w"].double(), state["targets"]
        live = (t != IGNORE).double()
        scale = state["dloss"].double() / (live.sum().clamp(min=1.0) if case["weights"] == "mean" else 1.0) * live
        loss, lse = torch.zeros(2, N, dtype=torch.float64, device="cuda")
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
        for a in range(0, N, 4096):  # rows in pieces: the 64-bit logits of all of them need not fit at once
            e = min(a + 4096, N)
            z = torch.einsum("nd,vd->nv", x[a:e], w)
            lse[a:e] = torch.logsumexp(z, 1)
            onehot = torch.arange(V, device="cuda")[None, :] == t[a:e, None]
            loss[a:e] = live[a:e] * (lse[a:e] - torch.where(onehot, z, 0.0).sum(1))
            if case["pass_"] == "step":
                g = (torch.exp(z - lse[a:e, None]) - onehot.double()) * scale[a:e, None]
                dx[a:e] = torch.einsum("nv,vd->nd", g, w)
                dw += torch.einsum("nv,nd->vd", g, x[a:e])
        out = {"loss": loss, "lse": lse, "total": torch.stack([loss.sum(), live.sum()])}
        return {**out, "dx": dx, "dw": dw} if case["pass_"] == "step" else out
    if case["op"] == "embed":
        ids, rows = state["ids"], state["rows"].double()
        good = torch.nonzero((ids >= 0) & (ids < case["V"]))[:, 0]
        if case["pass_"] == "forward":
            out = torch.zeros(case["N"], case["D"], dtype=torch.float64, device="cuda")
            out[good] = state["scale"] * rows[ids[good]]
            return out
        out = torch.zeros(case["V"], case["D"], dtype=torch.float64, device="cuda")
        return out.index_put_((ids[good],), state["scale"] * rows[good], accumulate=True)
    flat = [g.double() for g in state["grads"]]
    norm = math.sqrt(sum(float((g * g).sum()) for g in flat))
    factor = 1.0 if norm <= state["max_norm"] else state["max_norm"] / norm
    return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": [g * factor for g in flat]}
