"""Trains a small language model end to end with libslim: embedding lookup, a
stack of sliced Performer layers, the vocabulary loss, and one clipped update of
the tied table and the layers' features.

    python examples/language_model.py [--steps 40] [--vocab 4000] [--dtype bf16]

No step keeps anything of size tokens x layers: the stack recomputes its slices
and rolls its states back.  The loss recomputes its logits piece by piece and
holds one piece's gradient at a time; at the sizes below (8192 tokens, 4000 words)
the whole vocabulary is one piece.  --dtype sets the type at the two ends of the model; the
stack runs in fp32 (its bf16 kernels carry no residual of the rolled-back state,
and after some steps of training a sequence's first rows get gradients thousands
of times too large).  The data is synthetic: every symbol is followed by one
fixed other symbol most of the time, so the loss has somewhere to fall.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2012_11346_gb300 import slim  # noqa: E402

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def batch(gen, follow, B, L):
    """B sequences of L symbols and the symbol after each; the last symbol of a
    sequence is padding in the input and has no target."""
    V = follow.numel()
    seq = torch.empty(B, L + 1, dtype=torch.long, device=follow.device)
    seq[:, 0] = torch.randint(0, V, (B,), generator=gen, device=follow.device)
    other = torch.randint(0, V, (B, L + 1), generator=gen, device=follow.device)
    keep = torch.rand(B, L + 1, generator=gen, device=follow.device) < 0.9
    for t in range(L):
        seq[:, t + 1] = torch.where(keep[:, t], follow[seq[:, t]], other[:, t])
    ids, targets = seq[:, :-1].clone(), seq[:, 1:].clone()
    ids[:, -1], targets[:, -1] = -1, -100
    return ids, targets


class LanguageModel:
    """ids [B, L] -> embedding -> heads -> `layers` residual Performer layers ->
    rows -> loss against the embedding table itself (tied weights)."""

    def __init__(self, vocab, heads=4, d=64, features=128, layers=2, C=256, dtype="bf16", seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.d, self.C = heads, d, C
        self.dtype = DTYPES[dtype]
        D = heads * d
        # fp32 masters; the ends of the model read a `dtype` copy of the table
        self.table = torch.randn(vocab, D, generator=gen, device="cuda") / math.sqrt(D)
        self.omegas = torch.randn(layers, features, d, generator=gen, device="cuda")
        self.scale = math.sqrt(D)

    def to_heads(self, rows, B, L):
        return rows.view(B, L, self.heads, self.d).transpose(1, 2).contiguous()

    def to_rows(self, heads):
        B, H, L, d = heads.shape
        return heads.transpose(1, 2).reshape(B, L, H * d).contiguous()

    def step(self, ids, targets, lr, max_norm):
        """One training step; returns (mean loss, gradient norm) on the device."""
        B, L = ids.shape
        table = self.table.to(self.dtype)
        x = self.to_heads(slim.embed_forward(ids, table, self.scale).float(), B, L)
        y, S, z, S_lo, z_lo = slim.stack_forward(x, self.omegas, self.C)
        rows = self.to_rows(y).to(self.dtype)
        _, lse, total = slim.vocab_loss_forward(rows, table, targets)
        one = torch.ones(1, device=rows.device)
        drows, dtable = slim.vocab_loss_backward(rows, table, targets, lse, one, count=total[1:])
        dx, domegas = slim.stack_backward(x, self.omegas, self.to_heads(drows.float(), B, L), S,
                                          z, self.C, S_lo=S_lo, z_lo=z_lo)
        # the table's second gradient, from the lookup, is added to the first
        slim.embed_backward(ids, self.to_rows(dx).to(self.dtype), table.shape[0], self.scale,
                            dtable=dtable)
        norm = slim.clip_grad_norm([dtable, domegas], max_norm)
        self.table.sub_(dtable.float(), alpha=lr)
        self.omegas.sub_(domegas, alpha=lr)
        return total[0] / total[1], norm


def train(steps=40, vocab=4000, B=8, L=1024, lr=4.0, max_norm=1.0, dtype="bf16", seed=0, log=print):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = LanguageModel(vocab, dtype=dtype, seed=seed + 1)
    follow = torch.randperm(vocab, generator=gen, device="cuda")
    losses = []
    for i in range(steps):
        ids, targets = batch(gen, follow, B, L)
        loss, norm = model.step(ids, targets, lr, max_norm)
        losses.append(loss.item())
        if log and (i % 5 == 0 or i == steps - 1):
            log(f"step {i:3d}  loss {losses[-1]:.4f}  gradient norm {norm.item():.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--vocab", type=int, default=4000)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--length", type=int, default=1024)
    ap.add_argument("--lr", type=float, default=4.0)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dtype", choices=DTYPES, default="bf16")
    a = ap.parse_args()
    train(a.steps, a.vocab, a.batch, a.length, a.lr, a.max_norm, a.dtype)
